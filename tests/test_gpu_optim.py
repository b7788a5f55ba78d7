"""Gradient norm and AdamW step on the GPU against the 64-bit definitions of tests/update_ref.py."""
import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api, synth
from tests import gpu_util as G
from tests import update_ref as R
from tests.test_gpu_logits import to_bits, to_f64

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, b1=0.9, b2=0.97, eps=1e-8)


class Tensor:
    """One entry of a table in guarded buffers, and its fp64 values."""

    def __init__(self, rng, n, param="bf16", grad="bf16", state=32, master=False, wd=0.1, shift=0, fresh=False, size=1e-3):
        self.n, self.param, self.grad, self.state, self.wd = n, param, grad, state, wd
        w = (rng.standard_normal(n) * 0.02).astype(np.float32)
        self.p = to_bits(w, param)
        self.g = to_bits(rng.standard_normal(n) * size * np.exp(rng.standard_normal(n)), grad)
        self.master = w if master else None
        blocks = -(-n // 64)
        m, v = (rng.standard_normal(n) * size * 0.3).astype(np.float32), (rng.standard_normal(n) ** 2 * size ** 2).astype(np.float32)
        if fresh:
            m[:] = v[:] = 0
        if state == 8:
            self.ms, ma = R.block_scales(m.astype(np.float64))
            self.vs, va = R.block_scales(np.sqrt(v.astype(np.float64)))
            self.ms, self.vs = self.ms.astype(np.float32), self.vs.astype(np.float32)
            if fresh:
                self.ms[:] = self.vs[:] = 0
            q = lambda x, s: torch.tensor(x / np.repeat(np.where(s > 0, s, 1), 64)[:n], dtype=torch.float32).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            self.m, self.v = q(m, self.ms), q(np.sqrt(v), self.vs)
        else:
            self.m, self.v, self.ms, self.vs = m, v, None, None
        self.buf = {}
        for k in ("p", "g", "m", "v", "master", "ms", "vs"):
            a = getattr(self, k)
            if a is None:
                continue
            b = G.Guarded(a.nbytes + shift * a.itemsize)
            if n:
                b.view[shift * a.itemsize:] = torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).copy()).cuda()
            self.buf[k] = (b, shift * a.itemsize, a.dtype, a.shape)

    def get(self, k):
        b, off, dt, shape = self.buf[k]
        return b.numpy(np.uint8, (b.nbytes,))[off:].copy().view(dt).reshape(shape)

    def ptr(self, k):
        return self.buf[k][0].ptr() + self.buf[k][1] if k in self.buf else None

    def entry(self, first):
        kind = {"bf16": api.BF16, "f32": api.F32}
        return api.HiloreParam(self.ptr("p"), self.ptr("master"), self.ptr("g"), self.ptr("m"), self.ptr("v"), self.ptr("ms"),
                               self.ptr("vs"), self.n, first, kind[self.param], kind[self.grad],
                               api.STATE_E4M3FN if self.state == 8 else api.STATE_F32, self.wd)

    def moments(self):
        """fp64 moments that the state stands for."""
        if self.state == 8:
            return R.decode(self.m, self.ms), R.decode(self.v, self.vs) ** 2
        return self.m.astype(np.float64), self.v.astype(np.float64)

    def check(self, t, scale=1.0, **hyper):
        h = dict(HYPER, **hyper)
        p0 = self.master.astype(np.float64) if self.master is not None else to_f64(self.p)
        m0, v0 = self.moments()
        wd = float(np.float32(self.wd))
        p, m, v, ep, em, ev = R.adamw(p0, to_f64(self.g), m0, v0, t=t, wd=wd, scale=float(np.float32(scale)), **h)
        got = to_f64(self.get("p"))
        if self.master is not None:
            ms = self.get("master").astype(np.float64)
            assert (np.abs(ms - p) <= ep).all(), np.max(np.abs(ms - p) / ep)
            assert np.array_equal(self.get("p"), to_bits(self.get("master"), "bf16"))
        else:
            tol = ep + (R.BF16_HALF * (np.abs(p) + ep) if self.param == "bf16" else 0.0)
            assert (np.abs(got - p) <= tol).all(), np.max(np.abs(got - p) / np.maximum(tol, 1e-300))
        assert np.array_equal(self.get("g"), self.g)
        if self.state == 32:
            assert (np.abs(self.get("m") - m) <= em + 1e-45).all() and (np.abs(self.get("v") - v) <= ev + 1e-45).all()
            return
        for x, e, codes, scales, root in ((m, em, self.get("m"), self.get("ms"), False), (np.sqrt(v), 5 * R.U * np.sqrt(v), self.get("v"), self.get("vs"), True)):
            want, tiny = R.block_scales(x)
            top = np.repeat(want, 64)[:self.n]
            assert (np.abs(scales - want) <= 8 * R.U * want + np.maximum.reduceat(e, np.arange(0, self.n, 64)) / 448).all()
            q = x / top
            r = R.e4m3_round(q)
            if root:
                r = np.where((q > 0) & ~np.repeat(tiny, 64)[:self.n], np.maximum(r, 2.0 ** -9), r)
            differs = R.E4M3[codes] != r
            near = R.tie_distance(q) <= 1e-4 + e / top * 2.0 ** 9                   # rounding points move by the fp32 errors
            assert not (differs & ~near).any(), np.argwhere(differs & ~near)[:5]


def table(tensors):
    arr = (api.HiloreParam * len(tensors))()
    first = 0
    for i, t in enumerate(tensors):
        arr[i] = t.entry(first)
        first += -(-t.n // api.PARAM_TILE)
    return torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).cuda(), arr


def step(tensors, t=3, scale=None, **k):
    dev, host = table(tensors)
    h = dict(HYPER, **k)
    api.hilore_adamw_step(dev, host, len(tensors), h["lr"], None, h["b1"], h["b2"], h["eps"], t, None, scale)
    torch.cuda.synchronize()


KINDS = [("bf16", "bf16", 32, False), ("bf16", "bf16", 32, True), ("f32", "f32", 32, False), ("f32", "bf16", 32, False), ("bf16", "f32", 32, True),
         ("bf16", "bf16", 8, False), ("bf16", "f32", 8, True), ("f32", "f32", 8, False), ("f32", "bf16", 8, False)]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(map(str, k)))
@pytest.mark.parametrize("n", [1, 7, 8, 16, 63, 64, 65, 511, 512, 513, 1024, 1025, 5000])
def test_step_of_one_tensor(n, kind):
    rng = np.random.default_rng(n)
    x = Tensor(rng, n, *kind)
    step([x])
    x.check(3)


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(map(str, k)))
@pytest.mark.parametrize("shift", [1, 4, 8, 17])
def test_step_of_a_tensor_at_any_address(shift, kind):
    x = Tensor(np.random.default_rng(shift), 1300, *kind, shift=shift)
    step([x])
    x.check(3)


def test_table_of_many_tensors_of_all_kinds():
    rng = np.random.default_rng(11)
    sizes = [0, 1, 3000, 0, 0, 64, 2048, 17, 1024, 999, 100000, 0] + list(rng.integers(1, 400, 1500))
    xs = [Tensor(rng, int(n), *KINDS[i % len(KINDS)], wd=0.01 * (i % 3), shift=i % 5 if i % 7 == 0 else 0) for i, n in enumerate(sizes)]
    step(xs, t=1, scale=torch.tensor([0.37], device="cuda"))
    for x in xs:
        if x.n:
            x.check(1, scale=0.37)


@pytest.mark.parametrize("n_tensors", [1, 2, 31, 32, 33, 1023, 1024, 1025, 1100])
def test_every_tile_finds_its_tensor(n_tensors):
    """Equal tensors of two tiles: the update of a constant gradient is the same everywhere."""
    n = 1500
    p = torch.zeros(n_tensors, n, device="cuda")
    g = torch.ones(n_tensors, n, device="cuda") * torch.arange(1, n_tensors + 1, device="cuda")[:, None]
    m, v = torch.zeros_like(p), torch.zeros_like(p)
    dev, host = api.make_param_table([dict(p=p[i], g=g[i], m=m[i], v=v[i]) for i in range(n_tensors)])
    api.hilore_adamw_step(dev, host, n_tensors, 1.0, None, 0.5, 0.5, 0.0, 1, None, None)
    assert torch.equal(m, g * 0.5) and torch.equal(v, g * g * 0.5)
    assert ((p + 1).abs() < 1e-6).all()
    norm = torch.zeros(1, device="cuda")
    ws = torch.zeros(api.hilore_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")
    api.hilore_grad_norm(dev, host, n_tensors, 1.0, norm, None, ws, ws.numel())
    assert float(norm) == pytest.approx(float(g.double().norm()), rel=1e-6)


@pytest.mark.parametrize("state", [32, 8])
def test_first_step_from_zero_states(state):
    rng = np.random.default_rng(2)
    x = Tensor(rng, 777, "bf16", "bf16", state, True, fresh=True)
    step([x], t=1)
    x.check(1)


def test_eight_bit_states_special_values():
    """Blocks of zeros, of values too small to be scaled, a wide block (no positive root becomes zero), Inf and NaN."""
    rng = np.random.default_rng(8)
    x = Tensor(rng, 64 * 6, "f32", "f32", 8, fresh=True, wd=0.0)
    g = np.zeros((6, 64), np.float32)
    g[1] = 1e-37
    g[2] = 10.0 ** -np.linspace(0, 12, 64)
    g[3], g[3, 5] = 1.0, np.inf
    g[4], g[4, 9] = 1.0, np.nan
    g[5] = rng.standard_normal(64)
    x.g = g.reshape(-1)
    b, off, _, _ = x.buf["g"]
    b.view[off:] = torch.from_numpy(x.g.view(np.uint8).copy()).cuda()
    step([x], t=1, eps=1e-8)
    m, v = R.decode(x.get("m"), x.get("ms")).reshape(6, 64), R.decode(x.get("v"), x.get("vs")).reshape(6, 64)
    p, p0 = x.get("p").reshape(6, 64), x.p.reshape(6, 64)
    assert not m[0].any() and not v[0].any() and x.get("ms")[0] == 1 and x.get("vs")[0] == 1 and np.array_equal(p[0], p0[0])
    assert not m[1].any() and not v[1].any() and x.get("vs")[1] == 1 and np.allclose(p[1], p0[1], atol=1e-9)
    assert (v[2] > 0).all() and np.allclose(v[2, :20], np.sqrt(0.03) * g[2, :20], rtol=0.07)
    for row, at in ((3, 5), (4, 9)):
        others = np.arange(64) != at
        assert np.allclose(m[row, others], 0.1, rtol=1e-3) and np.allclose(v[row, others], np.sqrt(0.03), rtol=1e-3)
    assert m[3, 5] == pytest.approx(0.1, rel=1e-3) and v[3, 5] == pytest.approx(np.sqrt(0.03), rel=1e-3)      # Inf saturates
    assert np.isnan(m[4, 9]) and np.isnan(v[4, 9]) and np.isnan(p[4, 9])
    assert np.isfinite(np.delete(p.reshape(-1), [3 * 64 + 5, 4 * 64 + 9])).all()


def test_codes_are_those_of_the_codec():
    """hilore_recover decodes the states: value times scale, rounded to bf16."""
    x = Tensor(np.random.default_rng(3), 4096, "bf16", "bf16", 8)
    step([x])
    codes, scales = x.get("m").reshape(1, -1), x.get("ms").reshape(1, -1)
    got = G.recover(codes, scales, api.FMT_E4M3FN_BLK)
    want = synth._to_bf16_bits((R.E4M3[codes].astype(np.float32) * np.repeat(scales, 64, 1)).astype(np.float32))
    assert np.array_equal(got, want)


def test_many_steps_with_eight_bit_states_follow_the_exact_optimizer():
    """A quadratic bowl: 300 steps with 8-bit states end where 300 exact steps end."""
    rng = np.random.default_rng(5)
    n = 4096
    c = torch.tensor(rng.standard_normal(n), dtype=torch.float32, device="cuda")
    a = torch.tensor(np.exp(rng.standard_normal(n)), dtype=torch.float32, device="cuda")
    end = {}
    for state in (32, 8):
        p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        e = dict(p=p, g=g, m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
        if state == 8:
            e = dict(p=p, g=g, m=torch.zeros(n, dtype=torch.uint8, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                     m_scale=torch.zeros(64, device="cuda"), v_scale=torch.zeros(64, device="cuda"))
        dev, host = api.make_param_table([e])
        for t in range(1, 301):
            g.copy_(a * (p - c))
            api.hilore_adamw_step(dev, host, 1, 0.05 * (1 - t / 301), None, 0.9, 0.99, 1e-8, t, None, None)
        end[state] = float((a * (p - c) ** 2).sum() / (a * c ** 2).sum())
    assert end[32] < 1e-3 and end[8] < 1e-2, end


def test_norm_and_clip():
    rng = np.random.default_rng(7)
    sizes = [1, 0, 70000, 999, 64, 1025, 300001]
    xs = [Tensor(rng, n, "bf16", ("bf16", "f32")[i % 2], shift=i % 3) for i, n in enumerate(sizes)]
    want = np.sqrt(sum((to_f64(x.g) ** 2).sum() for x in xs))
    nws = api.hilore_grad_norm_workspace_bytes()
    for max_norm in (0.0, 1e-3, 1e9, float("inf")):
        dev, host = table(xs)
        ws, norm, scale = G.Guarded(nws), G.Guarded(4), G.Guarded(4)
        api.hilore_grad_norm(dev, host, len(xs), max_norm, norm.ptr(), scale.ptr(), ws.ptr(), nws)
        ws.numpy(np.uint8, (nws,))
        assert norm.numpy(np.float32, (1,))[0] == pytest.approx(want, rel=32 * R.U)           # 32 additions in fp32, the rest in fp64
        assert scale.numpy(np.float32, (1,))[0] == pytest.approx(min(1.0, max_norm / (want + 1e-6)), rel=33 * R.U, abs=0)
    dev, host = table([Tensor(rng, 0)])
    norm, scale = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.zeros(nws, dtype=torch.uint8, device="cuda")
    api.hilore_grad_norm(dev, host, 1, 1.0, norm, scale, ws, nws)
    assert float(norm) == 0 and float(scale) == 1


def test_norm_of_extreme_and_non_finite_gradients_and_the_step_it_skips():
    big = torch.zeros(5000, device="cuda")
    big[17], big[4000] = 3e25, 4e25                           # squares beyond fp32
    p, m, v = (torch.ones(5000, device="cuda") for _ in range(3))
    dev, host = api.make_param_table([dict(p=p, g=big, m=m, v=v)])
    nws = api.hilore_grad_norm_workspace_bytes()
    ws = torch.zeros(nws, dtype=torch.uint8, device="cuda")
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    api.hilore_grad_norm(dev, host, 1, 1.0, norm, scale, ws, nws)
    assert float(norm) == pytest.approx(5e25, rel=1e-6) and float(scale) == pytest.approx(2e-26, rel=1e-6)
    for bad in (float("inf"), float("nan")):
        big[3] = bad
        api.hilore_grad_norm(dev, host, 1, 1.0, norm, scale, ws, nws)
        assert not np.isfinite(float(norm)) and np.isnan(float(scale))
        api.hilore_adamw_step(dev, host, 1, 0.1, None, 0.9, 0.99, 1e-8, 1, None, scale)
        assert bool((p == 1).all() and (m == 1).all() and (v == 1).all())


def test_step_count_and_rate_on_the_device_in_a_graph():
    """One captured step replayed over a schedule equals the steps called one by one."""
    rng = np.random.default_rng(1)
    w, g = torch.tensor(rng.standard_normal(3000), dtype=torch.float32), torch.tensor(rng.standard_normal(3000), dtype=torch.float32).cuda()
    rates = [1e-2, 5e-3, 2e-3]
    a = dict(p=w.cuda(), g=g, m=torch.zeros(3000, device="cuda"), v=torch.zeros(3000, device="cuda"))
    b = dict(p=w.cuda(), g=g, m=torch.zeros(3000, device="cuda"), v=torch.zeros(3000, device="cuda"))
    dev, host = api.make_param_table([a])
    for t, lr in enumerate(rates, 1):
        api.hilore_adamw_step(dev, host, 1, lr, None, 0.9, 0.95, 1e-8, t, None, None)
    dev2, host2 = api.make_param_table([b])
    lr, k = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.hilore_adamw_step(dev2, host2, 1, 0.0, lr, 0.9, 0.95, 1e-8, 0, k, None)
    for t, rate in enumerate(rates, 1):
        lr.fill_(rate)
        k.fill_(t)
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a["m"], b["m"]) and torch.equal(a["v"], b["v"])
    # the corrections are fp64 on both sides and rounded once; the rate is rounded to fp32 on both
    assert torch.allclose(a["p"], b["p"], rtol=4 * R.U, atol=1e-8)


def test_a_tensor_beyond_2_31_elements():
    """2^31 + 777 elements with 8-bit states: the ends of the tensor against the definition."""
    n = (1 << 31) + 777
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(-(-n // 64), device="cuda"), torch.zeros(-(-n // 64), device="cuda")
    rng = np.random.default_rng(0)
    at = [0, (1 << 31) - 512, n - 777]
    vals = [torch.tensor(rng.standard_normal(512)).bfloat16().cuda() for _ in at]
    for a, x in zip(at, vals):
        g[a:a + 512] = x
    dev, host = api.make_param_table([dict(p=p, g=g, m=m, v=v, m_scale=ms, v_scale=vs)])
    api.hilore_adamw_step(dev, host, 1, 0.5, None, 0.9, 0.99, 1e-8, 1, None, None)
    norm = torch.zeros(1, device="cuda")
    ws = torch.zeros(api.hilore_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")
    api.hilore_grad_norm(dev, host, 1, 1.0, norm, None, ws, ws.numel())
    assert float(norm) == pytest.approx(float(sum((x.double() ** 2).sum() for x in vals).sqrt()), rel=1e-6)
    for a, x in zip(at, vals):
        q = p[a:a + 512].float()
        assert torch.allclose(q, -0.5 * torch.sign(x.float()), rtol=2.0 ** -8)               # the first step is lr * sign(g)
    assert int((p != 0).sum()) == sum(int((x != 0).sum()) for x in vals)


@pytest.mark.parametrize("shift", [0, 1], ids=["vectors", "elements"])
def test_roots_of_eight_bit_states_are_rounded_once(shift):
    """One gradient per block, beta2 = 1/2, no state before: v = fl(fl(g / 2) g) and v_scale = fl(root / 448).  A root of relative
    error 2^-22.9 (the approximation's bound) after one Newton step is off by 2^-43 before it is rounded."""
    blocks = 1 << 18
    n = blocks * 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = torch.zeros(n, device="cuda")
    some = torch.exp2(torch.rand(blocks, generator=gen, device="cuda") * 2 - 5) * torch.exp2(torch.randint(-40, 20, (blocks,), generator=gen, device="cuda").float())
    at = torch.arange(blocks, device="cuda") * 64 + torch.arange(blocks, device="cuda") % 64
    g[at] = some
    p = torch.zeros(n + shift, device="cuda")[shift:]              # off the vectors' alignment: element by element
    code = lambda: torch.zeros(n, dtype=torch.uint8, device="cuda")
    e = dict(p=p, g=g, m=code(), v=code(), m_scale=torch.zeros(blocks, device="cuda"), v_scale=torch.zeros(blocks, device="cuda"))
    dev, host = api.make_param_table([e])
    api.hilore_adamw_step(dev, host, 1, 1.0, None, 0.5, 0.5, 1e-8, 1, None, None)
    x = some.cpu().numpy()
    v = (x * np.float32(0.5) * x).astype(np.float64)                                 # both products rounded to fp32
    exact = np.sqrt(v)
    ulp = np.spacing(exact.astype(np.float32)).astype(np.float64)
    lo, hi = exact - ulp / 2 - exact * 2.0 ** -43, exact + ulp / 2 + exact * 2.0 ** -43
    c = np.float64(np.float32(1 / 448))
    got = e["v_scale"].cpu().numpy()
    assert ((got >= (lo * c).astype(np.float32)) & (got <= (hi * c).astype(np.float32))).all()
    assert bool((e["v"][at] == 0x7E).all()) and int((e["v"] != 0).sum()) == blocks   # 448, and nothing else


@pytest.mark.parametrize("shift", [0, 1], ids=["vectors", "elements"])
@pytest.mark.parametrize("state", [32, 8])
def test_moments_round_every_operation(state, shift):
    """Moments of fp32 states, and the scales of 8-bit ones, have the bits of operation-by-operation evaluation in fp32."""
    f = np.float32
    rng = np.random.default_rng(1)
    x = Tensor(rng, 64 * 3000, "f32", "f32", state, shift=shift)
    m0 = x.m if state == 32 else R.E4M3[x.m].astype(f) * np.repeat(x.ms, 64)
    v0 = x.v if state == 32 else (R.E4M3[x.v].astype(f) * np.repeat(x.vs, 64)) ** 2
    b1, b2, a1, a2 = f(HYPER["b1"]), f(HYPER["b2"]), f(1 - HYPER["b1"]), f(1 - HYPER["b2"])
    m, v = b1 * m0 + a1 * x.g, b2 * v0 + a2 * x.g * x.g
    assert m.dtype == v.dtype == f
    step([x])
    if state == 32:
        assert np.array_equal(x.get("m"), m) and np.array_equal(x.get("v"), v)
    else:
        assert np.array_equal(x.get("ms"), np.abs(m).reshape(-1, 64).max(1) * f(1 / 448))
