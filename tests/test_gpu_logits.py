"""Logit rules, token log-probabilities and their gradients on the GPU against the 64-bit definitions of
tests/update_ref.py, within bounds that count the roundings of the fp32 evaluation."""
import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api, synth
from tests import gpu_util as G
from tests import update_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": (api.BF16, np.uint16), "f32": (api.F32, np.float32)}


def to_bits(x, dtype):
    return synth._to_bf16_bits(x.astype(np.float32)) if dtype == "bf16" else x.astype(np.float32)


def to_f64(bits):
    if bits.dtype == np.uint16:
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return bits.astype(np.float64)


def make_rules(rng, rows, V, *, history=0, bias=0, grammar=None, temperature=True, prefix=False):
    r = {}
    if temperature:
        r["temperature"] = rng.uniform(0.5, 1.5, rows)
    if history is not None and history >= 0:
        length = np.full(rows, history) if prefix else rng.integers(0, history + 1, rows)
        if not prefix:
            length[0] = history
            end = np.cumsum(length)
            r["hist_begin"], r["hist_end"] = end - length, end
            r["resp_begin"] = end - rng.integers(0, length + 1)
            n = int(end[-1])
        else:
            r["hist_begin"], r["hist_end"] = np.zeros(rows, np.int64), np.arange(rows) % (history + 1)
            r["resp_begin"] = np.minimum(r["hist_end"], history // 3)
            n = history
        tok = (rng.random(n) ** 3 * V).astype(np.int32)
        tok[rng.random(n) < 0.02] = -1                      # padding and nonsense count nowhere
        tok[rng.random(n) < 0.02] = V + 3
        r["tokens"] = tok
        r["repetition"] = np.where(rng.random(rows) < 0.8, rng.uniform(0.7, 1.8, rows), 1.0)
        r["frequency"] = rng.uniform(-0.3, 0.6, rows)
        r["presence"] = rng.uniform(-0.3, 0.6, rows)
    if bias:
        count = rng.integers(0, bias + 1, rows)
        r["bias_offsets"] = np.concatenate([[0], np.cumsum(count)])
        n = int(count.sum())
        r["bias_tokens"] = rng.integers(-1, V + 1, n).astype(np.int32)
        r["bias_values"] = rng.normal(0, 4, n)
        for i in range(rows):                               # a token named twice
            a, b = r["bias_offsets"][i], r["bias_offsets"][i + 1]
            if b - a >= 2:
                r["bias_tokens"][b - 1] = r["bias_tokens"][a]
    if grammar:
        words = (V + 31) // 32
        n = max(1, rows - 1) if grammar == "indexed" else rows
        bits = rng.integers(0, 2**32, (n, words + 2), dtype=np.uint64).astype(np.uint32)
        bits[0] = 0                                         # nothing allowed
        if n > 1:
            bits[1] = 0
            bits[1, (V - 1) // 32] = np.uint32(1) << np.uint32((V - 1) % 32)      # the last token alone
        if n > 2:
            bits[2] &= np.uint32(0xFFFF)                    # halves of words
        r["allow"] = bits.view(np.int32)
        if grammar == "indexed":
            r["allow_row"] = rng.integers(-1, n + 1, rows).astype(np.int32)       # -1 and n: no mask
    for k in ("temperature", "repetition", "frequency", "presence", "bias_values"):
        if k in r:
            r[k] = np.asarray(r[k], np.float32)
    return r


def device_rules(r):
    kinds = dict(hist_begin=np.int64, resp_begin=np.int64, hist_end=np.int64, bias_offsets=np.int64)
    return api.make_logit_rules(**{k: G.dev(v.astype(kinds[k]) if k in kinds else v) for k, v in r.items()})


def logits(rng, rows, V, ld, dtype, spread=3.0):
    x = to_bits(rng.standard_normal((rows, ld)) * spread, dtype)
    x[:, V:] = to_bits(np.full(1, np.nan), dtype)[0]        # what lies between rows is never used
    return x


def placed(x, shift):
    """The array on the device with its first element `shift` elements behind a 256-byte boundary."""
    t = torch.zeros(x.size + 64, dtype=torch.int16 if x.dtype == np.uint16 else torch.float32, device="cuda")
    t[shift:shift + x.size] = G.dev(x).reshape(-1)
    return t[shift:shift + x.size]


def apply(x, V, r, dtype, ld_out, shift=0, backward=None):
    kind, npt = DT[dtype]
    rows, ld = x.shape
    out = G.Guarded((rows * ld_out + shift) * x.itemsize)
    dst = out.ptr() + shift * x.itemsize
    h = device_rules(r)
    if backward is None:
        api.hilore_logits_apply(placed(x, shift), kind, rows, V, ld, h, dst, ld_out)
    else:
        api.hilore_logits_apply_backward(placed(x, shift), kind, rows, V, ld, h, placed(backward, 3), backward.shape[1], dst, ld_out)
    raw = out.numpy(npt, (rows * ld_out + shift,))
    body = raw[shift:].reshape(rows, ld_out)
    untouched = np.frombuffer(bytes([G.CANARY]) * x.itemsize, npt)[0:1].view(np.uint8)
    assert (np.ascontiguousarray(body[:, V:]).view(np.uint8) == untouched[0]).all(), "wrote between the rows"
    return to_f64(np.ascontiguousarray(body[:, :V]))


def check(got, want, bound, dtype):
    tol = bound + (R.BF16_HALF * np.abs(want) * (1 + 1e-3) + 1e-40 if dtype == "bf16" else 2 * R.U * np.abs(want))
    with np.errstate(invalid="ignore"):
        ok = (got == want) | (np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want))
    bad = np.argwhere(~ok)
    assert ok.all(), (len(bad), bad[:5], got[~ok][:5], want[~ok][:5])


CASES = [  # rows, V, ld, shift, ld_out, history, bias, grammar, prefix
    (1, 1, 1, 0, 1, 0, 0, None, False),
    (1, 1, 3, 1, 2, 4, 1, "rows", False),
    (3, 2, 2, 0, 2, 5, 2, "rows", False),
    (3, 15, 16, 0, 16, 9, 0, None, False),
    (4, 16, 16, 0, 16, 9, 3, "rows", False),
    (4, 17, 17, 0, 17, 40, 3, "indexed", False),
    (5, 33, 40, 7, 35, 64, 0, "rows", False),
    (7, 1000, 1000, 0, 1000, 300, 20, None, True),
    (7, 1001, 1009, 5, 1001, 300, 20, "indexed", True),
    (5, 8191, 8191, 0, 8191, 1, 5, "rows", False),
    (5, 8192, 8192, 0, 8192, 2000, 5, None, False),
    (5, 8193, 8200, 0, 8193, 2000, 300, "rows", False),
    (9, 20011, 20011, 2, 20011, 5000, 40, "indexed", True),
    (2, 70001, 70016, 0, 70001, 90000, 500, "rows", False),
    (300, 257, 257, 0, 257, 100, 8, "rows", False),
    (3, 30011, 30011, 1, 30011, 3000, 1500, "indexed", False),      # bias lists too long to be kept beside the counts
    (4000, 301, 301, 0, 301, 500, 0, None, True),                   # blocks of rows: prefixes of one sequence, started anew ...
    (3700, 300, 305, 3, 300, 90, 3, "indexed", True),               # ... with bias lists and masks between
    (3600, 517, 517, 0, 520, 60, 0, None, False),                   # ... and histories that have nothing in common
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(v) for v in c[:5]))
def test_rules_forward_and_backward(case, dtype):
    rows, V, ld, shift, ld_out, history, bias, grammar, prefix = case
    rng = np.random.default_rng(rows * 1000003 + V)
    x = logits(rng, rows, V, ld, dtype)
    r = make_rules(rng, rows, V, history=history, bias=bias, grammar=grammar, prefix=prefix)
    ref = [R.rules_row(to_f64(x[i, :V]), r, i) for i in range(rows)]
    z, k, e = (np.stack([t[j] for t in ref]) for j in range(3))
    check(apply(x, V, r, dtype, ld_out, shift), z, e, dtype)
    dz = logits(rng, rows, V, ld_out + 2, dtype, 0.01)
    d = to_f64(dz[:, :V])
    check(apply(x, V, r, dtype, ld_out, shift, backward=dz), d * k, 4 * R.U * np.abs(d * k), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rules_in_place_and_without_any_rule(dtype):
    rng = np.random.default_rng(5)
    rows, V = 6, 9001
    kind, npt = DT[dtype]
    x = logits(rng, rows, V, V, dtype)
    r = make_rules(rng, rows, V, history=700, bias=9, grammar="indexed")
    want = apply(x, V, r, dtype, V)
    t = G.dev(x)
    api.hilore_logits_apply(t, kind, rows, V, V, device_rules(r), t, V)
    got = t.cpu().numpy().view(npt)
    assert np.array_equal(to_f64(got), want)                                        # the same bits
    assert np.array_equal(apply(x, V, {}, dtype, V), to_f64(x))                    # no rule: the logits themselves
    g = logits(rng, rows, V, V, dtype)
    want = apply(x, V, r, dtype, V, backward=g)
    t = G.dev(g)
    api.hilore_logits_apply_backward(G.dev(x), kind, rows, V, V, device_rules(r), t, V, t, V)
    assert np.array_equal(to_f64(t.cpu().numpy().view(npt)), want)


def test_rules_special_values():
    """Inf and NaN in masked places, a count that a byte does not hold, temperature 0, ranges outside the tokens."""
    V = 5000
    x = np.zeros((4, V), np.float32)
    x[:, 0], x[:, 1], x[:, 2], x[:, 3] = np.nan, np.inf, -np.inf, -3.4028235e38
    allow = np.full((4, 157), -1, np.int32)
    allow[1, 0] = ~0b1111                                                            # they are denied in row 1
    r = dict(tokens=np.full(70000, 77, np.int32), hist_begin=np.array([-5, 0, 10, 70000]), resp_begin=np.array([-9, 1, 70000, 0]),
             hist_end=np.array([70000, 1 << 40, 20, 0]), frequency=np.full(4, 0.5, np.float32), presence=np.full(4, 1.0, np.float32),
             repetition=np.full(4, 2.0, np.float32), temperature=np.array([0.0, -1.0, np.nan, 2.0], np.float32), allow=allow)
    z = apply(x, V, r, "f32", V)
    assert np.isnan(z[0, 0]) and z[0, 1] == np.inf and z[0, 2] == -np.inf and z[0, 3] == np.float32(-3.4028235e38)
    assert (z[1, :4] == -np.inf).all()
    assert z[0, 77] == -0.5 * 70000 - 1 and z[1, 77] == -0.5 * 69999 - 1 and z[2, 77] == 0 and z[3, 77] == 0
    assert not z[0, 78:].any()
    g = apply(x, V, r, "f32", V, backward=np.where(np.arange(V) < 4, np.nan, 1.0).astype(np.float32).reshape(1, V).repeat(4, 0))
    assert (g[1, :4] == 0).all() and np.isnan(g[0, :4]).all() and g[0, 77] == 2.0 and g[3, 77] == 0.5 and g[3, 78] == 0.5


def run_logp(x, V, r, targets, dtype, entropy=True, lse=True, shift=0):
    kind, _ = DT[dtype]
    rows, ld = x.shape
    out = [G.Guarded(rows * 4) for _ in range(3)]
    api.hilore_token_logp(placed(x, shift), kind, rows, V, ld, device_rules(r) if r is not None else None, G.dev(targets), out[0].ptr(),
                          out[1].ptr() if lse else None, out[2].ptr() if entropy else None)
    return [o.numpy(np.float32, (rows,)).astype(np.float64) for o in out]


def run_grad(x, V, r, targets, lse, omega, dtype, ld_out=None, shift=0):
    kind, npt = DT[dtype]
    rows, ld = x.shape
    ld_out = ld_out or V
    out = G.Guarded(rows * ld_out * x.itemsize)
    api.hilore_token_logp_backward(placed(x, shift), kind, rows, V, ld, device_rules(r) if r is not None else None, G.dev(targets),
                                   G.dev(lse.astype(np.float32)), G.dev(omega.astype(np.float32)), out.ptr(), ld_out)
    return to_f64(np.ascontiguousarray(out.numpy(npt, (rows, ld_out))[:, :V]))


@pytest.mark.parametrize("ruled", [False, True, "temperature"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(v) for v in c[:5]))
def test_logp_and_gradient(case, dtype, ruled):
    rows, V, ld, shift, ld_out, history, bias, grammar, prefix = case
    rng = np.random.default_rng(rows * 1000003 + V + 1)
    x = logits(rng, rows, V, ld, dtype)
    r = make_rules(rng, rows, V, history=history, bias=bias, grammar=grammar, prefix=prefix) if ruled is True else \
        make_rules(rng, rows, V, history=-1) if ruled else None
    targets = rng.integers(0, V, rows).astype(np.int32)
    targets[-1] = V - 1
    if rows > 2:
        targets[1], targets[2] = -1, V                      # slots without a token
    omega = rng.standard_normal(rows) / rows
    if rows > 4:
        omega[4] = 0.0
    omega = omega.astype(np.float32).astype(np.float64)
    got = run_logp(x, V, r, targets, dtype, shift=shift)
    lse = np.zeros(rows, np.float32)
    want, bounds, grads, gerr = [], [], [], []
    for i in range(rows):
        z, k, e = R.rules_row(to_f64(x[i, :V]), r or {}, i)
        want.append(R.logp_row(z, targets[i]))
        b = R.logp_bound(z, e, V)
        bounds.append(b)
        lse[i] = want[-1][1]
        grads.append(R.grad_row(z, k, targets[i], omega[i], want[-1][1]))
        gerr.append(R.grad_bound(z, e, k, omega[i], want[-1][1] if np.isfinite(want[-1][1]) else 0.0, R.U * abs(want[-1][1]) if np.isfinite(want[-1][1]) else 0.0))
    for name, a, j in (("logp", got[0], 0), ("lse", got[1], 1), ("entropy", got[2], 2)):
        for i in range(rows):
            w, tol = want[i][j], bounds[i][j] + 4 * R.U * abs(want[i][j]) if np.isfinite(want[i][j]) else 0.0
            assert a[i] == w or abs(a[i] - w) <= tol, (name, i, a[i], w, tol)
    plain = run_logp(x, V, r, targets, dtype, entropy=False, lse=False, shift=shift)
    assert all(a == w[0] or abs(a - w[0]) <= b[0] + 4 * R.U * abs(w[0]) for a, w, b in zip(plain[0], want, bounds))
    g = run_grad(x, V, r, targets, lse, omega, dtype, ld_out, shift)
    check(g, np.stack(grads), np.stack(gerr), dtype)


def test_gradient_is_the_difference_quotient_of_logp():
    """Central differences of the kernel's own fp32 logp, step 2^-4: truncation h^2/6 |f'''| <= 2^-8 / 6 * 1/4, rounding 2^-24-sized
    errors of logp (|logp| < 8: 2 * 4e-6 with the bound of the other tests) over 2 h."""
    rng = np.random.default_rng(0)
    V, h = 60, 2.0 ** -4
    x0 = rng.standard_normal((1, V)).astype(np.float32)
    r = make_rules(rng, 1, V, history=30, bias=4)
    t = np.array([7], np.int32)
    lse = run_logp(x0, V, r, t, "f32")[1]
    g = run_grad(x0, V, r, t, lse, np.ones(1), "f32")[0]
    rr = {k: np.repeat(v, 2 * V, 0) if k in ("temperature", "repetition", "frequency", "presence", "hist_begin", "resp_begin", "hist_end")
          else v for k, v in r.items()}
    n = int(r["bias_offsets"][1])
    rr["bias_tokens"], rr["bias_values"] = np.tile(r["bias_tokens"][:n], 2 * V), np.tile(r["bias_values"][:n], 2 * V)
    rr["bias_offsets"] = np.arange(2 * V + 1) * n
    x = np.repeat(x0, 2 * V, 0)
    for v in range(V):
        x[2 * v, v] += h
        x[2 * v + 1, v] -= h
    p = run_logp(x, V, rr, np.full(2 * V, 7, np.int32), "f32")[0]
    slope = R.rules_row(x0[0].astype(np.float64), r, 0)[1]
    for v in range(V):
        if abs(x0[0, v]) <= h:                               # the repetition penalty has a corner at zero
            continue
        q = (p[2 * v] - p[2 * v + 1]) / (2 * h)
        assert abs(q - g[v]) <= slope[v] ** 3 * h * h / 24 + 8e-6 / h, (v, q, g[v])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logp_special_rows(dtype):
    V = 3001
    low = -3.38e38 if dtype == "bf16" else -3.4028235e38
    x = np.full((8, V), -1.0)
    x[0] = -np.inf                                           # nothing to choose from
    x[1] = low                                               # masks of the type's lowest value ...
    x[1, 5:9] = 0.5                                          # ... around four tokens
    x[2] = low                                               # ... and nothing else: uniform by the formula
    x[3, 17] = np.nan
    x[4, 17] = np.inf
    x[5] = -np.inf
    x[5, 3000] = 2.0                                         # one token
    x[6, :3000] = -np.inf
    b = to_bits(x, dtype)
    t = np.array([4, 6, 4, 4, 4, 3000, 10, 0], np.int32)
    logp, lse, h = run_logp(b, V, None, t, dtype)
    assert logp[0] == -np.inf and lse[0] == -np.inf and h[0] == 0
    assert logp[1] == pytest.approx(-np.log(4), rel=1e-6) and h[1] == pytest.approx(np.log(4), rel=1e-6)
    assert logp[2] == pytest.approx(-np.log(V), rel=1e-6) and h[2] == pytest.approx(np.log(V), rel=1e-6)
    assert np.isnan([logp[3], lse[3], h[3]]).all()
    assert lse[4] == np.inf and logp[4] == -np.inf and np.isnan(h[4])
    assert logp[5] == 0 and lse[5] == 2 and h[5] == 0
    assert logp[6] == -np.inf and lse[6] == -1
    assert logp[7] == pytest.approx(-np.log(V), rel=1e-6)
    g = run_grad(b, V, None, t, lse, np.full(8, 0.5), dtype)
    assert not g[0].any() and not g[2].any()                 # an lse of the lowest value says nothing
    assert g[1, 6] == pytest.approx(0.375, rel=4e-3) and g[1, 5] == pytest.approx(-0.125, rel=4e-3) and not g[1, 9:].any()
    assert np.isnan(g[3]).all()
    assert not g[5, :3000].any() and abs(g[5, 3000]) < 1e-6
    # the same NaN and Inf where the grammar denies them change nothing
    allow = np.full((8, 94), -1, np.int32)
    allow[:, 0] = ~(1 << 17)
    lp, l2, h2 = run_logp(b, V, dict(allow=allow), t, dtype)
    for i in (3, 4):
        assert lp[i] == pytest.approx(-np.log(V - 1), rel=1e-6) and l2[i] == pytest.approx(np.log(V - 1) - 1, rel=1e-6)
    g = run_grad(b, V, dict(allow=allow), t, l2, np.full(8, 0.5), dtype)
    assert np.isfinite(g).all() and not g[:, 17].any()
    denied = np.full(8, 17, np.int32)
    lp, l2, _ = run_logp(b, V, dict(allow=allow), denied, dtype)
    assert (lp == -np.inf).all() and not run_grad(b, V, dict(allow=allow), denied, l2, np.ones(8), dtype).any()


def test_rows_of_a_cluster_and_of_one_cta_agree(monkeypatch):
    """The same rows with clusters allowed (few rows: up to eight CTAs each) and without."""
    rng = np.random.default_rng(9)
    V = 50001
    x = logits(rng, 5, V, V, "bf16")
    r = make_rules(rng, 5, V, history=3000, bias=10, grammar="indexed")
    t = rng.integers(0, V, 5).astype(np.int32)
    for rules in (None, r):
        a = run_logp(x, V, rules, t, "bf16")
        monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", "1")
        b = run_logp(x, V, rules, t, "bf16")
        monkeypatch.delenv("HILORE_DISABLE_CLUSTER_LAUNCH")
        c = run_logp(x, V, rules, t, "bf16")
        for p, q, s in zip(a, b, c):
            assert np.array_equal(p, s)                                      # the same call, the same bits
            same = (p == q) | (np.abs(p - q) <= 2e-5 + 2e-6 * np.abs(q))
            assert same.all(), (p, q)


def test_the_same_call_gives_the_same_bits():
    """Twenty calls over dense histories: sums do not depend on the order in which listed tokens were found."""
    rng = np.random.default_rng(12)
    rows, V = 24, 20011
    x = logits(rng, rows, V, V, "f32")
    r = make_rules(rng, rows, V, history=9000, bias=60, grammar="indexed")
    t = rng.integers(0, V, rows).astype(np.int32)
    first = run_logp(x, V, r, t, "f32")
    for _ in range(20):
        assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(run_logp(x, V, r, t, "f32"), first))


def test_gradient_in_place_and_on_another_stream():
    rng = np.random.default_rng(4)
    rows, V = 33, 12345
    x = logits(rng, rows, V, V, "bf16")
    r = make_rules(rng, rows, V, history=500, grammar="indexed", prefix=True)
    t = rng.integers(0, V, rows).astype(np.int32)
    _, lse, _ = run_logp(x, V, r, t, "bf16")
    omega = rng.standard_normal(rows)
    want = run_grad(x, V, r, t, lse, omega, "bf16")
    h, td, ld_, om = device_rules(r), G.dev(t), G.dev(lse.astype(np.float32)), G.dev(omega.astype(np.float32))
    xd = G.dev(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    api.hilore_token_logp_backward(xd, api.BF16, rows, V, V, h, td, ld_, om, xd, V, stream=side)
    side.synchronize()
    assert np.array_equal(to_f64(xd.cpu().numpy().view(np.uint16)), want)


def test_rows_beyond_32_bit_offsets():
    """Three rows 2^30 + 8 elements apart (6.4 GB) and a history that begins beyond 2^31 tokens."""
    rng = np.random.default_rng(6)
    ld, V, rows = (1 << 30) + 8, 4099, 3
    big = torch.empty(rows * ld, dtype=torch.int16, device="cuda")
    x = logits(rng, rows, V, V, "bf16")
    for i in range(rows):
        big[i * ld:i * ld + V] = G.dev(x[i])
    n = (1 << 31) + 500
    tokens = torch.empty(n, dtype=torch.int32, device="cuda")
    hist = rng.integers(0, V, 500).astype(np.int32)
    tokens[1 << 31:] = G.dev(hist)
    r = dict(repetition=np.full(rows, 1.5, np.float32), frequency=np.full(rows, 0.2, np.float32))
    span = [np.zeros(rows, np.int64), np.full(rows, 100, np.int64), np.full(rows, 500, np.int64)]
    h = api.make_logit_rules(tokens=tokens, hist_begin=G.dev(span[0] + (1 << 31)), resp_begin=G.dev(span[1] + (1 << 31)),
                             hist_end=G.dev(span[2] + (1 << 31)), **{k: G.dev(v) for k, v in r.items()})
    t = rng.integers(0, V, rows).astype(np.int32)
    logp, lse = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    api.hilore_token_logp(big, api.BF16, rows, V, ld, h, G.dev(t), logp, lse, None)
    ref = dict(r, tokens=hist, hist_begin=span[0], resp_begin=span[1], hist_end=span[2])
    for i in range(rows):
        z, k, e = R.rules_row(to_f64(x[i]), ref, i)
        w, b = R.logp_row(z, t[i]), R.logp_bound(z, e, V)
        assert abs(float(logp[i]) - w[0]) <= b[0] + 4 * R.U * abs(w[0])
    api.hilore_token_logp_backward(big, api.BF16, rows, V, ld, h, G.dev(t), lse, torch.ones(rows, device="cuda"), big, ld)
    for i in range(rows):
        z, k, e = R.rules_row(to_f64(x[i]), ref, i)
        l = float(lse[i])
        got = to_f64(big[i * ld:i * ld + V].cpu().numpy().view(np.uint16))
        check(got, R.grad_row(z, k, t[i], 1.0, l), R.grad_bound(z, e, k, 1.0, l, 0.0), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lists", [(9000, 60, False), (300, 1500, False), (5000, 0, True), (90000, 500, False), (0, 7, False)],
                         ids=lambda l: "-".join(map(str, l)))
def test_in_place_gives_the_bits_of_out_of_place(lists, dtype):
    """Few and dense lists, short and long bias lists, and prefixes of one sequence, with a grammar beside them."""
    history, bias, prefix = lists
    rng = np.random.default_rng(history + bias)
    rows, V = 9, 20011
    kind, npt = DT[dtype]
    x, g = logits(rng, rows, V, V, dtype), logits(rng, rows, V, V, dtype)
    r = make_rules(rng, rows, V, history=history, bias=bias, grammar="indexed", prefix=prefix)
    h = device_rules(r)
    t = G.dev(x)
    api.hilore_logits_apply(t, kind, rows, V, V, h, t, V)
    assert np.array_equal(to_f64(t.cpu().numpy().view(npt)), apply(x, V, r, dtype, V))
    t = G.dev(g)
    api.hilore_logits_apply_backward(G.dev(x), kind, rows, V, V, h, t, V, t, V)
    assert np.array_equal(to_f64(t.cpu().numpy().view(npt)), apply(x, V, r, dtype, V, backward=g))
    targets = rng.integers(0, V, rows).astype(np.int32)
    _, lse, _ = run_logp(x, V, r, targets, dtype)
    omega = rng.standard_normal(rows)
    t = G.dev(x)
    api.hilore_token_logp_backward(t, kind, rows, V, V, h, G.dev(targets), G.dev(lse.astype(np.float32)), G.dev(omega.astype(np.float32)), t, V)
    assert np.array_equal(to_f64(t.cpu().numpy().view(npt)), run_grad(x, V, r, targets, lse, omega, dtype))


def test_a_row_of_more_ranges_than_a_few_thousand():
    """One row of 2^27 + 5 bf16 logits with three biased tokens: both ends of the row, and every range between them."""
    V = (1 << 27) + 5
    x = torch.randn(V, device="cuda").to(torch.bfloat16)
    at = torch.tensor([0, 70000001, V - 1], dtype=torch.int32, device="cuda")
    h = api.make_logit_rules(bias_tokens=at, bias_values=torch.tensor([1.0, 2.0, 4.0], device="cuda"),
                             bias_offsets=torch.tensor([0, 3], device="cuda"))
    y = torch.full_like(x, 7.0)
    api.hilore_logits_apply(x, api.BF16, 1, V, V, h, y, V)
    want = x.clone()
    want[at.long()] = (x[at.long()].float() + torch.tensor([1.0, 2.0, 4.0], device="cuda")).to(torch.bfloat16)
    assert torch.equal(y, want)
    api.hilore_token_logp_backward(x, api.BF16, 1, V, V, h, torch.tensor([V - 1], dtype=torch.int32, device="cuda"),
                                   torch.tensor([9.0], device="cuda"), torch.ones(1, device="cuda"), y, V)
    z = x.float()
    z[at.long()] += torch.tensor([1.0, 2.0, 4.0], device="cuda")
    p = -(z - 9.0).exp_()
    p[V - 1] += 1.0
    # the rounding to bf16, and the exponent's fp32 error: |z - 9| < 32 at 2^-23, three roundings and the function's two units
    assert bool(((y.float() - p).abs() <= p.abs() * (2.0 ** -8 + 2.0 ** -16) + 2.0 ** -22 + 1e-38).all())
