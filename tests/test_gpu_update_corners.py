"""Corners of the logit rules, the token log-probabilities and the optimizer calls: work splits that only large or many-row calls
take, rows of different alignment, equal bits on different paths, and values at the ends of the ranges."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api
from tests import update_ref as R
from tests.test_gpu_logits import check, device_rules, make_rules

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["apply", "apply_backward", "logp_backward"])
def test_rows_that_end_before_the_last_range(call):
    """Prefix rows whose leading elements alternate between 15 and 7 (8 and 0 for the gradient of logp), with the last token of the
    vocabulary as a fresh one of the second row.  At 148 SMs the last range of these vocabularies begins 14 (2) positions behind V, so
    every other row has none in it.  All values are powers of two, or far from a rounding point of bf16."""
    rows, V, ld, lead, n = (21, 2018302, 2018312, 8, 21000) if call == "logp_backward" else (16, 2427250, 2427256, 15, 16)
    assert ld % 16 == 8
    raw = torch.full((rows * ld + 16,), 1.0, dtype=torch.bfloat16, device="cuda")
    assert raw.data_ptr() % 32 == 0
    at = raw.data_ptr() + 2 * lead
    tokens = torch.arange(100, 100 + n, dtype=torch.int32, device="cuda")
    tokens[1] = V - 1
    rules = api.make_logit_rules(repetition=torch.full((rows,), 2.0, device="cuda"), tokens=tokens,
                                 hist_begin=torch.zeros(rows, dtype=torch.int64, device="cuda"),
                                 resp_begin=torch.zeros(rows, dtype=torch.int64, device="cuda"),
                                 hist_end=torch.arange(1, rows + 1, device="cuda"))
    out = torch.full_like(raw, 9.0)
    got = out[lead:lead + rows * ld].view(rows, ld)[:, :V]
    to = out.data_ptr() + 2 * lead
    plain, seen = 1.0, 0.5
    if call == "apply":
        api.hilore_logits_apply(at, api.BF16, rows, V, ld, rules, to, ld)
    elif call == "apply_backward":
        api.hilore_logits_apply_backward(at, api.BF16, rows, V, ld, rules, at, ld, to, ld)
    else:
        targets = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
        api.hilore_token_logp_backward(at, api.BF16, rows, V, ld, rules, targets, torch.full((rows,), 3.0, device="cuda"),
                                       torch.ones(rows, device="cuda"), to, ld)
        plain, seen = -np.exp(-2.0), -0.5 * np.exp(-2.5)
    want = torch.full((rows, V), plain, dtype=torch.bfloat16, device="cuda")
    for i in range(rows):
        want[i, tokens[:i + 1].long()] = seen
    if call == "logp_backward":
        want[:, 7] = 1.0 - np.exp(-2.0)
    assert torch.equal(got, want), torch.argwhere(got != want)[:5].tolist()


def test_threads_with_tables_of_unequal_size(monkeypatch):
    """Log-probabilities under rules from three host threads on streams of their own: the shared memory of a call goes by the size
    of its vocabulary (76 KB and 36 KB here, a CTA per row), and no thread's opt-in may take away another's.  Every call
    has to be accepted; the last one gives the bits of the first, which was issued alone.  Two rows and the plain ctypes call, so
    that the threads spend their time in the library."""
    monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", "1")
    rows, calls = 2, 20000
    jobs = []
    for i, V in enumerate((32000, 12000, 12000)):
        gen = torch.Generator(device="cuda").manual_seed(i)
        x = torch.randn(rows, V, generator=gen, device="cuda").to(torch.bfloat16)
        where = torch.arange(rows, device="cuda")
        rules = api.make_logit_rules(repetition=torch.full((rows,), 1.5, device="cuda"), hist_begin=torch.zeros_like(where),
                                     tokens=torch.randint(0, V, (rows,), generator=gen, device="cuda", dtype=torch.int32),
                                     resp_begin=torch.zeros_like(where), hist_end=where + 1)
        targets = torch.randint(0, V, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        alone, logp, stream = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.cuda.Stream()
        api.hilore_token_logp(x, api.BF16, rows, V, V, rules, targets, alone, None, None)
        args = (x.data_ptr(), api.BF16, rows, V, V, ctypes.addressof(rules), targets.data_ptr(), logp.data_ptr(), None, None, stream.cuda_stream)
        jobs.append(dict(args=args, alone=alone, logp=logp, refused=0, keep=(x, rules, targets, stream)))

    def run(job):
        call, args = api.lib().hilore_token_logp, job["args"]
        for _ in range(calls):
            job["refused"] += call(*args) != api.OK

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(job,)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert [job["refused"] for job in jobs] == [0, 0, 0]
    assert all(torch.equal(job["alone"], job["logp"]) for job in jobs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_has_the_same_bits_in_every_batch(dtype, monkeypatch):
    """Prefix rows, whose tables are carried from row to row of a block, against the same rows called alone and by sevens: equal
    alignment, one CTA per row in every call, so the sums are the same, whichever row a block began with."""
    monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", "1")
    kind, tt = (api.BF16, torch.bfloat16) if dtype == "bf16" else (api.F32, torch.float32)
    rows, V, ld, length = 3000, 5003, 5008, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn(rows, ld, generator=gen, device="cuda") * 3).to(tt)
    row = torch.arange(rows, device="cuda")
    tokens = (torch.rand(rows, generator=gen, device="cuda") ** 2 * V).int()
    parts = dict(repetition=torch.full((rows,), 1.3, device="cuda"), frequency=torch.full((rows,), 0.2, device="cuda"),
                 presence=torch.full((rows,), 0.1, device="cuda"), hist_begin=row // length * length, hist_end=row,
                 resp_begin=torch.minimum(row // length * length + length // 4, row))
    targets = torch.randint(0, V, (rows,), generator=gen, device="cuda", dtype=torch.int32)

    def call(a, b):
        rules = api.make_logit_rules(tokens=tokens, **{k: v[a:b].contiguous() for k, v in parts.items()})
        out = torch.zeros(3, b - a, device="cuda")
        api.hilore_token_logp(x[a:b], kind, b - a, V, ld, rules, targets[a:b], out[0], out[1], out[2])
        return out

    whole = call(0, rows)
    for a in list(range(0, 16)) + list(range(1000, 1040)) + [rows - 1]:
        assert torch.equal(call(a, a + 1), whole[:, a:a + 1]), a
    for a in (3, 290, 2001, rows - 7):
        assert torch.equal(call(a, a + 7), whole[:, a:a + 7]), a


def eight_bit_step(g, shift):
    """First step of one fp32 tensor with 8-bit moments from zeros and no eps, p `shift` elements off the vectors' alignment."""
    n = g.numel()
    p = torch.zeros(n + shift, device="cuda")[shift:]
    e = dict(p=p, g=g, m=torch.zeros(n, dtype=torch.uint8, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"),
             m_scale=torch.zeros(-(-n // 64), device="cuda"), v_scale=torch.zeros(-(-n // 64), device="cuda"))
    dev, host = api.make_param_table([e])
    api.hilore_adamw_step(dev, host, 1, 0.01, None, 0.9, 0.99, 0.0, 1, None, None)
    return e


def same_bits(a, b, names=("p", "m", "v", "m_scale", "v_scale")):
    kinds = {1: torch.uint8, 4: torch.int32}
    return [k for k in names if not torch.equal(a[k].view(kinds[a[k].element_size()]), b[k].view(kinds[b[k].element_size()]))]


def test_eight_bit_step_has_the_same_bits_on_every_path():
    """2^24 gradients as vectors, element by element, and as vectors in warps that hold an Inf or a NaN.  A third of the blocks has
    squares down to 2^-126, where the residual of the root's last step is no longer exact.  Blocks with the planted value are left out
    of the comparison."""
    n = 1 << 24
    gen = torch.Generator(device="cuda").manual_seed(11)
    size = torch.randint(-20, 20, (n // 64,), generator=gen, device="cuda")
    size = torch.where(torch.arange(n // 64, device="cuda") % 3 == 0, size - 40, size)
    g = torch.randn(n, generator=gen, device="cuda") * torch.exp2(size.float()).repeat_interleave(64)
    vectors = eight_bit_step(g, 0)
    elements = eight_bit_step(g, 1)
    assert same_bits(vectors, elements) == []
    del elements
    odd = g.clone()
    odd[5::1024] = float("inf")                                # a block in every run of 512, one kind in the even and one in the odd runs
    odd[512 + 9::1024] = float("nan")
    for shift in (0, 1):
        got = eight_bit_step(odd, shift)
        for k in ("p", "m", "v"):
            kind = torch.uint8 if got[k].element_size() == 1 else torch.int32
            assert torch.equal(got[k].view(kind).view(-1, 512)[:, 64:], vectors[k].view(kind).view(-1, 512)[:, 64:]), (k, shift)
        for k in ("m_scale", "v_scale"):
            assert torch.equal(got[k].view(-1, 8)[:, 1:], vectors[k].view(-1, 8)[:, 1:]), (k, shift)


@pytest.mark.parametrize("kind", ["bf16", "f32", "master"])
def test_eight_bit_step_of_shifted_tensors_has_the_same_bits(kind):
    """Small tensors with moments behind them, of every parameter kind, at aligned and at shifted addresses, ragged ends included."""
    n = 3 * 1024 + 77
    gen = torch.Generator(device="cuda").manual_seed(4)
    w, g = torch.randn(n, generator=gen, device="cuda") * 0.02, torch.randn(n, generator=gen, device="cuda") * 1e-3
    done = []
    for shift in (0, 1, 5):
        put = lambda t: torch.cat([t.new_zeros(shift), t])[shift:]
        p = put(w if kind == "f32" else w.bfloat16())
        code = lambda: put(torch.zeros(n, dtype=torch.uint8, device="cuda"))
        e = dict(p=p, g=put(g.bfloat16()), m=code(), v=code(), m_scale=torch.zeros(-(-n // 64), device="cuda"), v_scale=torch.zeros(-(-n // 64), device="cuda"),
                 weight_decay=0.1)
        if kind == "master":
            e["master"] = put(w)
        dev, host = api.make_param_table([e])
        for t in range(1, 6):
            api.hilore_adamw_step(dev, host, 1, 0.01, None, 0.9, 0.99, 1e-8, t, None, None)
        done.append({k: t.contiguous().view(torch.int16).int() if t.dtype == torch.bfloat16 else t.clone() for k, t in e.items() if isinstance(t, torch.Tensor)})
    names = [k for k in done[0] if k != "g"]
    assert same_bits(done[0], done[1], names) == [] and same_bits(done[0], done[2], names) == []


@pytest.mark.parametrize("shift", [0, 1], ids=["vectors", "elements"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_gradients_whose_squares_leave_fp32(dtype, shift):
    """Sizes from subnormal numbers to 1e38, alone and beside zeros and ordinary ones: 32 additions in fp32 and the rest in fp64, so a
    relative error of 33 * 2^-24 at most.  The norm of 1e38s does not fit fp32, its scale does."""
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n = 40 * 1024 + 333
    gen = torch.Generator(device="cuda").manual_seed(2)
    ws = torch.zeros(api.hilore_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")
    for sizes in ((1e-24,), (1e-19,), (1e-16,), (3e-39,), (0.0, 1e-30), (1e-24, 1e-3), (0.0,), (1e18, 1e20), (1e38,)):
        g = torch.randn(n, generator=gen, device="cuda").clamp_(-3, 3).double() * torch.tensor(sizes, device="cuda", dtype=torch.float64).repeat_interleave(64).repeat(n)[:n]
        g = torch.cat([torch.zeros(shift, device="cuda", dtype=tt), g.to(tt)])[shift:]
        z = torch.zeros(n, device="cuda")
        dev, host = api.make_param_table([dict(p=z, g=g, m=z, v=z)])
        norm, scale = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
        api.hilore_grad_norm(dev, host, 1, 1e-2, norm, scale, ws, ws.numel())
        want = float(g.double().norm())
        assert want < 3.4e38 and float(norm) == pytest.approx(want, rel=33 * 2.0 ** -24, abs=1e-45) or want > 3.5e38 and float(norm) == float("inf"), (sizes, float(norm), want)
        assert float(scale) == pytest.approx(min(1.0, 1e-2 / (want + 1e-6)), rel=35 * 2.0 ** -24, abs=1e-45), sizes


@pytest.mark.parametrize("entropy", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ruled", ["temperature", "grammar", "lists"])
def test_infinite_temperature_is_uniform_over_what_is_allowed(ruled, dtype, entropy):
    """z = x / inf = 0 for every allowed token: logp = -ln n, lse = entropy = ln n (a logarithm and V / 256 + 40 additions of fp32), a
    denied target -inf; the gradient is zero.  Odd sizes, so that both ends of a row are taken element by element."""
    kind, tt = (api.BF16, torch.bfloat16) if dtype == "bf16" else (api.F32, torch.float32)
    rows, V = 3, 1003
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = (torch.randn(rows, V, generator=gen, device="cuda") * 4).to(tt)
    allow = torch.full((rows, 32), -1, dtype=torch.int32, device="cuda")
    allow[:, 3] = 0
    allow[2, 31] = 0
    parts = dict(temperature=torch.full((rows,), float("inf"), device="cuda"))
    if ruled != "temperature":
        parts["allow"] = allow
    if ruled == "lists":
        parts.update(repetition=torch.full((rows,), 1.5, device="cuda"), tokens=torch.arange(90, 130, dtype=torch.int32, device="cuda"),
                     hist_begin=torch.zeros(rows, dtype=torch.int64, device="cuda"), resp_begin=torch.zeros(rows, dtype=torch.int64, device="cuda"),
                     hist_end=torch.full((rows,), 40, device="cuda"))
    rules = api.make_logit_rules(**parts)
    n = np.array([V, V, V] if ruled == "temperature" else [V - 32, V - 32, V - 32 - 11])
    targets = torch.tensor([5, 100, 700], dtype=torch.int32, device="cuda")
    out = torch.full((3, rows), 9.0, device="cuda")
    api.hilore_token_logp(x, kind, rows, V, V, rules, targets, out[0], out[1], out[2] if entropy else None)
    logp, lse, h = out.double().cpu().numpy()
    want = -np.log(n)
    if ruled != "temperature":
        want[1] = -np.inf                                       # token 100 is denied
    tol = (V / 256 + 48) * 2.0 ** -24 * 8
    assert np.allclose(logp, want, rtol=0, atol=tol) and np.allclose(lse, np.log(n), rtol=0, atol=tol)
    assert not entropy or np.allclose(h, np.log(n), rtol=0, atol=tol)
    grad = torch.full_like(x, 7.0)
    api.hilore_token_logp_backward(x, kind, rows, V, V, rules, targets, out[1], torch.ones(rows, device="cuda"), grad, V)
    assert bool((grad == 0).all())
    z = torch.full_like(x, 7.0)
    api.hilore_logits_apply(x, kind, rows, V, V, rules, z, V)
    denied = torch.zeros(rows, V, dtype=torch.bool, device="cuda")
    if ruled != "temperature":
        denied[:, 96:128] = True
        denied[2, 992:] = True
    assert bool((z[denied] == -float("inf")).all()) and bool((z[~denied] == 0).all())


SPLIT = [  # rows, V, leading dimensions of the input and the output, history, bias, grammar, prefix: in blocks x ranges on 148 SMs
    (96, 151936, 151936, 151936, 16384, 48, "indexed", False),    # rules 2 x 6
    (450, 128256, 128256, 128256, 1536, 0, None, True),           # rules 7 x 4
    (450, 128251, 128257, 128252, 150, 6, "indexed", True),       # the same, every row of another alignment, input and output unlike
    (1500, 32063, 32063, 32063, 1200, 0, None, True),             # gradient of logp 7 x 2
    (900, 40001, 40003, 40009, 100, 600, "indexed", True),        # gradient of logp 5 x 2; bias lists in the table among others
    (1021, 50001, 50008, 50001, 900, 24, "indexed", True),        # logp 5 rows of two CTAs
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SPLIT, ids=lambda c: "x".join(str(v) for v in c[:3]))
def test_blocks_of_rows_over_several_ranges(case, dtype):
    """The work splits of large calls, whose tables go from row to row of a block in each of several ranges (or CTAs of a cluster): all
    four calls against the definition, at the first rows, at the last and at one block's worth of others in between."""
    rows, V, ld, ld_out, history, bias, grammar, prefix = case
    kind, tt = (api.BF16, torch.bfloat16) if dtype == "bf16" else (api.F32, torch.float32)
    rng = np.random.default_rng(rows + V)
    gen = torch.Generator(device="cuda").manual_seed(V)
    r = make_rules(rng, rows, V, history=history, bias=bias, grammar=grammar, prefix=prefix)
    rules = device_rules(r)
    x = (torch.randn(rows, ld, generator=gen, device="cuda") * 3).to(tt)
    dz = (torch.randn(rows, ld_out, generator=gen, device="cuda") * 0.01).to(tt)
    middle = int(rng.integers(10, rows - 20))
    sample = sorted(set(range(10)) | set(range(middle, middle + 9)) | {rows - 2, rows - 1})
    pull = lambda t: t[sample][:, :V].float().double().cpu().numpy()
    xs, ds = pull(x), pull(dz)
    ref = [R.rules_row(xs[j], r, i) for j, i in enumerate(sample)]
    z, k, e = (np.stack([t[j] for t in ref]) for j in range(3))
    y = torch.full((rows, ld_out), 7.0, dtype=tt, device="cuda")
    api.hilore_logits_apply(x, kind, rows, V, ld, rules, y, ld_out)
    check(pull(y), z, e, dtype)
    assert bool((y[:, V:] == 7).all())
    api.hilore_logits_apply_backward(x, kind, rows, V, ld, rules, dz, ld_out, y, ld_out)
    check(pull(y), ds * k, 4 * R.U * np.abs(ds * k), dtype)
    targets = rng.integers(0, V, rows).astype(np.int32)
    targets[4] = -1
    omega = rng.standard_normal(rows).astype(np.float32)
    omega[6] = 0
    t, w = torch.from_numpy(targets).cuda(), torch.from_numpy(omega).cuda()
    out = torch.zeros(3, rows, device="cuda")
    api.hilore_token_logp(x, kind, rows, V, ld, rules, t, out[0], out[1], out[2])
    got = out[:, sample].double().cpu().numpy()
    grads, errors = [], []
    for j, i in enumerate(sample):
        want, bound = R.logp_row(z[j], targets[i]), R.logp_bound(z[j], e[j], V)
        for q in range(3):
            assert got[q, j] == want[q] or abs(got[q, j] - want[q]) <= bound[q] + 4 * R.U * abs(want[q]), (q, i, got[q, j], want[q])
        finite = np.isfinite(want[1])
        grads.append(R.grad_row(z[j], k[j], targets[i], float(omega[i]), want[1]))
        errors.append(R.grad_bound(z[j], e[j], k[j], float(omega[i]), want[1] if finite else 0.0, bound[1] + 4 * R.U * abs(want[1]) if finite else 0.0))
    api.hilore_token_logp_backward(x, kind, rows, V, ld, rules, t, out[1], w, y, ld_out)
    check(pull(y), np.stack(grads), np.stack(errors), dtype)
    api.hilore_logits_apply(x, kind, rows, V, ld, rules, x, ld)                       # in place
    check(pull(x), z, e, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ld,ld_out,shift", [(1, 1, 1, 0), (31, 33, 32, 1), (2051, 2051, 2051, 0), (40003, 40003, 40010, 5), (151936, 151936, 151936, 0)])
def test_rules_without_lists(V, ld, ld_out, shift, dtype):
    """Temperature and a grammar alone, at equal and unequal alignments, and the temperature alone in place, forward and backward."""
    kind, tt = (api.BF16, torch.bfloat16) if dtype == "bf16" else (api.F32, torch.float32)
    rows = 5
    rng = np.random.default_rng(V)
    r = make_rules(rng, rows, V, history=-1, grammar="indexed")
    rules = device_rules(r)
    raw = (torch.randn(rows * ld + shift, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda") * 3).to(tt)
    x = raw[shift:].view(rows, ld)
    host = lambda t: t[:, :V].float().double().cpu().numpy()
    xs = host(x)
    ref = [R.rules_row(xs[i], r, i) for i in range(rows)]
    z, k, e = (np.stack([t[j] for t in ref]) for j in range(3))
    y = torch.full((rows, ld_out), 7.0, dtype=tt, device="cuda")
    api.hilore_logits_apply(x, kind, rows, V, ld, rules, y, ld_out)
    check(host(y), z, e, dtype)
    g = torch.randn(rows, ld_out, device="cuda").to(tt)
    gs = host(g)
    api.hilore_logits_apply_backward(x, kind, rows, V, ld, rules, g, ld_out, y, ld_out)
    check(host(y), gs * k, 4 * R.U * np.abs(gs * k), dtype)
    assert bool((y[:, V:] == 7).all())
    api.hilore_logits_apply_backward(x, kind, rows, V, ld, rules, g, ld_out, g, ld_out)
    assert torch.equal(g[:, :V], y[:, :V])
    t = np.float32(r["temperature"])[:, None].astype(np.float64)
    api.hilore_logits_apply(x, kind, rows, V, ld, api.make_logit_rules(temperature=torch.from_numpy(r["temperature"]).cuda()), x, ld)
    check(host(x), xs / t, 4 * R.U * np.abs(xs / t), dtype)


@pytest.mark.parametrize("kind", ["bf16", "f32", "master"])
def test_step_with_fp32_moments_has_the_same_bits_at_any_address(kind):
    n = 3 * 1024 + 77
    gen = torch.Generator(device="cuda").manual_seed(8)
    w, g = torch.randn(n, generator=gen, device="cuda") * 0.02, torch.randn(n, generator=gen, device="cuda") * 1e-3
    done = []
    for shift in (0, 1, 5):
        put = lambda t: torch.cat([t.new_zeros(shift), t])[shift:]
        e = dict(p=put(w if kind == "f32" else w.bfloat16()), g=put(g.bfloat16()), m=put(g * 0.5), v=put(g * g), weight_decay=0.1)
        if kind == "master":
            e["master"] = put(w)
        dev, host = api.make_param_table([e])
        for t in range(1, 4):
            api.hilore_adamw_step(dev, host, 1, 0.01, None, 0.9, 0.99, 1e-8, t, None, None)
        done.append({k: t.contiguous().view(torch.int16).int() if t.dtype == torch.bfloat16 else t.clone() for k, t in e.items() if isinstance(t, torch.Tensor)})
    names = [k for k in done[0] if k != "g"]
    assert same_bits(done[0], done[1], names) == [] and same_bits(done[0], done[2], names) == []
