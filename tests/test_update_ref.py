"""Pins of the plain definitions in tests/update_ref.py (hand values, finite differences, invariants) and everything of
the new entry points that is decided on the host: refusals, struct layouts, the marshalling helpers."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api, build
from tests import update_ref as R


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.lib()


def _rules(rng, V, rows=1):
    n = 60
    return dict(temperature=rng.uniform(0.5, 2, rows), repetition=rng.uniform(1, 2, rows), frequency=rng.uniform(0, 1, rows),
                presence=rng.uniform(-1, 1, rows), tokens=rng.integers(-1, V + 2, n).astype(np.int32),
                hist_begin=np.full(rows, 3), resp_begin=np.full(rows, 20), hist_end=np.full(rows, n),
                bias_tokens=np.array([1, 2, 1], np.int32), bias_values=np.array([0.5, -1.0, 2.0]), bias_offsets=np.arange(rows + 1) * 3,
                allow=rng.integers(-2**31, 2**31, (rows, (V + 31) // 32)).astype(np.int32))


def test_rules_by_hand():
    x = np.array([2.0, -2.0, 1.0, 0.0, 5.0])
    r = dict(temperature=[2.0], repetition=[4.0], frequency=[0.5], presence=[0.25], tokens=np.array([0, 1, 9, 1, 1, 2], np.int32),
             hist_begin=[0], resp_begin=[3], hist_end=[6], bias_tokens=[3, 3], bias_values=[7.0, 1.0], bias_offsets=[0, 2],
             allow=np.array([[0b01111]], np.int32))
    z, k, _ = R.rules_row(x, r, 0)
    # token 0: prompt only, 2 / 4; token 1: prompt and twice generated, -2 * 4 - 1 - 0.25; token 2: once, 1 / 4 - 0.75
    assert z.tolist() == [0.25, -4.625, -0.25, 0.5, -np.inf]
    assert k.tolist() == [0.125, 2.0, 0.125, 0.5, 0.0]


@pytest.mark.parametrize("V", [5, 37, 200])
def test_gradient_of_logp_is_its_difference_quotient(V):
    rng = np.random.default_rng(V)
    r = _rules(rng, V)
    x = rng.standard_normal(V) * 2
    a = int(np.flatnonzero(R.allowed_row(r, 0, V))[0])
    z, k, _ = R.rules_row(x, r, 0)
    _, lse, _ = R.logp_row(z, a)
    g = R.grad_row(z, k, a, 0.7, lse)
    h = 1e-6
    for v in range(V):
        if abs(x[v]) < 2 * h:
            continue
        d = []
        for s in (h, -h):
            y = x.copy()
            y[v] += s
            d.append(R.logp_row(R.rules_row(y, r, 0)[0], a)[0])
        assert 0.7 * (d[0] - d[1]) / (2 * h) == pytest.approx(g[v], rel=1e-6, abs=1e-9)
    free = dict(r, allow=None, repetition=None)
    z, k, _ = R.rules_row(x, free, 0)
    assert R.grad_row(z, k, a, 1.0, R.logp_row(z, a)[1]).sum() == pytest.approx(0.0, abs=1e-12)   # softmax: rows sum to zero


def test_logp_edges():
    z = np.array([0.0, 1.0, -np.inf])
    p = np.exp(z) / np.exp(z).sum()
    logp, lse, h = R.logp_row(z, 1)
    assert logp == pytest.approx(np.log(p[1])) and lse == pytest.approx(np.log(np.exp(z).sum()))
    assert h == pytest.approx(-(p[:2] * np.log(p[:2])).sum())
    assert R.logp_row(z, 2)[0] == -np.inf and R.logp_row(z, 3) == (0, 0, 0) and R.logp_row(z, -1) == (0, 0, 0)
    assert R.logp_row(np.full(3, -np.inf), 0) == (-np.inf, -np.inf, 0.0)
    assert not R.grad_row(np.full(3, -np.inf), np.zeros(3), 0, 1.0, -np.inf).any()


def test_e4m3_values_and_rounding():
    assert R.E4M3[0x7E] == 448 and R.E4M3[1] == 2.0 ** -9 and np.isnan(R.E4M3[0x7F]) and R.E4M3[0x80 + 0x38] == -1
    v = R.E4M3[:127]
    assert np.array_equal(R.e4m3_round(v), v)
    q = np.random.default_rng(0).uniform(-460, 460, 4000) * np.exp2(-np.random.default_rng(1).integers(0, 18, 4000))
    want = torch.tensor(q, dtype=torch.float32).clamp(-448, 448).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(R.e4m3_round(np.float64(np.float32(q))), want)


def test_adamw_against_torch_in_double():
    rng = np.random.default_rng(3)
    p0 = rng.standard_normal(50)
    p = torch.tensor(p0, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    m = v = np.zeros(50)
    for t in range(1, 5):
        g = rng.standard_normal(50)
        p.grad = torch.tensor(g)
        before = p.detach().numpy().copy()
        opt.step()
        q, m, v, *_ = R.adamw(before, g, m, v, lr=1e-2, b1=0.9, b2=0.95, eps=1e-8, t=t, wd=0.1)
        # torch shrinks the parameter before the step of the moments, the definition takes both from the old one
        assert np.allclose(q, p.detach().numpy(), rtol=1e-12, atol=1e-12)


def test_struct_layouts_match_the_header(lib):
    assert ctypes.sizeof(api.HiloreLogitRules) == 17 * 8 and api.HiloreLogitRules.allow_ld.offset == 128
    assert ctypes.sizeof(api.HiloreParam) == 9 * 8 + 4 * 4 and api.HiloreParam.weight_decay.offset == 84


A = 0x1000  # a fake, suitably aligned device address: never dereferenced on these paths


def test_refusals_of_the_logit_calls(lib):
    ok = dict(dtype=api.BF16, rows=4, V=100, ld=100, x=A, out=A, ld_out=100)

    def rules(**k):
        return api.HiloreLogitRules(**k)

    def apply(r=rules(), **k):
        k = {**ok, **k}
        return api.hilore_logits_apply(k["x"], k["dtype"], k["rows"], k["V"], k["ld"], r, k["out"], k["ld_out"], stream=0, check=False)

    def apply_bw(r=rules(), **k):
        k = {**ok, **k}
        return api.hilore_logits_apply_backward(k["x"], k["dtype"], k["rows"], k["V"], k["ld"], r, k.get("g", A), k.get("ld_g", 100),
                                                k["out"], k["ld_out"], stream=0, check=False)

    def logp(r=None, **k):
        k = {**ok, **k}
        return api.hilore_token_logp(k["x"], k["dtype"], k["rows"], k["V"], k["ld"], r, k.get("t", A), k.get("logp", A), k.get("lse"),
                                     k.get("h"), stream=0, check=False)

    def logp_bw(r=None, **k):
        k = {**ok, **k}
        return api.hilore_token_logp_backward(k["x"], k["dtype"], k["rows"], k["V"], k["ld"], r, k.get("t", A), k.get("lse", A),
                                              k.get("omega", A), k["out"], k["ld_out"], stream=0, check=False)

    for call in (apply, apply_bw, logp, logp_bw):
        assert call(dtype=2) == api.INVALID_ARG
        assert call(rows=-1) == api.INVALID_ARG
        assert call(V=0, ld=0) == api.INVALID_ARG
        assert call(x=None) == api.INVALID_ARG
        assert call(ld=99) == api.SHAPE
        assert call(V=0x7FFF8000, ld=1 << 32, ld_out=1 << 32, ld_g=1 << 32) == api.SHAPE
        assert call(x=A + 1) == api.ALIGN
        assert call(dtype=api.F32, x=A + 2) == api.ALIGN
        assert call(rows=0) == api.OK
        assert call(rules(n_tokens=5)) == api.INVALID_ARG                                  # tokens missing
        assert call(rules(tokens=A, n_tokens=5, hist_begin=A, resp_begin=A)) == api.INVALID_ARG
        assert call(rules(n_tokens=-1)) == api.INVALID_ARG
        assert call(rules(bias_tokens=A, n_bias=1, bias_values=A)) == api.INVALID_ARG
        assert call(rules(n_bias=2)) == api.INVALID_ARG
        assert call(rules(allow=A, n_allow=3, allow_ld=4)) == api.INVALID_ARG              # four rows, three masks
        assert call(rules(allow=A, n_allow=4, allow_ld=3)) == api.SHAPE                    # 100 bits take four words
        assert call(rules(temperature=A + 2)) == api.ALIGN
        assert call(rules(tokens=A, n_tokens=5, hist_begin=A + 4, resp_begin=A, hist_end=A)) == api.ALIGN
    for call in (apply, apply_bw):
        assert call(None) == api.INVALID_ARG
    for call in (apply, apply_bw, logp_bw):
        assert call(out=None) == api.INVALID_ARG
        assert call(ld_out=99) == api.SHAPE
        assert call(out=A + 1) == api.ALIGN
    assert apply_bw(g=None) == api.INVALID_ARG and apply_bw(ld_g=99) == api.SHAPE and apply_bw(g=A + 1) == api.ALIGN
    assert apply(ld_out=101) == api.SHAPE and logp_bw(ld_out=101) == api.SHAPE             # in place, at another distance
    assert apply_bw(g=2 * A) == api.INVALID_ARG and apply_bw(x=2 * A, ld_g=101) == api.SHAPE
    assert logp(t=None) == api.INVALID_ARG and logp(logp=None) == api.INVALID_ARG and logp(h=A + 1) == api.ALIGN
    assert logp_bw(lse=None) == api.INVALID_ARG and logp_bw(omega=None) == api.INVALID_ARG
    with pytest.raises(api.HiloreError, match="hilore_token_logp"):
        api.hilore_token_logp(A, 7, 1, 1, 1, None, A, A, None, None, stream=0)


def _entry(**k):
    e = dict(p=A, g=A, m=A, v=A, n=2000, first=0, p_dtype=api.BF16, g_dtype=api.BF16, state=api.STATE_F32)
    e.update(k)
    return api.HiloreParam(**e)


def _table(*entries):
    return (api.HiloreParam * len(entries))(*entries)


def test_refusals_of_the_optimizer_calls(lib):
    def step(t, n=None, dev=A, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, k=1, lr_dev=None, step_dev=None, scale=None):
        return api.hilore_adamw_step(dev, t, len(t) if n is None else n, lr, lr_dev, b1, b2, eps, k, step_dev, scale, stream=0, check=False)

    def norm(t, n=None, dev=A, max_norm=1.0, out=A, scale=None, ws=A, nws=1 << 20):
        return api.hilore_grad_norm(dev, t, len(t) if n is None else n, max_norm, out, scale, ws, nws, stream=0, check=False)

    good = _table(_entry())
    for call in (step, norm):
        assert call(good, n=-1) == api.INVALID_ARG
        assert call(good, dev=None) == api.INVALID_ARG
        assert call(good, dev=A + 4) == api.ALIGN
        assert call(_table(_entry(n=-1))) == api.INVALID_ARG
        assert call(_table(_entry(g=None))) == api.INVALID_ARG
        assert call(_table(_entry(g_dtype=5))) == api.INVALID_ARG
        assert call(_table(_entry(g=A + 1))) == api.ALIGN
        assert call(_table(_entry(first=1))) == api.SHAPE
        assert call(_table(_entry(), _entry(first=1))) == api.SHAPE              # 2000 elements are two tiles
    assert step(good, b1=1.0) == api.INVALID_ARG and step(good, b2=-0.1) == api.INVALID_ARG
    assert step(good, eps=-1.0) == api.INVALID_ARG and step(good, lr=float("nan")) == api.INVALID_ARG
    assert step(good, k=0) == api.INVALID_ARG
    assert step(good, lr_dev=A + 2) == api.ALIGN and step(good, step_dev=A + 4) == api.ALIGN and step(good, scale=A + 1) == api.ALIGN
    assert step(_table(_entry(p=None))) == api.INVALID_ARG and step(_table(_entry(v=None))) == api.INVALID_ARG
    assert step(_table(_entry(p_dtype=2))) == api.INVALID_ARG and step(_table(_entry(state=2))) == api.INVALID_ARG
    assert step(_table(_entry(state=api.STATE_E4M3FN))) == api.INVALID_ARG       # no scales
    assert step(_table(_entry(p_dtype=api.F32, master=A))) == api.INVALID_ARG
    assert step(_table(_entry(m=A + 2))) == api.ALIGN and step(_table(_entry(p=A + 1))) == api.ALIGN
    assert step(_table(_entry(n=0, p=None, g=None, m=None, v=None))) == api.OK   # nothing to do
    assert step(good, n=0) == api.OK
    assert norm(good, max_norm=-1.0) == api.INVALID_ARG and norm(good, max_norm=float("nan")) == api.INVALID_ARG
    assert norm(good, out=None) == api.INVALID_ARG and norm(good, ws=None) == api.INVALID_ARG
    assert norm(good, ws=A + 8) == api.ALIGN
    assert norm(good, nws=api.hilore_grad_norm_workspace_bytes() - 1) == api.WORKSPACE


def test_marshalling_helpers():
    t = torch.zeros(130, dtype=torch.bfloat16)
    f = torch.zeros(130)
    codes, scales = torch.zeros(130, dtype=torch.uint8), torch.zeros(3)
    dev, host = api.make_param_table([dict(p=t, g=t, m=f, v=f), dict(p=t, g=f, m=codes, v=codes, m_scale=scales, v_scale=scales,
                                                                      weight_decay=0.5, master=f),
                                      dict(p=torch.zeros(2049), g=torch.zeros(2049), m=torch.zeros(2049), v=torch.zeros(2049)),
                                      dict(p=f, g=f, m=f, v=f)], device="cpu")
    assert [e.first for e in host] == [0, 1, 2, 5] and [e.n for e in host] == [130, 130, 2049, 130]
    assert [e.state for e in host] == [0, 1, 0, 0] and host[1].weight_decay == 0.5 and host[1].master == f.data_ptr()
    assert [e.p_dtype for e in host] == [api.BF16, api.BF16, api.F32, api.F32] and [e.g_dtype for e in host] == [0, 1, 1, 1]
    assert bytes(dev.numpy().tobytes()) == bytes(host)
    assert api.make_param_table([], device="cpu")[0] is None
    with pytest.raises(ValueError, match="m_scale"):
        api.make_param_table([dict(p=t, g=t, m=codes, v=codes, m_scale=torch.zeros(2), v_scale=scales)], device="cpu")
    with pytest.raises(ValueError, match="codes with scales"):
        api.make_param_table([dict(p=t, g=t, m=codes, v=codes)], device="cpu")
    with pytest.raises(TypeError, match="g: expected"):
        api.make_param_table([dict(p=t, g=torch.zeros(130, dtype=torch.float16), m=f, v=f)], device="cpu")
    with pytest.raises(TypeError, match="tokens"):
        api.make_logit_rules(tokens=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="contiguous"):
        api.make_logit_rules(temperature=torch.zeros(6)[::2])
    r = api.make_logit_rules(allow=torch.zeros(3, 7, dtype=torch.int32), bias_tokens=torch.zeros(5, dtype=torch.int32))
    assert (r.n_allow, r.allow_ld, r.n_bias, r.n_tokens) == (3, 7, 5, 0)
