"""The definitions that the GPU tests of the advantages, the policy loss and the preference loss compare with: gradients against
differences, hand-worked values; and what the calls refuse, which needs no GPU."""
import math

import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api, build
from tests import objective_ref as R


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.lib()


def batch(seed, lengths, masked=0.3):
    rng = np.random.default_rng(seed)
    bounds = np.concatenate([[0], np.cumsum(lengths)])
    n = int(bounds[-1])
    return rng, bounds, n, (rng.random(n) >= masked).astype(np.uint8)


def test_advantages_by_hand():
    """Two valid tokens around a masked one, gamma 1/2, lambda 1/2: A_2 = 3 + 1/2 * 4 + 1 - 2 = 4, A_1 = 1 + 1/2 * 2 - 1 + 1/4 * 4 = 2."""
    adv, ret, (mean, std), _ = R.advantages([1, 9, 3], [1], [1, 9, 2], [4], None, [1, 0, 1], [0, 3], 3, 0.5, 0.5)
    assert adv.tolist() == [2, 0, 4] and ret.tolist() == [3, 0, 6] and (mean, std) == (3, 1)


def test_advantages_backward_is_the_gradient():
    rng, bounds, n, mask = batch(0, [5, 0, 1, 9])
    S, step = 4, 1e-6
    x = dict(rewards=rng.normal(size=n), outcome=rng.normal(size=S), values=rng.normal(size=n), bootstrap=rng.normal(size=S), trace=rng.uniform(0.2, 1.2, n))
    ga, gr = rng.normal(size=n), rng.normal(size=n)
    f = lambda **k: (lambda a: (ga * a[0] + gr * a[1]).sum())(R.advantages(*[{**x, **k}[i] for i in x], mask, bounds, n, 0.9, 0.8))
    ga, gr = ga * mask, gr * mask
    adv = R.advantages(*x.values(), mask, bounds, n, 0.9, 0.8)[0]
    got, _ = R.advantages_backward(ga, gr, adv, x["trace"], mask, bounds, n, 0.9, 0.8)
    for name, v in x.items():
        for i in range(v.size):
            d = np.zeros(v.size)
            d[i] = step
            assert abs((f(**{name: v + d}) - f(**{name: v - d})) / (2 * step) - got[name][i]) < 1e-7, (name, i)


@pytest.mark.parametrize("ratio,mean,kl,dual,rollout,per_token", [(0, 0, 3, 0.0, False, True), (0, 1, 2, 2.0, True, True), (0, 1, 1, 1.5, True, False),
                                                                  (1, 1, 3, 2.0, True, False), (1, 0, 2, 0.0, False, False)])
def test_policy_gradient(ratio, mean, kl, dual, rollout, per_token):
    rng, bounds, n, mask = batch(ratio + 2 * kl, [6, 0, 1, 11, 4])
    lp = rng.normal(-2, 0.5, n)
    old, ref = lp + rng.normal(0, 0.5, n), lp + rng.normal(0, 0.5, n)
    if ratio:  # sequences on both sides of the bounds
        old = lp + np.repeat([0.4, 0.0, -0.5, 0.05, -1.2], np.diff(bounds)) + rng.normal(0, 0.05, n)
    t = dict(clip_low=0.2, clip_high=0.3, dual_clip=dual, beta=0.1, rollout_cap=1.1, adv_eps=1e-6, ratio=ratio, mean=mean, kl=kl, adv_per_token=per_token)
    args = (old, ref, old + rng.normal(0, 0.2, n) if rollout else None, mask, rng.normal(size=n if per_token else 5), [0.1, 0.7], bounds, t, 13)
    stats, omega, *_ = R.policy(lp, *args)
    for i in range(n):
        d = np.zeros(n)
        d[i] = 1e-6
        slope = (R.policy(lp + d, *args)[0][0] - R.policy(lp - d, *args)[0][0]) / 2e-6
        assert abs(slope - omega[i]) < 1e-7
    assert stats[3] > 0 and np.array_equal(omega == 0, mask == 0)


def test_policy_is_grpo_where_it_should_be():
    import oracle
    rng = np.random.default_rng(5)
    lp = rng.normal(-1.5, 0.5, (4, 8)).astype(np.float32)
    old, ref = (lp + rng.normal(0, 0.3, lp.shape)).astype(np.float32), (lp + rng.normal(0, 0.3, lp.shape)).astype(np.float32)
    mask = (rng.random(lp.shape) < 0.7).astype(np.uint8)
    adv = rng.normal(size=4)
    want, _, _ = oracle.grpo_coeffs(adv, lp, old, ref, mask, N_norm=17, clip_eps=0.2, beta=0.05)
    t = dict(clip_low=0.2, clip_high=0.2, dual_clip=0.0, beta=0.05, rollout_cap=math.inf, adv_eps=0.0, ratio=0, mean=0, kl=3, adv_per_token=0)
    _, omega, *_ = R.policy(lp.ravel(), old.ravel(), ref.ravel(), None, mask.ravel(), adv, None, np.arange(5) * 8, t, 17)
    assert np.allclose(omega.reshape(4, 8), want, rtol=1e-5, atol=1e-9)


@pytest.mark.parametrize("loss", [0, 1, 2])
@pytest.mark.parametrize("length_mean,nll,ref", [(0, 0.0, True), (1, 0.3, False)])
def test_preference_gradient(loss, length_mean, nll, ref):
    rng, bounds, n, mask = batch(loss, [4, 3, 0, 7, 2, 5])
    lp = rng.normal(-2, 0.5, n)
    t = dict(beta=0.3, margin=0.1, margin_reward=0.2, smoothing=0.1 if loss == 0 else 0.0, nll=nll, loss=loss, length_mean=length_mean)
    args = (lp + rng.normal(0, 0.5, n) if ref else None, mask, [1.0, 0.0, 2.0, 0.5, 1.0, 1.0], 3, bounds, t)
    stats, omega, _, pairs, *_ = R.preference(lp, *args)
    assert pairs == 3 and abs(omega).sum() > 0  # the empty response is in no pair; one pair of the first three, two of the others
    for i in range(n):
        d = np.zeros(n)
        d[i] = 1e-6
        assert abs((R.preference(lp + d, *args)[0][0] - R.preference(lp - d, *args)[0][0]) / 2e-6 - omega[i]) < 1e-7


def test_preference_by_hand():
    """One token each: h = 2 (s - s_ref) = 2 and -1, gap 3: ln(1 + e^-3)."""
    t = dict(beta=2.0, margin=0.0, margin_reward=0.0, smoothing=0.0, nll=0.0, loss=0, length_mean=0)
    stats, omega, h, pairs, *_ = R.preference([-1.0, -2.0], [-2.0, -1.5], None, [1, 0], 2, [0, 1, 2], t)
    assert pairs == 1 and h.tolist() == [2, -1]
    assert np.allclose(stats, [math.log1p(math.exp(-3)), 1, 3, 1])
    assert np.allclose(omega, [-2 / (1 + math.exp(3)), 2 / (1 + math.exp(3))])


# ------------------------------------------------------------------------------------------------------------- refusals
A = 0x1000  # a fake, aligned device address: the calls below are refused before anything reads it
BIG = 2 ** 31 - 2 ** 16


def advantages(**k):
    g = lambda name, default: k.get(name, default)
    return api.hilore_advantages(g("rewards", A), None, g("values", A), g("dtype", api.F32), None, None, g("mask", A), g("cu", A), g("S", 4), g("n", 64),
                                 g("gamma", 0.9), g("lam", 0.9), g("adv", A), g("returns", A), g("moments", None), g("ws", A), g("size", 1 << 20), stream=0,
                                 check=False)


def backward(**k):
    g = lambda name, default: k.get(name, default)
    return api.hilore_advantages_backward(g("ga", A), A, g("adv", A), A, A, g("cu", A), g("S", 4), g("n", 64), g("gamma", 0.9), g("lam", 0.9), g("dr", A),
                                          None, A, None, g("dc", A), g("ws", A), g("size", 1 << 20), stream=0, check=False)


def policy(**k):
    g = lambda name, default: k.get(name, default)
    terms = None if g("terms", {}) is None else api.make_policy_terms(**g("terms", {}))
    return api.hilore_policy_loss(g("logp", A), g("old", A), g("ref", A), g("rollout", None), A, g("adv", A), g("white", None), g("cu", A), g("S", 4),
                                  g("n", 64), terms, g("N", 7), g("N_dev", None), g("grad", None), g("stats", A), g("omega", A), g("ws", A),
                                  g("size", 1 << 20), stream=0, check=False)


def preference(**k):
    g = lambda name, default: k.get(name, default)
    terms = None if g("terms", {}) is None else api.make_preference_terms(**g("terms", {}))
    return api.hilore_preference_loss(g("logp", A), g("ref", A), A, g("rewards", A), g("G", 2), g("cu", A), g("S", 4), g("n", 64), terms, g("N", 0),
                                      g("N_dev", None), None, g("scores", None), g("pairs", None), g("stats", A), g("omega", A), g("ws", A),
                                      g("size", 1 << 20), stream=0, check=False)


@pytest.mark.parametrize("call", [advantages, backward, policy, preference])
def test_refusals_of_sizes(lib, call):
    assert call(S=-1) == api.INVALID_ARG and call(n=-1) == api.INVALID_ARG
    assert call(S=0) == api.SHAPE and call(n=BIG + 1) == api.SHAPE and call(S=BIG + 1) == api.SHAPE
    assert call(cu=None, n=66) == api.SHAPE          # 66 slots in 4 rows
    assert call(cu=A + 2) == api.ALIGN
    assert call(ws=None) == api.INVALID_ARG and call(ws=A + 8) == api.ALIGN and call(size=16) == api.WORKSPACE


def test_refusals_of_advantages(lib):
    for bad in (-0.1, 1.1, math.nan, math.inf):
        assert advantages(gamma=bad) == advantages(lam=bad) == backward(gamma=bad) == backward(lam=bad) == api.INVALID_ARG
    assert advantages(dtype=2) == api.INVALID_ARG
    assert advantages(adv=None, returns=None) == api.INVALID_ARG
    assert advantages(rewards=A + 2) == advantages(adv=A + 1) == advantages(values=A + 2) == advantages(values=A + 1, dtype=api.BF16) == api.ALIGN
    assert backward(adv=None) == api.INVALID_ARG and backward(ga=A + 2) == backward(dr=A + 2) == api.ALIGN
    assert backward(S=0, n=0) == api.OK


def test_refusals_of_policy(lib):
    assert policy(terms=None) == api.INVALID_ARG
    for name, values in dict(clip_low=(-0.1, 1.1, math.nan), clip_high=(-0.1, math.nan), dual_clip=(0.5, -1.0, math.nan), beta=(math.inf, math.nan),
                             rollout_cap=(0.0, -1.0, math.nan), adv_eps=(-1.0, math.inf, math.nan), ratio=(2, -1), mean=(2, -1), kl=(0, 4)).items():
        for v in values:
            assert policy(terms={name: v}) == api.INVALID_ARG, (name, v)
    assert policy(terms=dict(ratio=api.RATIO_SEQUENCE, adv_per_token=True)) == api.INVALID_ARG
    assert policy(logp=None) == policy(old=None) == policy(adv=None) == policy(omega=None) == policy(stats=None) == api.INVALID_ARG
    assert policy(ref=None, terms=dict(beta=0.1)) == api.INVALID_ARG
    assert policy(N=0) == policy(N=-3) == api.ZERO_NORM
    assert policy(logp=A + 2) == policy(white=A + 1) == policy(N_dev=A + 4) == policy(grad=A + 2) == api.ALIGN


def test_refusals_of_preference(lib):
    assert preference(terms=None) == api.INVALID_ARG
    for name, values in dict(beta=(0.0, -1.0, math.inf, math.nan), margin=(math.inf, math.nan), margin_reward=(math.inf, math.nan),
                             smoothing=(-0.1, 1.1, math.nan), nll=(math.inf, math.nan), loss=(-1, 3)).items():
        for v in values:
            assert preference(terms={name: v}) == api.INVALID_ARG, (name, v)
    assert preference(terms=dict(smoothing=0.1, loss=api.PREF_HINGE)) == api.INVALID_ARG
    assert preference(G=0) == api.INVALID_ARG and preference(G=3) == api.SHAPE and preference(G=2048, S=2048) == api.SHAPE
    assert preference(logp=None) == preference(omega=None) == preference(rewards=None) == preference(stats=None) == api.INVALID_ARG
    assert preference(N=-1) == api.ZERO_NORM
    assert preference(logp=A + 2) == preference(pairs=A + 4) == preference(scores=A + 2) == api.ALIGN


def test_terms_are_structs_of_their_call(lib):
    assert api.C.sizeof(api.HilorePolicyTerms) == 6 * 8 + 4 * 4 and api.C.sizeof(api.HilorePreferenceTerms) == 5 * 8 + 2 * 4
    with pytest.raises(TypeError, match="HilorePolicyTerms"):
        api.hilore_policy_loss(A, A, A, None, A, A, None, A, 4, 64, api.make_preference_terms(), 7, None, None, A, A, A, 1 << 20, stream=0)
    with pytest.raises(TypeError, match="HilorePreferenceTerms"):
        api.hilore_preference_loss(A, A, A, A, 2, A, 4, 64, api.make_policy_terms(), 0, None, None, None, None, A, A, A, 1 << 20, stream=0)


def test_workspaces_grow_with_the_call(lib):
    for f in (lambda n: api.hilore_advantages_workspace_bytes(n), lambda n: api.hilore_policy_loss_workspace_bytes(n, n),
              lambda n: api.hilore_preference_loss_workspace_bytes(n, n)):
        sizes = [f(n) for n in (0, 1, 4096, 10 ** 6, BIG)]
        assert all(0 < a <= b for a, b in zip(sizes, sizes[1:])) and f(-5) == f(0)
