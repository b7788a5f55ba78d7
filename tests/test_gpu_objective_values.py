"""Policy and preference loss at values that are not finite or hardly larger than nothing: infinite advantages on flat branches, tokens
that could not be sampled, responses that win nothing."""
import math

import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api
from tests import test_gpu_objective as T

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF, NAN = math.inf, math.nan


def case(lengths, masked=None, seed=0):
    c = T.Call("one token", seed=seed)
    c.bounds = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    c.S, c.n = len(lengths), int(c.bounds[-1])
    c.live, c.cu = c.n, T.G.dev(c.bounds.astype(np.int32))
    c.mask = None if masked is None else (c.rng.random(c.n) >= masked).astype(np.uint8)
    return c


# ------------------------------------------------------------------------------------------------------- preference loss
def pairs_of(c, x, t, group):
    """Winners and losers, scores, means, and the loss of each pair, one after the other in 64 bits."""
    lp = x["logp"].astype(np.float64)
    d = lp - (0.0 if x["ref"] is None else x["ref"].astype(np.float64))
    valid = np.ones(c.n, bool) if c.mask is None else c.mask > 0
    at = [np.flatnonzero(valid[a:b]) + a for a, b in zip(c.bounds[:-1], c.bounds[1:])]
    h = np.array([t["beta"] * (d[a].mean() if t["length_mean"] else d[a].sum()) for a in at])
    mean = np.array([lp[a].mean() for a in at])
    R, found = x["rewards"], []
    for i in range(c.S):
        for j in range(i // group * group, i // group * group + group):
            if R[i] > R[j]:
                z = h[i] - h[j]
                sm = t["smoothing"]
                lose, win = (0.0 if q == INF else -q if q < -700 else math.log1p(math.exp(-q)) for q in (z, -z))
                each = {0: (lose if sm < 1 else 0.0) * (1 - sm) + (sm * win if sm else 0.0), 1: max(0.0, 1 - z), 2: ((z - 0.5) / t["beta"]) ** 2}[t["loss"]]
                found.append((i, j, z, each))
    return found, h, mean


@pytest.mark.parametrize("group", [2, 16, 300])  # threads of their own, teams, a group over several CTAs
@pytest.mark.parametrize("loss,length_mean,nll", [(0, 0, 0.0), (0, 1, 0.3), (1, 0, 0.3)])
def test_a_loser_with_a_token_that_could_not_be_sampled(group, loss, length_mean, nll):
    """Its score is -infinity and every pair with it is in order: loss, order and the winners' likelihood are as finite as they are."""
    c = case([3, 5] * group, seed=group)
    t = dict(T.PREF, loss=loss, length_mean=length_mean, nll=nll)
    x = T.preference_inputs(c)
    x["rewards"] = np.tile(np.arange(group, dtype=np.float32), 2)
    x["logp"][c.bounds[group]] = -INF  # the first response of the second group, which wins nothing
    T.run_preference(c, x, t, group)
    found, h, mean = pairs_of(c, x, t, group)
    N = len(found)
    assert N == group * (group - 1) and int(c.got("pairs", np.int64)[0]) == N
    nlls = sum(-mean[i] for i, *_ in found) / N
    want = [sum(p[3] for p in found) / N + nll * nlls, sum(p[2] > 0 for p in found) / N, INF, nlls]
    T.close(c.got("stats"), want, [1.01 * U * abs(w) + 1e-9 if math.isfinite(w) else 0 for w in want], "stats")
    assert np.isfinite(c.got("omega")).all() and np.isneginf(c.got("scores")[group])


@pytest.mark.parametrize("bad", [-INF, NAN])
@pytest.mark.parametrize("group", [2, 16, 300])
def test_a_response_without_a_pair_changes_nothing(bad, group):
    """All rewards of its group are equal: whatever its log-probabilities are, no statistic and no gradient has anything of it."""
    t = dict(T.PREF, nll=0.5, length_mean=1)
    found = []
    for value in (-1.0, bad):
        c = case([4] * (2 * group), seed=3)
        x = T.preference_inputs(c)
        x["rewards"] = np.concatenate([np.zeros(group), np.arange(group)]).astype(np.float32)
        x["logp"][5] = value
        T.run_preference(c, x, t, group)
        found.append([c.got(k).tobytes() for k in ("stats", "omega")])
        assert np.isfinite(c.got("stats")).all() and c.got("stats")[3] > 0
    assert found[0] == found[1]
    c = case([4] * group, seed=3)  # and alone in its call
    x = dict(T.preference_inputs(c), rewards=np.zeros(group, np.float32))
    x["logp"][2] = bad
    T.run_preference(c, x, t, group)
    assert not c.got("stats").any() and not c.got("omega").any() and int(c.got("pairs", np.int64)[0]) == 0


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 0.5, 1.0])
@pytest.mark.parametrize("sign", [-1, 1])
def test_smoothing_at_infinite_gaps(smoothing, sign):
    """-(1 - e) ln sigma(z) - e ln sigma(-z) at z of either infinity: infinite unless the infinite logarithm has no weight; the slope is
    e - 1 or e."""
    c = case([4] * 4)
    t = dict(T.PREF, smoothing=smoothing, beta=0.5)
    x = dict(T.preference_inputs(c), rewards=np.array([1, 0, 0, 1], np.float32))  # the second pair is finite
    x["logp"][1 if sign < 0 else 5] = -INF  # of the winner or the loser
    T.run_preference(c, x, t, 2)
    stats, omega = c.got("stats"), c.got("omega")
    weight = 1 - smoothing if sign < 0 else smoothing  # of the infinite logarithm
    found, h, _ = pairs_of(c, x, t, 2)
    if weight:
        assert np.isposinf(stats[0])
    else:
        want = found[1][3] / 2  # the finite pair's loss, as the other one's is 0
        T.close(stats[:1], [want], [1.01 * U * abs(want)])
    slope = (smoothing - 1 if sign < 0 else smoothing) * 0.5 / 2
    T.close(omega[:8], np.repeat([slope, -slope], 4), 1.01 * U * abs(slope) + 1e-45)
    assert stats[1] == (0 if sign < 0 else 0.5) + 0.5 * (found[1][2] > 0)


def test_smoothing_of_ordinary_gaps_against_the_definition():
    """Both logarithms with their weights, from gaps of 2^-30 to some hundreds on either side."""
    r = np.random.default_rng(1)
    gaps = np.concatenate([r.normal(0, 1, 40), r.normal(0, 100, 20), [2.0 ** -30, -2.0 ** -30, 0.0, 40.0, -40.0]])
    for smoothing in (0.0, 0.25, 1.0):
        t = dict(T.PREF, smoothing=smoothing, beta=1.0)
        for gap in gaps:
            c = case([1, 1])
            x = dict(logp=np.array([gap, 0.0], np.float32), ref=None, rewards=np.array([1, 0], np.float32))
            T.run_preference(c, x, t, 2)
            z = float(x["logp"][0])
            want = (1 - smoothing) * np.logaddexp(0, -z) + smoothing * np.logaddexp(0, z)
            T.close(c.got("stats")[:1], [want], [U * abs(want) * 1.01 + 1e-45])


# ----------------------------------------------------------------------------------------------------------- policy loss
FLAT = [(1.0, 0.6), (-1.0, -0.6), (-1.0, 0.9)]            # sign of the advantage, s - s_old: beyond 1.28, below 0.8, beyond a dual clip of 2
OPEN = [(1.0, -0.6), (1.0, 0.1), (-1.0, 0.3), (-1.0, 0.0)]  # and on no bound


def policy_case(tokens, ratio, per_token, near, rollout=False, mean=0):
    """A sequence of 16 equal tokens for each (advantage, s - s_old), among ordinary ones in blocks of 256 tokens.  near: every block has
    a token whose ratio is a rounding from its bound, so that sides are decided in 64 bits, and one whose reference is far away."""
    t = dict(T.TERMS, dual_clip=2.0, beta=0.0, ratio=ratio, mean=mean, adv_per_token=int(per_token))
    seqs = [(float(x), 0.05) for x in np.random.default_rng(0).normal(size=40)]
    at = [3, 12, 21, 30, 39, 10, 19]
    for i, k in enumerate(tokens):
        seqs[at[i]] = k
    c = case([16] * 40)
    d = np.repeat([k[1] for k in seqs], 16).astype(np.float32)
    x = dict(logp=np.zeros(c.n, np.float32), old=-d, ref=None, rollout=-d if rollout else None, white=None,
             adv=np.array([k[0] for k in seqs], np.float32))
    if near:
        x["old"][::128] = -np.float32(math.log1p(0.28))  # the sequences of these tokens are numbers 0, 8, 16, 24, 32
        x["ref"] = x["logp"] - np.float32(0.1)
        x["ref"][::128] = 5.0
    if per_token:
        x["adv"] = np.repeat(x["adv"], 16)
    where = np.zeros(c.n, bool)
    for i in at[:len(tokens)]:
        where[16 * i:16 * i + 16] = True
    assert not where[::128].any()
    return c, t, x, where


FORMS = [(0, True, 0), (0, True, 1), (0, False, 0), (0, False, 1), (1, False, 0), (1, False, 1)]  # ratio, advantages per token, mean


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("ratio,per_token,mean", FORMS)
@pytest.mark.parametrize("size", [INF, 1.4e-45, 3.4e38])
def test_flat_branches_of_advantages_of_any_size(size, ratio, per_token, mean, near):
    """The gradient there is exactly zero and the tokens count as clipped, whatever their neighbours hold."""
    c, t, x, where = policy_case([(s * size, d) for s, d in FLAT], ratio, per_token, near, mean=mean)
    T.run_policy(c, x, t, 100, grad=2.0 ** 20)
    omega, stats = c.got("omega"), c.got("stats")
    assert not omega[where].any() and np.isfinite(omega).all()
    w = 1 / 100 if mean == 0 else 1 / 1600
    share = 48 * w
    if near and ratio == 0:  # ln 1.28 in fp32 is beyond or not, and the others' advantages have either sign
        beyond = float(np.float32(math.log1p(0.28))) > math.log1p(0.28)
        A = x["adv"][::128] if per_token else x["adv"][::8]
        share += w * (A > 0).sum() * beyond
    T.close(stats[3:4], [share], 100 * U * share)


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("ratio,per_token,mean", FORMS)
def test_infinite_advantages_on_no_bound_show(ratio, per_token, mean, near):
    c, t, x, where = policy_case([(s * INF, d) for s, d in OPEN], ratio, per_token, near, mean=mean)
    T.run_policy(c, x, t, 100)
    A = x["adv"] if per_token else np.repeat(x["adv"], 16)
    omega = c.got("omega")
    assert np.isinf(omega[where]).all() and np.isfinite(omega[~where]).all() and (np.sign(omega[where]) == -np.sign(A[where])).all()


@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("ratio,per_token,mean", FORMS)
def test_advantages_that_are_no_number_show_on_either_side_of_the_bounds(ratio, per_token, mean, near):
    c, t, x, where = policy_case([(NAN, d) for _, d in FLAT + OPEN], ratio, per_token, near, mean=mean)
    T.run_policy(c, x, t, 100)
    omega, stats = c.got("omega"), c.got("stats")
    assert np.isnan(omega[where]).all() and np.isfinite(omega[~where]).all() and np.isnan(stats[:2]).all() and np.isfinite(stats[2:]).all()


@pytest.mark.parametrize("mean", [0, 1])
@pytest.mark.parametrize("near", [False, True])
def test_flat_branches_of_tokens_with_tiny_rollout_weights(near, mean):
    """Rollout weights of exp(-79) times small advantages leave the range of normal numbers: still flat, still counted."""
    c, t, x, where = policy_case([(s * 1e-10, d) for s, d in FLAT], 0, True, near, rollout=True, mean=mean)
    x["rollout"][where] = x["old"][where] + 79.0
    T.run_policy(c, x, t, 100, grad=2.0 ** 20)
    assert not c.got("omega")[where].any()
    count = 48 + (near and float(np.float32(math.log1p(0.28))) > math.log1p(0.28)) * (x["adv"][::128] > 0).sum()
    share = count * (1 / 100 if mean == 0 else 1 / 1600)
    T.close(c.got("stats")[3:4], [share], 100 * U * share)


@pytest.mark.parametrize("beta", [0.0, 0.05])
@pytest.mark.parametrize("ratio,per_token,mean", FORMS)
def test_results_do_not_depend_on_what_makes_a_block_look_closer(ratio, per_token, mean, beta):
    """The same tokens beside a neighbour that is next to a bound, and beside one that is not: the same bits."""
    found = []
    for shift in (0.0, 0.02):
        r = np.random.default_rng(2)
        t = dict(T.TERMS, dual_clip=2.0, beta=beta, ratio=ratio, mean=mean, adv_per_token=int(per_token))
        c = case([16] * 40)
        x = dict(logp=np.zeros(c.n, np.float32), old=r.normal(0, 0.5, c.n).astype(np.float32), ref=r.normal(0, 0.5, c.n).astype(np.float32), white=None,
                 rollout=None, adv=r.normal(size=c.n if per_token else c.S).astype(np.float32))
        x["rollout"] = (x["old"] + r.normal(0, 0.05, c.n)).astype(np.float32)
        x["old"][::128] = -np.float32(math.log1p(0.28)) - np.float32(shift)
        T.run_policy(c, x, t, 100)
        keep = np.ones(c.n, bool)
        keep[::128] = False
        if ratio:  # their sequences move with them
            keep = ~np.repeat(np.arange(40) % 8 == 0, 16)
        found.append(c.got("omega")[keep])
    assert np.array_equal(*found)


@pytest.mark.parametrize("ratio,per_token,mean", FORMS)
@pytest.mark.parametrize("far", ["ratio", "weight", "both"])
def test_advantages_of_nothing_at_ratios_beyond_every_number(ratio, per_token, mean, far):
    """Without bounds a ratio of exp(800) is infinite in any type here; times an advantage of 0 it is nothing."""
    t = dict(T.TERMS, clip_high=INF, rollout_cap=INF, beta=0.0, ratio=ratio, mean=mean, adv_per_token=int(per_token))
    for d in (100.0, 800.0):
        c, _, x, where = policy_case([(0.0, 0.0)], ratio, per_token, False, rollout=True, mean=mean)
        if far != "weight":
            x["logp"][where] += np.float32(d)
        if far != "ratio":
            x["rollout"][where] -= np.float32(d)
        T.run_policy(c, x, t, 100)
        omega, stats = c.got("omega"), c.got("stats")
        assert not omega[where].any() and np.isfinite(omega).all() and omega.any() and np.isfinite(stats).all()
