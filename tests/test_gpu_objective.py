"""Advantages with their backward pass, policy loss and preference loss against the definitions in 64 bits (tests/objective_ref.py),
at the lengths, masks, types, addresses and values where they can go wrong."""
import math

import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api
from tests import gpu_util as G
from tests import objective_ref as R

pytestmark = pytest.mark.gpu

TILE = 2048  # tokens of a CTA
LENGTHS = {
    "one token": [1],
    "few": [3, 0, 1, 8, 7, 9, 0, 0, 2],
    "all empty": [0, 0, 0],
    "tile edges": [TILE - 1, 1, TILE, TILE + 1, 0, 5, TILE - 6, 2 * TILE],
    "many short": [1, 0, 2, 0, 0, 3, 1] * 700,
    "across tiles": [9000, 3, 7001, 0, 517],
    "over 32 tiles": [33 * TILE + 77, 40, 12 * TILE],
    "rows": None,
}


def bounds_of(name):
    lengths = [37] * 61 if name == "rows" else LENGTHS[name]
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


class Call:
    """Inputs on the device, `shift` elements off a 256-byte boundary; guarded outputs likewise."""

    def __init__(self, name, shift=0, seed=0, masked=0.3, beyond=0):
        self.bounds = bounds_of(name)
        self.S, self.live = len(self.bounds) - 1, int(self.bounds[-1])
        self.n = self.live + beyond
        self.shift = shift
        self.rng = np.random.default_rng(seed)
        self.cu = None if name == "rows" else G.dev(self.bounds.astype(np.int32))
        self.mask = None if masked is None else (self.rng.random(self.n) >= masked).astype(np.uint8)
        self.outputs = {}

    def put(self, a, shift=None):
        if a is None:
            return None
        a = torch.from_numpy(np.ascontiguousarray(a)) if not isinstance(a, torch.Tensor) else a
        shift = self.shift if shift is None else shift
        buf = torch.zeros(a.numel() + shift + 8, dtype=a.dtype, device="cuda")
        view = buf[shift:shift + a.numel()]
        view.copy_(a)
        return view

    def out(self, name, count, size=4):
        g = G.Guarded((count + self.shift) * size)
        self.outputs[name] = (g, count)
        return g.ptr() + self.shift * size

    def got(self, name, dtype=np.float32):
        g, count = self.outputs[name]
        whole = g.numpy(dtype, (count + self.shift,))
        assert (whole[:self.shift].view(np.uint8) == G.CANARY).all()
        return whole[self.shift:]

    def left_alone(self, name):
        """What lies behind the last sequence is as it was."""
        return (self.got(name)[self.live:].view(np.uint8) == G.CANARY).all()

    def normal(self, n=None, std=1.0, mean=0.0):
        return self.rng.normal(mean, std, self.n if n is None else n).astype(np.float32)


def close(got, want, tol, what=""):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), what
    ok = np.isfinite(want)
    off = np.abs(got - want)[ok]
    bad = off > np.broadcast_to(tol, want.shape)[ok]
    assert not bad.any(), (what, int(bad.sum()), float(off[bad].max()), np.flatnonzero(ok)[bad][:5])


def once(x):
    return R.U * np.abs(x) * 1.0001 + 1e-45  # one rounding to fp32


# ------------------------------------------------------------------------------------------------------------ advantages
def run_advantages(c, x, gamma, lam, moments=True, stream=None, both=True):
    ws = torch.empty(api.hilore_advantages_workspace_bytes(c.n), dtype=torch.uint8, device="cuda")
    x = {k: c.put(v, 0 if k in ("outcome", "bootstrap") else None) for k, v in x.items()}
    dtype = api.BF16 if x["values"] is not None and x["values"].dtype == torch.bfloat16 else api.F32
    adv, ret = c.out("adv", c.n), c.out("returns", c.n) if both else None
    mom = c.out("moments", 2)
    api.hilore_advantages(x["rewards"], x["outcome"], x["values"], dtype, x["bootstrap"], x["trace"], c.put(c.mask), c.cu, c.S, c.n, gamma, lam, adv, ret,
                          mom if moments else None, ws, ws.numel(), stream=stream)
    torch.cuda.synchronize()


def check_advantages(c, x, gamma, lam):
    values = None if x["values"] is None else x["values"].double().numpy() if isinstance(x["values"], torch.Tensor) else x["values"]
    adv, ret, (mean, std), slack = R.advantages(x["rewards"], x["outcome"], values, x["bootstrap"], x["trace"], c.mask, c.bounds, c.n, gamma, lam)
    for name, want in (("adv", adv), ("returns", ret)):
        close(c.got(name)[:c.live], want[:c.live], (once(want) + slack)[:c.live], name)
        assert c.left_alone(name)
    live = adv[:c.live][(np.ones(c.n, bool) if c.mask is None else c.mask > 0)[:c.live]]
    # fp64 sums over the unrounded advantages: the variance is off by what they are, twice
    size = np.abs(live).max(initial=0.0) + slack.max(initial=0.0)
    e = (len(live) + 50) * R.E * (1 + size) + slack.max(initial=0.0)
    got = c.got("moments")
    close(got[:1], [mean], once(mean) + e)
    close(got[1:] ** 2.0, [std ** 2], 4 * R.U * std ** 2 + 4 * e * (1 + size))


def reward_inputs(c, values="f32", trace=False):
    v = c.normal(std=0.5, mean=0.3)
    return dict(rewards=c.normal(std=0.1), outcome=c.normal(c.S), values=torch.from_numpy(v).to(torch.bfloat16) if values == "bf16" else v,
                bootstrap=c.normal(c.S), trace=c.rng.uniform(0.0, 1.0, c.n).astype(np.float32) if trace else None)


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("values,trace,gamma,lam", [("f32", False, 1.0, 0.95), ("bf16", True, 0.99, 1.0), ("f32", False, 1.0, 1.0)])
def test_advantages(name, values, trace, gamma, lam):
    c = Call(name, seed=len(name))
    x = reward_inputs(c, values, trace)
    run_advantages(c, x, gamma, lam)
    check_advantages(c, x, gamma, lam)


@pytest.mark.parametrize("shift", [1, 3, 4])
@pytest.mark.parametrize("name", ["few", "tile edges", "across tiles", "rows"])
def test_advantages_at_any_address_are_the_same_bits(name, shift):
    found = []
    for s in (0, shift):
        c = Call(name, shift=s, seed=3, beyond=0 if name == "rows" else 1000)
        x = reward_inputs(c, "bf16", True)
        run_advantages(c, x, 0.99, 0.9)
        check_advantages(c, x, 0.99, 0.9)
        found.append([c.got(k).tobytes() for k in ("adv", "returns", "moments")])
    assert found[0] == found[1]


@pytest.mark.parametrize("masked", [None, 0.0, 0.999, 1.0])
def test_advantages_of_masks(masked):
    c = Call("across tiles", masked=masked)
    x = reward_inputs(c)
    run_advantages(c, x, 0.999, 0.98)
    check_advantages(c, x, 0.999, 0.98)


@pytest.mark.parametrize("gamma,lam", [(0.0, 1.0), (1.0, 0.0), (0.0, 0.0)])
def test_advantages_without_memory(gamma, lam):
    c = Call("across tiles")
    x = reward_inputs(c)
    run_advantages(c, x, gamma, lam)
    check_advantages(c, x, gamma, lam)


def test_rewards_alone_and_values_alone():
    for keep in ("rewards", "values", "outcome", "bootstrap"):
        c = Call("tile edges")
        x = {k: v if k == keep else None for k, v in reward_inputs(c).items()}
        run_advantages(c, x, 0.99, 0.9)
        check_advantages(c, x, 0.99, 0.9)


def test_outputs_are_optional():
    c = Call("few")
    x = reward_inputs(c)
    run_advantages(c, x, 0.9, 0.9, moments=False, both=False)
    adv, *_, slack = R.advantages(*[x[k] for k in ("rewards", "outcome", "values", "bootstrap", "trace")], c.mask, c.bounds, c.n, 0.9, 0.9)
    close(c.got("adv"), adv, once(adv) + slack)
    assert (c.got("moments").view(np.uint8) == G.CANARY).all()


def test_masked_tokens_may_hold_anything():
    c = Call("across tiles", seed=9)
    x = reward_inputs(c, trace=True)
    clean = {k: v.copy() for k, v in x.items()}
    hidden = c.mask == 0
    for k, bad in (("rewards", np.nan), ("values", np.inf), ("trace", -np.inf)):
        x[k][hidden] = bad
    run_advantages(c, x, 0.99, 0.9)
    check_advantages(c, clean, 0.99, 0.9)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_what_is_not_finite_stays_in_its_sequence(bad):
    c = Call("tile edges", seed=4, masked=None)
    x = reward_inputs(c)
    at = int(c.bounds[3]) + 900  # in the sequence of TILE + 1 tokens
    x["rewards"][at] = bad
    run_advantages(c, x, 1.0, 0.95)
    got = c.got("adv")
    clean = dict(x, rewards=np.where(np.arange(c.n) == at, 0, x["rewards"]))
    want, *_, slack = R.advantages(*[clean[k] for k in ("rewards", "outcome", "values", "bootstrap", "trace")], c.mask, c.bounds, c.n, 1.0, 0.95)
    hit = np.zeros(c.n, bool)
    hit[int(c.bounds[3]):at + 1] = True
    assert not np.isfinite(got[hit]).any()
    close(got[~hit], want[~hit], (once(want) + slack)[~hit])


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("trace", [False, True])
def test_what_is_not_finite_stays_in_its_short_sequence(bad, trace):
    """Many sequences to a block: nothing comes through their ends, forward or backward."""
    c = Call("many short", seed=5, masked=0.2)
    c.bounds = np.concatenate([[0], np.cumsum(np.tile([40, 1, 0, 7, 3, 30], 40))])
    c.S, c.n = len(c.bounds) - 1, int(c.bounds[-1])
    c.live, c.cu = c.n, G.dev(c.bounds.astype(np.int32))
    c.mask = (c.rng.random(c.n) >= 0.2).astype(np.uint8)
    x = reward_inputs(c, trace=trace)
    seqs = [3, 6, 60, 100, 150, 201]  # of seven, forty and one tokens
    at = np.array([int(c.bounds[s + 1]) - 1 - (int(c.bounds[s + 1] - c.bounds[s]) > 2) for s in seqs])
    c.mask[at] = 1
    x["rewards"][at] = bad
    run_advantages(c, x, 1.0, 0.95, moments=False)
    got = c.got("adv")
    clean = dict(x, rewards=np.where(np.isin(np.arange(c.n), at), 0, x["rewards"]))
    want, *_, slack = R.advantages(*[clean[k] for k in ("rewards", "outcome", "values", "bootstrap", "trace")], c.mask, c.bounds, c.n, 1.0, 0.95)
    hit = np.zeros(c.n, bool)
    for s, t in zip(seqs, at):
        hit[c.bounds[s]:t + 1] = c.mask[c.bounds[s]:t + 1] > 0
    assert not np.isfinite(got[hit]).any()
    close(got[~hit], want[~hit], (once(want) + slack)[~hit])
    back = dict(ga=c.normal(), gr=c.normal(), adv=c.normal(), trace=x["trace"])
    back["ga"][at] = bad
    names = run_backward(c, back, 1.0, 0.95)
    ga = np.where(np.isin(np.arange(c.n), at), 0, back["ga"]).astype(np.float32)
    want, slack = R.advantages_backward(ga, back["gr"], back["adv"], back["trace"], c.mask, c.bounds, c.n, 1.0, 0.95)
    hit = np.zeros(c.n, bool)
    for s, t in zip(seqs, at):
        hit[t:c.bounds[s + 1]] = True
    for k in names:
        ok = ~hit if k in ("rewards", "values", "trace") else ~np.isin(np.arange(c.S), seqs)
        close(c.got(k)[ok], want[k][ok], (once(want[k]) + slack[k])[ok], k)
        assert not np.isfinite(c.got("rewards")[at]).any()


def run_backward(c, x, gamma, lam, only=None):
    ws = torch.empty(api.hilore_advantages_workspace_bytes(c.n), dtype=torch.uint8, device="cuda")
    p = {k: c.put(v) for k, v in x.items()}
    sizes = dict(rewards=c.n, outcome=c.S, values=c.n, bootstrap=c.S, trace=c.n)
    o = {k: c.out(k, m) if only is None or k in only else None for k, m in sizes.items()}
    api.hilore_advantages_backward(p["ga"], p["gr"], p["adv"], p["trace"], c.put(c.mask), c.cu, c.S, c.n, gamma, lam, o["rewards"], o["outcome"], o["values"],
                                   o["bootstrap"], o["trace"], ws, ws.numel())
    torch.cuda.synchronize()
    return [k for k in sizes if o[k]]


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("trace,gamma,lam,shift", [(True, 0.99, 0.95, 0), (False, 1.0, 1.0, 3), (True, 0.0, 1.0, 0)])
def test_advantages_backward(name, trace, gamma, lam, shift):
    c = Call(name, seed=len(name), shift=shift, beyond=0 if name == "rows" else 700)
    x = dict(ga=c.normal(), gr=c.normal(), adv=c.normal(), trace=c.rng.uniform(0.0, 1.0, c.n).astype(np.float32) if trace else None)
    names = run_backward(c, x, gamma, lam)
    want, slack = R.advantages_backward(x["ga"], x["gr"], x["adv"], x["trace"], c.mask, c.bounds, c.n, gamma, lam)
    for k in names:
        m = c.live if k in ("rewards", "values", "trace") else c.S
        close(c.got(k)[:m], want[k][:m], (once(want[k]) + slack[k])[:m], k)
        if m == c.live:
            assert c.left_alone(k)


@pytest.mark.parametrize("only", [["rewards"], ["values"], ["trace"], ["outcome"], ["bootstrap"]])
def test_single_gradients(only):
    c = Call("tile edges", seed=2)
    x = dict(ga=c.normal(), gr=None, adv=c.normal() if "trace" in only else None, trace=None)
    assert run_backward(c, x, 0.9, 0.8, only) == only
    want, slack = R.advantages_backward(x["ga"], None, x["adv"], None, c.mask, c.bounds, c.n, 0.9, 0.8)
    close(c.got(only[0]), want[only[0]], once(want[only[0]]) + slack[only[0]])


def test_backward_against_differences_of_the_kernel():
    """The sum of gA A is linear in rewards and values: its change over a whole step is the gradient times the step."""
    c = Call("across tiles", seed=11)
    x = reward_inputs(c)
    run_advantages(c, x, 0.99, 0.95)
    ga, base = c.normal() * c.mask, c.got("adv").astype(np.float64)
    g = Call("across tiles", seed=11)
    run_backward(g, dict(ga=ga, gr=None, adv=None, trace=None), 0.99, 0.95, ["rewards", "values"])
    for name in ("rewards", "values"):
        step = c.normal()
        run_advantages(c, dict(x, **{name: x[name] + step}), 0.99, 0.95)
        moved = c.got("adv").astype(np.float64)
        real = (x[name] + step).astype(np.float64) - x[name]  # the step that fp32 took
        grads = g.got(name).astype(np.float64)
        # three results of one rounding each; products of numbers known to a rounding
        tol = R.U * ((np.abs(ga) * (np.abs(base) + np.abs(moved))).sum() + (np.abs(grads) * np.abs(real)).sum()) + 1e-9
        assert abs((ga * (moved - base)).sum() - (grads * real * c.mask).sum()) < tol


# ----------------------------------------------------------------------------------------------------------- policy loss
TERMS = dict(clip_low=0.2, clip_high=0.28, dual_clip=0.0, beta=0.05, rollout_cap=1.05, adv_eps=1e-6, ratio=0, mean=0, kl=3, adv_per_token=0)


def policy_inputs(c, t, ref=True, rollout=False, white=False, spread=0.2):
    lp = c.normal(std=0.7, mean=-1.5)
    old = lp + c.normal(std=spread) if t["ratio"] == 0 else lp + np.repeat(c.normal(c.S, spread), np.diff(np.append(c.bounds[:-1], c.n))).astype(np.float32)
    return dict(logp=lp, old=old, ref=lp + c.normal(std=0.3) if ref else None, rollout=old + c.normal(std=0.05) if rollout else None,
                adv=c.normal() if t["adv_per_token"] else c.normal(c.S), white=np.array([0.2, 0.9], np.float32) if white else None)


def run_policy(c, x, t, N, grad=None, N_dev=False, stream=None):
    ws = torch.empty(api.hilore_policy_loss_workspace_bytes(c.S, c.n), dtype=torch.uint8, device="cuda")
    p = {k: c.put(v, 0 if k == "white" or (k == "adv" and not t["adv_per_token"]) else None) for k, v in x.items()}
    dev = torch.tensor([N], dtype=torch.int64, device="cuda") if N_dev else None
    g = None if grad is None else torch.tensor([grad], dtype=torch.float32, device="cuda")
    api.hilore_policy_loss(p["logp"], p["old"], p["ref"], p["rollout"], c.put(c.mask), p["adv"], p["white"], c.cu, c.S, c.n, api.make_policy_terms(**t),
                           0 if N_dev else N, dev, g, c.out("stats", 5), c.out("omega", c.n), ws, ws.numel(), stream=stream)
    torch.cuda.synchronize()


def check_policy(c, x, t, N, grad=1.0):
    stats, omega, slack, tol = R.policy(x["logp"], x["old"], x["ref"], x["rollout"], c.mask, x["adv"], x["white"], c.bounds, t, N, grad)
    close(c.got("omega")[:c.live], omega[:c.live], tol[:c.live] + 1e-45, "omega")
    assert c.left_alone("omega")
    close(c.got("stats"), stats, slack * 1.01 + 1e-45, "stats")


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("ratio,mean,kl,per_token", [(0, 0, 3, 1), (0, 1, 2, 0), (1, 1, 3, 0), (1, 0, 1, 0)])
def test_policy(name, ratio, mean, kl, per_token):
    t = dict(TERMS, ratio=ratio, mean=mean, kl=kl, adv_per_token=per_token)
    c = Call(name, seed=ratio + 2 * mean)
    x = policy_inputs(c, t)
    run_policy(c, x, t, 1234)
    check_policy(c, x, t, 1234)


@pytest.mark.parametrize("ratio,mean,per_token", [(0, 0, 1), (0, 1, 1), (0, 1, 0), (1, 1, 0)])
@pytest.mark.parametrize("ref,rollout,white,dual,beta", [(True, True, True, 1.3, 0.1), (False, True, False, 1.0, 0.0), (True, False, True, 0.0, 0.0)])
def test_policy_parts(ratio, mean, per_token, ref, rollout, white, dual, beta):
    t = dict(TERMS, ratio=ratio, mean=mean, adv_per_token=per_token, dual_clip=dual, beta=beta)
    c = Call("tile edges", seed=7, beyond=333, shift=0 if white else 1)
    x = policy_inputs(c, t, ref, rollout, white, spread=0.6)
    run_policy(c, x, t, 77, grad=8.0, N_dev=True)
    check_policy(c, x, t, 77, 8.0)


@pytest.mark.parametrize("ratio,mean", [(0, 0), (0, 1), (1, 1)])
def test_policy_at_any_address_is_the_same_bits(ratio, mean):
    t, found = dict(TERMS, ratio=ratio, mean=mean, adv_per_token=0), []
    for shift in (0, 1, 5):
        c = Call("across tiles", shift=shift, seed=3, beyond=99)
        x = policy_inputs(c, t, rollout=True)
        run_policy(c, x, t, 1000)
        check_policy(c, x, t, 1000)
        found.append([c.got(k).tobytes() for k in ("omega", "stats")])
    assert found[0] == found[1] == found[2]


@pytest.mark.parametrize("ratio", [0, 1])
def test_policy_next_to_the_borders(ratio):
    """Ratios a rounding inside, on and outside each bound: the branch is the formula's, in 64 bits."""
    t = dict(TERMS, clip_low=0.25, clip_high=0.5, dual_clip=2.0, beta=0.0, ratio=ratio, adv_per_token=0)
    steps = [np.log1p(0.5), np.log1p(-0.25), np.log(2.0)]
    d = np.concatenate([[np.float32(v) * np.float32(1 + k * 2.0 ** -23) for k in range(-4, 5)] for v in steps]).astype(np.float32)
    c = Call("one token")
    c.bounds = np.arange(len(d) * 2 + 1, dtype=np.int64)
    c.S = c.n = c.live = len(d) * 2
    c.cu, c.mask = G.dev(c.bounds.astype(np.int32)), None
    # log-probabilities whose difference is d exactly
    x = dict(logp=np.tile(d, 2), old=np.zeros(c.n, np.float32), ref=None, rollout=None, adv=np.repeat([1.0, -1.0], len(d)).astype(np.float32), white=None)
    run_policy(c, x, t, 10)
    check_policy(c, x, t, 10)
    _, omega, *_ = R.policy(*[x[k] for k in ("logp", "old", "ref", "rollout")], None, x["adv"], None, c.bounds, t, 10)
    assert np.array_equal(c.got("omega") == 0, omega == 0) and (omega == 0).any() and (omega != 0).any()


def test_policy_of_tokens_that_could_not_be_sampled():
    """-inf among the log-probabilities: the formula's values, and nothing beyond the tokens concerned."""
    t = dict(TERMS, beta=0.0, adv_per_token=1)
    c = Call("few", masked=None)
    x = policy_inputs(c, t, ref=False)
    x["logp"][4] = -np.inf
    x["adv"][4] = -1.0  # rho = 0 is below the lower bound: flat
    x["old"][6] = -np.inf
    x["adv"][6] = 1.0   # rho = inf is above the upper one: flat
    run_policy(c, x, t, 10)
    stats, omega, _, tol = R.policy(*[x[k] for k in ("logp", "old", "ref", "rollout")], c.mask, x["adv"], None, c.bounds, t, 10)
    assert omega[4] == 0 and omega[6] == 0 and np.isfinite(omega).all()
    close(c.got("omega"), omega, tol + 1e-45)
    assert np.isfinite(c.got("stats")[:4]).all()


def test_policy_masked_tokens_may_hold_anything():
    for ratio, mean in ((0, 0), (0, 1), (1, 1)):
        t = dict(TERMS, ratio=ratio, mean=mean, adv_per_token=1 - ratio)
        c = Call("across tiles", seed=6)
        x = policy_inputs(c, t, rollout=True)
        clean = {k: None if v is None else v.copy() for k, v in x.items()}
        for k, bad in (("logp", np.nan), ("old", -np.inf), ("ref", np.inf), ("rollout", np.nan)):
            x[k][c.mask == 0] = bad
        run_policy(c, x, t, 99)
        check_policy(c, clean, t, 99)


@pytest.mark.parametrize("mean", [0, 1])
def test_policy_of_masked_tokens_whose_advantages_are_whitened_by_nothing(mean):
    """A standard deviation of zero makes valid advantages infinite or NaN; where all are masked nothing may come of it."""
    for per_token in (0, 1):
        t = dict(TERMS, ratio=0, mean=mean, adv_per_token=per_token, adv_eps=0.0)
        for white in ([0.5, 0.0], [np.nan, np.nan], [np.inf, 1.0]):
            c = Call("across tiles", masked=1.0)
            x = policy_inputs(c, t)
            x["white"] = np.array(white, np.float32)
            run_policy(c, x, t, 5)
            assert not c.got("omega").any() and not c.got("stats").any()


@pytest.mark.parametrize("mean", [0, 1])
def test_policy_what_is_not_finite_shows(mean):
    """A NaN advantage makes its own token's gradient NaN; a reference of -infinity without a KL weight nothing at all in the gradient."""
    t = dict(TERMS, ratio=0, mean=mean, adv_per_token=1, beta=0.0, kl=2)
    c = Call("across tiles", masked=None)
    x = policy_inputs(c, t)
    x["adv"][[77, 9100]] = np.nan
    x["ref"][[5, 9200]] = -np.inf
    run_policy(c, x, t, 99)
    omega = c.got("omega")
    assert np.flatnonzero(np.isnan(omega)).tolist() == [77, 9100] and np.isnan(c.got("stats")[:2]).all()


@pytest.mark.parametrize("ratio,mean", [(0, 0), (0, 1), (1, 1)])
def test_policy_of_nothing(ratio, mean):
    t = dict(TERMS, ratio=ratio, mean=mean)
    for name, masked, N in (("all empty", 0.3, 5), ("across tiles", 1.0, 5), ("across tiles", 0.3, 0), ("few", None, -4)):
        c = Call(name, masked=masked)
        x = policy_inputs(c, t)
        run_policy(c, x, t, N, N_dev=True)
        assert not c.got("omega").any() and not c.got("stats").any()


def test_policy_microbatches_add_up():
    """Sequences dealt to two calls with the batch's normaliser: the same gradients bit for bit, statistics that add up."""
    t = dict(TERMS, mean=1, adv_per_token=0)
    whole = Call("across tiles", seed=8)
    x = policy_inputs(whole, t)
    run_policy(whole, x, t, whole.S)
    omega, stats = [], np.zeros(5)
    for a, b in ((0, 2), (2, 5)):
        c = Call("across tiles")
        lo, hi = int(whole.bounds[a]), int(whole.bounds[b])
        c.bounds, c.S, c.n, c.live, c.mask = whole.bounds[a:b + 1] - lo, b - a, hi - lo, hi - lo, whole.mask[lo:hi]
        c.cu = G.dev(c.bounds.astype(np.int32))
        run_policy(c, {k: None if v is None else v[a:b] if k == "adv" else v[lo:hi] for k, v in x.items()}, t, whole.S)
        omega.append(c.got("omega"))
        stats += c.got("stats")
    assert np.array_equal(np.concatenate(omega), whole.got("omega"))
    assert np.abs(stats - whole.got("stats")).max() <= 4 * R.U * np.abs(stats).max()


def test_policy_agrees_with_the_grpo_coefficients():
    rows, T = 16, 512
    rng = np.random.default_rng(1)
    f = lambda std=1.0, mean=0.0, n=rows * T: torch.from_numpy(rng.normal(mean, std, n).astype(np.float32)).cuda()
    lp = f(0.5, -1.5)
    old, ref, rewards = lp + f(0.1), lp + f(0.1), f(n=rows)
    mask = torch.from_numpy((rng.random(rows * T) < 0.8).astype(np.uint8)).cuda()
    adv, want, got, stats = torch.empty(rows, device="cuda"), torch.empty(rows * T, device="cuda"), torch.empty(rows * T, device="cuda"), torch.empty(5, device="cuda")
    N = int(mask.sum())
    api.hilore_grpo_coeffs(rewards, rows, 8, 0, rows, T, lp, old, ref, mask, N, None, 0.2, 0.04, 1e-6, adv, want, None, None)
    ws = torch.empty(api.hilore_policy_loss_workspace_bytes(rows, rows * T), dtype=torch.uint8, device="cuda")
    api.hilore_policy_loss(lp, old, ref, None, mask, adv, None, None, rows, rows * T, api.make_policy_terms(beta=0.04), N, None, None, stats, got, ws, ws.numel())
    # sixteen roundings in each, relative to the two terms of the coefficient; 1 - exp(e) of the other call cancels
    size = (torch.exp(lp - old) * adv.abs().repeat_interleave(T) + 0.04 * (1 + torch.exp(ref - lp))) / N
    near = ((lp - old).exp() - 1.2).abs().minimum(((lp - old).exp() - 0.8).abs()) < 1e-6  # decided in fp32 there, in fp64 here
    assert ((got - want).abs() <= 40 * R.U * size)[~near].all()


# ------------------------------------------------------------------------------------------------------- preference loss
PREF = dict(beta=0.1, margin=0.0, margin_reward=0.0, smoothing=0.0, nll=0.0, loss=0, length_mean=0)


def run_preference(c, x, t, group, N=0, N_dev=None, grad=None, stream=None):
    ws = torch.empty(api.hilore_preference_loss_workspace_bytes(c.S, c.n), dtype=torch.uint8, device="cuda")
    p = {k: c.put(v, 0 if k == "rewards" else None) for k, v in x.items()}
    dev = None if N_dev is None else torch.tensor([N_dev], dtype=torch.int64, device="cuda")
    g = None if grad is None else torch.tensor([grad], dtype=torch.float32, device="cuda")
    api.hilore_preference_loss(p["logp"], p["ref"], c.put(c.mask), p["rewards"], group, c.cu, c.S, c.n, api.make_preference_terms(**t), N, dev, g,
                               c.out("scores", c.S), c.out("pairs", 1, 8), c.out("stats", 4), c.out("omega", c.n), ws, ws.numel(), stream=stream)
    torch.cuda.synchronize()


def check_preference(c, x, t, group, N=0, grad=1.0):
    stats, omega, h, pairs, tol, slack, off = R.preference(x["logp"], x["ref"], c.mask, x["rewards"], group, c.bounds, t, N, grad)
    assert int(c.got("pairs", np.int64)[0]) == pairs
    close(c.got("scores"), h, off * 1.01 + 1e-45, "scores")
    close(c.got("omega")[:c.live], omega[:c.live], tol[:c.live] * 1.01 + 1e-45, "omega")
    assert c.left_alone("omega")
    close(c.got("stats"), stats, slack * 1.01 + 1e-45, "stats")


def preference_inputs(c, ref=True, levels=3):
    lp = c.normal(std=0.7, mean=-1.5)
    return dict(logp=lp, ref=lp + c.normal(std=0.05) if ref else None, rewards=c.rng.integers(0, levels, c.S).astype(np.float32))


GROUPS = {"one token": 1, "few": 3, "all empty": 3, "tile edges": 8, "many short": 7, "across tiles": 5, "over 32 tiles": 3, "rows": 61}


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("loss,length_mean,nll,ref,smoothing", [(0, 0, 0.0, True, 0.0), (0, 1, 0.2, True, 0.1), (1, 1, 0.0, False, 0.0), (2, 0, 0.1, True, 0.0)])
def test_preference(name, loss, length_mean, nll, ref, smoothing):
    t = dict(PREF, loss=loss, length_mean=length_mean, nll=nll, smoothing=smoothing, margin=0.05, margin_reward=0.1, beta=2.0 if length_mean else 0.1)
    c = Call(name, seed=len(name) + loss, shift=loss, beyond=0 if name == "rows" else 50)
    x = preference_inputs(c, ref)
    run_preference(c, x, t, GROUPS[name])
    check_preference(c, x, t, GROUPS[name])


@pytest.mark.parametrize("group", [2, 4, 100, 245, 700])
def test_preference_group_sizes(group):
    c = Call("many short", seed=group)
    x = preference_inputs(c, levels=5)
    t = dict(PREF, beta=0.5)
    c.S, c.bounds = group * (4900 // group), c.bounds[:group * (4900 // group) + 1]
    c.live = int(c.bounds[-1])
    c.cu = G.dev(c.bounds.astype(np.int32))
    x["rewards"] = x["rewards"][:c.S]
    run_preference(c, x, t, group, N=500, grad=0.5)
    check_preference(c, x, t, group, 500, 0.5)


def test_preference_normalisers():
    t = dict(PREF, nll=0.3)
    for N, N_dev, want in ((40, None, 40), (0, 25, 25), (9, 25, 25), (0, 0, None), (0, -3, None)):
        c = Call("tile edges", seed=1)
        x = preference_inputs(c)
        run_preference(c, x, t, 4, N=N, N_dev=N_dev)
        check_preference(c, x, t, 4, want)


def test_preference_without_pairs_and_odd_rewards():
    c = Call("tile edges", seed=1)
    x = dict(preference_inputs(c), rewards=np.full(c.S, 0.5, np.float32))
    run_preference(c, x, PREF, 8)
    check_preference(c, x, PREF, 8)
    assert not c.got("omega").any() and not c.got("stats").any()
    x["rewards"] = np.array([np.nan, np.inf, 0.0, -0.0, -np.inf, np.nan, 1.0, 1e-40], np.float32)
    run_preference(c, x, PREF, 8)
    check_preference(c, x, PREF, 8)


def test_preference_far_scores():
    """Gaps of hundreds either way: the loss is the gap, the slope 0 or 1, nothing overflows."""
    c = Call("few", masked=None, seed=3)
    x = dict(logp=c.normal(std=300.0), ref=c.normal(std=300.0), rewards=np.arange(c.S, dtype=np.float32))
    for loss in (0, 1, 2):
        t = dict(PREF, beta=5.0, loss=loss, smoothing=0.1 if loss == 0 else 0.0)
        run_preference(c, x, t, 9)
        check_preference(c, x, t, 9)


def test_preference_masked_tokens_may_hold_anything():
    c = Call("across tiles", seed=6)
    x = preference_inputs(c)
    clean = {k: v.copy() for k, v in x.items()}
    x["logp"][c.mask == 0], x["ref"][c.mask == 0] = np.nan, -np.inf
    run_preference(c, x, PREF, 5)
    check_preference(c, clean, PREF, 5)


def test_preference_not_finite_stays_in_its_group():
    t = dict(PREF, length_mean=1)
    c = Call("rows", masked=None, seed=6)
    c.S, c.bounds = 60, c.bounds[:61]
    c.n = c.live = 60 * 37
    x = {k: v[:c.S if k == "rewards" else c.n] for k, v in preference_inputs(c).items()}
    clean = {k: v.copy() for k, v in x.items()}
    x["logp"][37 * 13 + 5] = np.nan  # in the group of responses 12 .. 15
    run_preference(c, x, t, 4, N=30)
    _, omega, *_, tol, _, _ = R.preference(clean["logp"], clean["ref"], None, clean["rewards"], 4, c.bounds, t, 30)
    other = np.ones(c.n, bool)
    other[37 * 12:37 * 16] = False
    close(c.got("omega")[other], omega[other], tol[other] * 1.01 + 1e-45)
    assert np.isnan(c.got("scores")[13]) and np.isfinite(np.delete(c.got("scores"), 13)).all()


# ------------------------------------------------------------------------------------- streams, graphs, boundaries, devices
def everything(c, inputs, ws, out, stream=None):
    """Advantages with moments, the whitened policy loss on them, the preference loss, and the advantages' gradient from omega."""
    api.hilore_advantages(inputs["rewards"], None, inputs["values"], api.F32, None, None, inputs["mask"], inputs["cu"], c.S, c.n, 1.0, 0.95, out["adv"],
                          out["returns"], out["moments"], ws, ws.numel(), stream=stream)
    terms = api.make_policy_terms(beta=0.1, mean=api.MEAN_SEQUENCES, adv_per_token=True)
    api.hilore_policy_loss(inputs["logp"], inputs["old"], inputs["ref"], None, inputs["mask"], out["adv"], out["moments"], inputs["cu"], c.S, c.n, terms, c.S,
                           None, None, out["stats"], out["omega"], ws, ws.numel(), stream=stream)
    api.hilore_preference_loss(inputs["logp"], inputs["ref"], inputs["mask"], inputs["verdict"], 1 if c.S % 2 else 2, inputs["cu"], c.S, c.n,
                               api.make_preference_terms(), 0, None, None, out["scores"], out["pairs"], out["pref_stats"], out["pref_omega"], ws, ws.numel(),
                               stream=stream)
    api.hilore_advantages_backward(out["omega"], None, out["adv"], None, inputs["mask"], inputs["cu"], c.S, c.n, 1.0, 0.95, out["d_rewards"], out["d_outcome"],
                                   out["d_values"], None, out["d_trace"], ws, ws.numel(), stream=stream)


def buffers(c):
    z = lambda n, dtype=torch.float32: torch.full((n,), -7, dtype=dtype, device="cuda")
    out = {k: z(c.n) for k in ("adv", "returns", "omega", "pref_omega", "d_rewards", "d_values", "d_trace")}
    out.update(moments=z(2), stats=z(5), pref_stats=z(4), scores=z(c.S), d_outcome=z(c.S), pairs=z(1, torch.int64))
    size = max(api.hilore_advantages_workspace_bytes(c.n), api.hilore_policy_loss_workspace_bytes(c.S, c.n),
               api.hilore_preference_loss_workspace_bytes(c.S, c.n))
    return out, torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")


def drawn(c, seed):
    r = np.random.default_rng(seed)
    f = lambda n, std=1.0, mean=0.0: torch.from_numpy(r.normal(mean, std, n).astype(np.float32)).cuda()
    lp = f(c.n, 0.5, -1.5)
    return dict(rewards=f(c.n, 0.1), values=f(c.n), logp=lp, old=lp + f(c.n, 0.2), ref=lp + f(c.n, 0.2), verdict=f(c.S),
                mask=torch.from_numpy((r.random(c.n) < 0.8).astype(np.uint8)).cuda(), cu=c.cu.clone())


def bits(out):
    torch.cuda.synchronize()
    return {k: v.cpu().numpy().tobytes() for k, v in out.items()}


def test_the_same_bits_every_time_and_on_any_stream():
    c = Call("tile edges")
    x = drawn(c, 0)
    found = []
    for stream in (None, torch.cuda.Stream(), None, torch.cuda.Stream()):
        out, ws = buffers(c)
        torch.cuda.synchronize()
        everything(c, x, ws, out, stream)
        found.append(bits(out))
    assert all(f == found[0] for f in found)


def test_captured_calls_follow_their_inputs_and_share_a_workspace():
    """Two graphs with one workspace, replayed in turn over new data and new sequence lengths."""
    c = Call("tile edges")
    d = Call("across tiles")
    d.n, d.S = c.n, 5
    boundaries = [c.cu.clone(), torch.tensor(sorted({0, *np.random.default_rng(1).integers(0, c.n, 7).tolist(), c.n - 100}), dtype=torch.int32, device="cuda")]
    assert boundaries[1].numel() == 9 and c.S == 8
    states = []
    out_ws = buffers(c)[1]
    for call, seed in ((c, 1), (d, 2)):
        x, (out, _) = drawn(call, seed), buffers(call)
        if call is d:
            x["cu"] = torch.clamp(d.cu, max=c.n).contiguous()
        everything(call, x, out_ws, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            everything(call, x, out_ws, out)
        states.append((call, x, out, graph))
    for step in range(3):
        for call, x, out, graph in states:
            new = drawn(call, 10 + step)
            if call is c:
                new["cu"] = boundaries[step % 2]
            else:
                new["cu"] = x["cu"].clone()
            for k in x:
                x[k].copy_(new[k])
            for v in out.values():
                v.fill_(-7)
            graph.replay()
            want, ws = buffers(call)
            everything(call, x, ws, want)
            assert bits(out) == bits(want)


def test_boundaries_of_any_content_stay_inside():
    """Decreasing, negative and far boundaries: indices stay inside, guards hold (values are the caller's responsibility)."""
    for bad in ([0, 50, 10, 2 ** 31 - 1], [0, -5, -9, 60], [7, 3, 900, 2], [2 ** 31 - 1] * 4, [0, 0, 0, 2 ** 30]):
        c = Call("one token")
        c.bounds, c.S, c.n, c.live = np.array([0, 20, 40, 60]), 3, 60, 60
        c.mask = (c.rng.random(60) < 0.7).astype(np.uint8)
        c.cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        run_advantages(c, reward_inputs(c, trace=True), 0.9, 0.9)
        run_policy(c, policy_inputs(c, dict(TERMS, ratio=1, mean=1)), dict(TERMS, ratio=1, mean=1), 7)
        run_preference(c, preference_inputs(c), PREF, 3)
        for k in ("adv", "returns", "omega", "scores", "stats"):
            c.got(k)
        run_backward(c, dict(ga=c.normal(), gr=None, adv=c.normal(), trace=None), 0.9, 0.9)
        for k in ("rewards", "trace", "outcome"):
            c.got(k)


def test_boundaries_of_any_content_over_many_chunks_and_a_workspace_of_any_content():
    """Maps of chunks that the boundaries leave unmade are whatever the workspace held: numbers, but no places."""
    n = 60000
    trace, adv, ga = (torch.rand(n, device="cuda") for _ in range(3))
    for bad in ([0, 40000, 100, 59000], [0, 59999, 300, 60000], [9000, 3, 2 ** 31 - 1, 77], [0, -5, 50000, 600]):
        ws = torch.full((api.hilore_advantages_workspace_bytes(n),), 0x7F, dtype=torch.uint8, device="cuda")
        out = [G.Guarded(n * 4) for _ in range(3)]
        per = [G.Guarded(3 * 4) for _ in range(2)]
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        api.hilore_advantages_backward(ga, None, adv, trace, None, cu, 3, n, 0.9, 0.9, out[0].ptr(), per[0].ptr(), out[1].ptr(), per[1].ptr(), out[2].ptr(),
                                       ws, ws.numel())
        torch.cuda.synchronize()
        for g in out:
            g.numpy(np.float32, (n,))
        for g in per:
            g.numpy(np.float32, (3,))


def test_no_sequences_at_all():
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    stats, moments, pairs = torch.full((5,), 3.0, device="cuda"), torch.full((2,), 3.0, device="cuda"), torch.full((1,), 3, dtype=torch.int64, device="cuda")
    api.hilore_advantages(None, None, None, api.F32, None, None, None, None, 0, 0, 1.0, 1.0, None, None, moments, ws, ws.numel())
    api.hilore_policy_loss(None, None, None, None, None, None, None, None, 0, 0, api.make_policy_terms(), 1, None, None, stats, None, ws, ws.numel())
    assert not stats.any() and not moments.any()
    stats.fill_(3.0)
    api.hilore_preference_loss(None, None, None, None, 2, None, 0, 0, api.make_preference_terms(), 0, None, None, None, pairs, stats, None, ws, ws.numel())
    assert not stats[:4].any() and int(pairs) == 0
    api.hilore_advantages_backward(None, None, None, None, None, None, 0, 0, 1.0, 1.0, None, None, None, None, None, ws, ws.numel())


def test_a_run_from_logits_to_their_gradient():
    """token_logp -> advantages -> whitened policy loss -> token_logp_backward, against autograd in 64 bits."""
    rng = np.random.default_rng(0)
    bounds = np.array([0, 37, 37, 90, 160])
    n, S, V = 160, 4, 301
    x = torch.from_numpy(rng.normal(size=(n, V)).astype(np.float32)).cuda()
    f = lambda m, std=1.0: torch.from_numpy(rng.normal(0, std, m).astype(np.float32)).cuda()
    targets = torch.from_numpy(rng.integers(0, V, n).astype(np.int32)).cuda()
    mask = torch.from_numpy((rng.random(n) < 0.8).astype(np.uint8)).cuda()
    cu = G.dev(bounds.astype(np.int32))
    logp, lse, omega, adv, ret = (torch.empty(n, device="cuda") for _ in range(5))
    moments, stats, grad = torch.empty(2, device="cuda"), torch.empty(5, device="cuda"), torch.empty_like(x)
    values, outcome = f(n), f(S)
    ws = torch.empty(max(api.hilore_advantages_workspace_bytes(n), api.hilore_policy_loss_workspace_bytes(S, n)), dtype=torch.uint8, device="cuda")
    api.hilore_token_logp(x, api.F32, n, V, V, None, targets, logp, lse, None)
    old, ref = logp + f(n, 0.1), logp + f(n, 0.2)
    api.hilore_advantages(None, outcome, values, api.F32, None, None, mask, cu, S, n, 1.0, 0.9, adv, ret, moments, ws, ws.numel())
    terms = dict(TERMS, mean=1, adv_per_token=1, rollout_cap=math.inf)
    api.hilore_policy_loss(logp, old, ref, None, mask, adv, moments, cu, S, n, api.make_policy_terms(**terms), S, None, None, stats, omega, ws, ws.numel())
    api.hilore_token_logp_backward(x, api.F32, n, V, V, None, targets, lse, omega, grad, V)
    h = lambda t: t.cpu().double().numpy()
    a, _, (mean, std), _ = R.advantages(None, h(outcome), h(values), None, None, h(mask), bounds, n, 1.0, 0.9)
    xd = x.cpu().double().requires_grad_()
    s = torch.log_softmax(xd, 1).gather(1, targets.cpu().long()[:, None])[:, 0]
    want_stats, w, *_ = R.policy(s.detach().numpy(), h(old), h(ref), None, h(mask), a, (mean, std), bounds, terms, S)
    (s * torch.from_numpy(w)).sum().backward()
    # log-probabilities are some 20 roundings of numbers up to 8 off, and omega moves as much as they do
    tol = 400 * R.U * np.abs(w).max()
    close(h(omega), w, tol)
    close(h(grad), xd.grad.numpy(), 2 * tol)
    close(h(stats), want_stats, 400 * R.U * 10)
