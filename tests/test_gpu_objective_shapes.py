"""Advantages and losses where their work is dealt out at its limits: calls of one thread-block cluster and the next larger ones, sequences
of tens of millions of tokens, a long sequence behind many short ones."""
import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api
from tests import test_gpu_objective as T
from tests import test_gpu_objective_large as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("off", ["0", "1"])
@pytest.mark.parametrize("tokens", [1, 255, 256, 257, 2048, 2049, 8192, 8193, 16384, 16385])
def test_small_policy_losses_with_and_without_a_cluster(tokens, off, monkeypatch):
    """A warp has a block of 256 tokens, a CTA eight of them, a cluster up to eight CTAs: each side of every edge, in both forms, against
    the definition."""
    monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", off)
    cuts = np.unique(np.random.default_rng(tokens).integers(0, tokens + 1, 9))
    for beyond in (0, 700):
        t = dict(T.TERMS, ratio=0, mean=0, adv_per_token=1, dual_clip=1.5)
        c = T.Call("few", seed=tokens)
        c.bounds = np.unique(np.concatenate([[0], cuts, [tokens]])).astype(np.int64)
        c.S, c.live, c.n = len(c.bounds) - 1, tokens, tokens + beyond
        c.cu, c.mask = T.G.dev(c.bounds.astype(np.int32)), (c.rng.random(c.n) >= 0.2).astype(np.uint8)
        x = T.policy_inputs(c, t, rollout=True, white=True)
        T.run_policy(c, x, t, 321)
        T.check_policy(c, x, t, 321)


@pytest.mark.parametrize("trace", [False, True])
def test_sums_over_sequences_of_millions_of_tokens(trace):
    """With weights of 1 the recurrence adds up small whole numbers, in 64 bits without a rounding: exact sums, rounded once."""
    lengths = [30_000_001, 3, 0, 9_000_000, 70_000]
    bounds = np.concatenate([[0], np.cumsum(lengths)])
    n, S = int(bounds[-1]), len(lengths)
    g = torch.Generator(device="cuda").manual_seed(3)
    whole = lambda: torch.randint(-9, 10, (n,), generator=g, device="cuda").float()  # noqa: E731
    r, mask = whole(), (torch.rand(n, generator=g, device="cuda") < 0.9).to(torch.uint8)
    cu = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    outcome = torch.tensor([5.0, -3.0, 2.0, 1.0, 8.0], device="cuda")
    ones = torch.ones(n, device="cuda") if trace else None
    ws = torch.full((api.hilore_advantages_workspace_bytes(n),), 0x7F, dtype=torch.uint8, device="cuda")
    adv = torch.empty(n, device="cuda")
    api.hilore_advantages(r, outcome, None, api.F32, None, ones, mask, cu, S, n, 1.0, 1.0, adv, None, None, ws, ws.numel())
    back, d_r, d_o, d_c = whole(), torch.empty(n, device="cuda"), torch.empty(S, device="cuda"), torch.empty(n, device="cuda")
    api.hilore_advantages_backward(back, None, adv, ones, mask, cu, S, n, 1.0, 1.0, d_r, d_o, None, None, d_c, ws, ws.numel())
    m = mask.bool()
    for a, b, o, got_o in zip(bounds[:-1], bounds[1:], outcome.tolist(), d_o.tolist()):
        at, x = m[a:b], torch.where(m[a:b], r[a:b], 0.0).double()
        want = torch.flip(torch.cumsum(torch.flip(x, (0,)), 0), (0,)) + o
        assert torch.equal(adv[a:b], torch.where(at, want, 0.0).float())
        G = torch.cumsum(torch.where(at, back[a:b], 0.0).double(), 0)
        assert torch.equal(d_r[a:b], torch.where(at, G, 0.0).float())
        assert got_o == (float(G[-1].float()) if b > a else 0.0)
        where = torch.nonzero(at)[:, 0]
        follow = torch.cat([adv[a:b][where[1:]], adv.new_zeros(min(1, len(where)))])
        # an advantage in fp32 times a gradient in fp64, of whole numbers that fit: rounded once
        assert torch.equal(d_c[a:b][where], (follow.double() * G[where]).float()) and not bool(d_c[a:b][~at].any())


@pytest.mark.parametrize("ratio,mean,kl,per_token", [(0, 1, 3, True), (0, 1, 1, False), (1, 1, 2, False), (1, 0, 3, False)])
def test_policy_of_a_long_sequence_behind_many_short_ones(ratio, mean, kl, per_token, monkeypatch):
    """A block's last sequence, behind some twenty that end in it, lies over thousands of shares."""
    monkeypatch.setattr(L, "lengths_of", lambda kind: np.array([3] * 20 + [2_000_000] + [1, 2] * 30 + [0, 700_000] + [2] * 100 + [300_000]))
    L.test_policy("long behind short", ratio, mean, kl, per_token)


@pytest.mark.parametrize("length_mean", [0, 1])
def test_preference_of_long_responses_among_short_ones(length_mean, monkeypatch):
    lengths = np.tile(np.array([3] * 22 + [2_000_000, 5, 0, 90_000] + [2] * 11), 92)  # 92 * 37 = 851 * 4
    lengths[lengths > 100] //= 60
    lengths[22] = 5_000_000
    monkeypatch.setattr(L, "lengths_of", lambda kind: lengths)
    L.test_preference("long among short", 0, length_mean, 4)
