"""Advantages, policy loss and preference loss at sizes where warps have shares of many blocks, sequences go over several of them and the
work is dealt out in other ways, against 64-bit tensor operations on the same device; and the forms that small calls can take."""
import numpy as np
import pytest
import torch

from paper_2609_33570_b200 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def ragged(seed, lengths, masked=0.2):
    """Boundaries, the sequence of every token, a mask, and a maker of normal numbers."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    length = torch.as_tensor(lengths, device="cuda")
    cu = torch.cat([length.new_zeros(1), torch.cumsum(length, 0)])
    n = int(cu[-1])
    seq = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), length, output_size=n)
    mask = (torch.rand(n, generator=g, device="cuda") >= masked).to(torch.uint8)
    # stretches with no valid token and with nothing masked
    part = torch.arange(n, device="cuda") // 700 % 5
    mask = torch.where(part == 1, 0, torch.where(part >= 3, 1, mask)).to(torch.uint8)
    normal = lambda k=n, std=1.0, mean=0.0: torch.empty(k, device="cuda").normal_(mean, std, generator=g)  # noqa: E731
    return cu.int(), seq, mask, n, normal


def lengths_of(kind):
    r = np.random.default_rng(3)
    if kind == "pieces":      # more tokens than warps that run at once take in even chunks, some sequences longer than a piece
        return np.concatenate([r.integers(0, 6000, 2600), [20001, 16384, 16385, 70000, 0, 1], r.integers(1, 40, 2000)])
    if kind == "short":       # blocks with many ends, sequences without a token among them
        return np.concatenate([r.integers(0, 40, 20000), [700, 0, 0, 3000], np.zeros(3000, int), r.integers(1, 3, 9000), [1]])
    if kind == "waves":       # pieces in more chunks than warps run at once
        return np.concatenate([r.integers(0, 9000, 7600), [31000]])
    if kind == "long":        # even chunks, more than warps run at once
        return np.concatenate([r.integers(0, 900000, 50), r.integers(0, 9, 500)])
    return np.concatenate([r.integers(0, 3000, 400), [150000, 1, 0, 5000], r.integers(0, 9, 3000)])  # even chunks


def recurrence(gate, add, longest):
    """x_k = add_k + gate_k x_{k+1}, in rounds that double what an element has taken in."""
    step = 1
    while step < longest:
        head = add[:-step] + gate[:-step] * add[step:]
        add = torch.cat([head, add[-step:]])
        gate = torch.cat([gate[:-step] * gate[step:], torch.zeros_like(gate[-step:])])
        step *= 2
    return add


def close(got, want, scale):
    """A rounding to fp32 of sums whose terms are `scale` large, in 64 bits: 2^-24 of the result, and 2^-36 of the terms, which is more
    than the longest sequence's roundings of 2^-53 each."""
    off = (got.double() - want).abs()
    assert bool((off <= U * 1.0001 * want.abs() + 2.0 ** -36 * scale).all()), float(off.max())


@pytest.mark.parametrize("kind", ["even", "pieces", "waves", "long", "short"])
@pytest.mark.parametrize("trace", [False, True])
def test_advantages_and_their_gradient(kind, trace):
    lengths = lengths_of(kind)
    cu, seq, mask, n, normal = ragged(1, lengths)
    S, gamma, lam = len(lengths), 0.999, 0.97
    rewards, values, outcome, bootstrap = normal(std=0.1), normal(), normal(S), normal(S)
    c = normal(std=0.3).exp_().clamp_(max=1.0) if trace else None
    ws = torch.full((api.hilore_advantages_workspace_bytes(n),), 0xFF, dtype=torch.uint8, device="cuda")
    adv, ret, moments = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(2, device="cuda")
    api.hilore_advantages(rewards, outcome, values, api.F32, bootstrap, c, mask, cu, S, n, gamma, lam, adv, ret, moments, ws, ws.numel())
    at = torch.nonzero(mask)[:, 0]
    s = seq[at]
    last = torch.ones_like(s, dtype=torch.bool)
    last[:-1] = s[1:] != s[:-1]
    v = values[at].double()
    after = torch.where(last, outcome[s].double() + gamma * bootstrap[s].double(), gamma * torch.roll(v, -1))
    gate = gamma * lam * (torch.ones_like(v) if c is None else c[at].double())
    A = recurrence(torch.where(last, 0.0, gate), rewards[at].double() + after - v, int(lengths.max()))
    full = lambda x: torch.zeros(n, dtype=torch.float64, device="cuda").index_copy_(0, at, x)  # noqa: E731
    close(adv, full(A), 1e2)
    close(ret, full(A + v), 1e2)
    close(moments, torch.stack([A.mean(), A.std(correction=0)]), 1e2)
    # backwards: from the first token of a sequence on
    ga, gr = normal(), normal()
    out = {k: torch.empty(n, device="cuda") for k in ("rewards", "values", "trace")}
    out.update(outcome=torch.empty(S, device="cuda"), bootstrap=torch.empty(S, device="cuda"))
    api.hilore_advantages_backward(ga, gr, adv, c, mask, cu, S, n, gamma, lam, out["rewards"], out["outcome"], out["values"], out["bootstrap"], out["trace"],
                                   ws, ws.numel())
    first = torch.cat([torch.ones_like(last[:1]), last[:-1]])
    g2 = gr[at].double()
    back = lambda x: torch.flip(x, (0,))  # noqa: E731
    G = back(recurrence(back(torch.where(first, 0.0, torch.roll(gate, 1))), back(ga[at].double() + g2), int(lengths.max())))
    close(out["rewards"], full(G), 1e2)
    close(out["values"], full(g2 - G + gamma * torch.where(first, 0.0, torch.roll(G, 1))), 1e2)
    close(out["trace"], full(torch.where(last, 0.0, gamma * lam * torch.roll(adv[at].double(), -1) * G)), 1e3)
    final = torch.zeros(S, dtype=torch.float64, device="cuda").index_copy_(0, s[last], G[last])
    close(out["outcome"], final, 1e2)
    close(out["bootstrap"], gamma * final, 1e2)


TERMS = dict(clip_low=0.2, clip_high=0.28, dual_clip=1.5, beta=0.02, rollout_cap=1.05, adv_eps=1e-6)


def policy_call(cu, mask, n, S, x, t, per_token, N):
    ws = torch.full((api.hilore_policy_loss_workspace_bytes(S, n),), 0xFF, dtype=torch.uint8, device="cuda")
    stats, omega = torch.empty(5, device="cuda"), torch.empty(n, device="cuda")
    api.hilore_policy_loss(x["logp"], x["old"], x["ref"], x["rollout"], mask, x["adv"], x["white"], cu, S, n,
                           api.make_policy_terms(**TERMS, **t, adv_per_token=per_token), N, None, None, stats, omega, ws, ws.numel())
    return stats, omega


def policy_inputs(seq, n, S, normal, ratio, per_token):
    lp = normal(std=0.7, mean=-1.5)
    old = lp + (normal(std=0.2) if ratio == 0 else normal(S, 0.3)[seq])
    return dict(logp=lp, old=old, ref=lp + normal(std=0.4), rollout=old + normal(std=0.03), adv=normal(n if per_token else S),
                white=torch.tensor([0.1, 0.9], device="cuda") if per_token else None)


@pytest.mark.parametrize("kind", ["even", "short"])
@pytest.mark.parametrize("ratio,mean,kl,per_token", [(0, 0, 3, True), (0, 1, 3, True), (0, 1, 1, False), (1, 1, 2, False), (1, 0, 3, False)])
def test_policy(kind, ratio, mean, kl, per_token):
    lengths = lengths_of(kind)
    cu, seq, mask, n, normal = ragged(2, lengths)
    S, N = len(lengths), 12345
    x = policy_inputs(seq, n, S, normal, ratio, per_token)
    stats, omega = policy_call(cu, mask, n, S, x, dict(ratio=ratio, mean=mean, kl=kl), per_token, N)
    at = torch.nonzero(mask)[:, 0]
    s = seq[at]
    lp, old, ref, roll = (x[k][at].double() for k in ("logp", "old", "ref", "rollout"))
    by = lambda v: torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, s, v)  # noqa: E731
    size = by(torch.ones_like(lp))
    d, gap = lp - old, old - roll
    if ratio:
        d, gap = (by(d) / size)[s], (by(gap) / size)[s]
    A = x["adv"][at if per_token else s].double()
    if x["white"] is not None:
        A = (A - x["white"][0].double()) / (x["white"][1].double() + TERMS["adv_eps"])
    w = torch.full_like(lp, 1 / N) if mean == 0 else 1 / (N * size[s])
    rho, i = d.exp(), gap.exp().clamp(max=TERMS["rollout_cap"])
    flat = torch.where(A >= 0, rho > 1.28, (rho < 0.8) | (rho > 1.5))
    held = torch.where(A >= 0, rho.clamp(max=1.28), rho.clamp(0.8, 1.5))
    term, grad = -w * i * A * held, torch.where(flat, 0.0, -w * i * A * rho)
    e = ref - lp
    k, slope = {1: (-e, torch.ones_like(e)), 2: (e * e / 2, -e), 3: (torch.expm1(e) - e, -torch.expm1(e))}[kl]
    beta = TERMS["beta"]
    want = torch.zeros(n, dtype=torch.float64, device="cuda").index_copy_(0, at, grad + beta * w * slope)
    size_of = torch.zeros(n, dtype=torch.float64, device="cuda").index_copy_(0, at, w * ((1 + d.abs() + gap.abs()) * A.abs() * rho + beta * (1 + e.abs()) * (1 + e.exp())))
    assert bool(((omega.double() - want).abs() <= 24 * U * size_of).all())  # some twenty roundings, those of exponents by their size
    sums = torch.stack([term.sum() + beta * (w * k).sum(), term.sum(), (w * k).sum(), (w * (flat & (A != 0))).sum(),
                        (w * (x["old"][at].double() - lp)).sum()])
    big = torch.stack([term.abs().sum() + (w * k.abs()).sum(), term.abs().sum(), (w * (k.abs() + e * e)).sum(), w.sum(), (w * (x["old"][at].double() - lp).abs()).sum()])
    assert bool(((stats.double() - sums).abs() <= 32 * U * big).all())


@pytest.mark.parametrize("kind", ["even", "short"])
@pytest.mark.parametrize("loss,length_mean,group", [(0, 1, 4), (1, 0, 2), (2, 1, 851)])
def test_preference(kind, loss, length_mean, group):
    lengths = lengths_of(kind)
    lengths = lengths[:len(lengths) // 851 // 4 * 851 * 4]
    cu, seq, mask, n, normal = ragged(4, lengths)
    S = len(lengths)
    assert S % group == 0
    lp = normal(std=0.7, mean=-1.5)
    ref, R = lp + normal(std=0.1), torch.round(normal(S))
    t = dict(beta=2.0 if length_mean else 0.05, margin=0.1, margin_reward=0.05, nll=0.1, loss=loss, length_mean=bool(length_mean),
             smoothing=0.1 if loss == 0 else 0.0)
    ws = torch.full((api.hilore_preference_loss_workspace_bytes(S, n),), 0xFF, dtype=torch.uint8, device="cuda")
    scores, stats, omega = torch.empty(S, device="cuda"), torch.empty(4, device="cuda"), torch.empty(n, device="cuda")
    pairs = torch.empty(1, dtype=torch.int64, device="cuda")
    api.hilore_preference_loss(lp, ref, mask, R, group, cu, S, n, api.make_preference_terms(**t), 0, None, None, scores, pairs, stats, omega, ws, ws.numel())
    at = torch.nonzero(mask)[:, 0]
    s = seq[at]
    by = lambda v: torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, s, v)  # noqa: E731
    size = by(torch.ones(at.numel(), dtype=torch.float64, device="cuda"))
    per = torch.where(size > 0, 1 / size.clamp(min=1), 0.0)
    like = (by(lp[at].double()) * per).requires_grad_()
    h = (t["beta"] * by(lp[at].double() - ref[at].double()) * (per if length_mean else 1.0)).requires_grad_()
    B, r, real = h.view(-1, group), R.double().view(-1, group), (size > 0).view(-1, group)
    better = (r[:, :, None] > r[:, None, :]) & real[:, :, None] & real[:, None, :]
    gap = (B[:, :, None] - B[:, None, :])[better]
    z = gap - t["margin"] - t["margin_reward"] * (r[:, :, None] - r[:, None, :])[better]
    f = torch.nn.functional.logsigmoid
    each = {0: -0.9 * f(z) - 0.1 * f(-z), 1: torch.relu(1 - z), 2: ((z - 0.5) / t["beta"]) ** 2}[loss]
    N = each.numel()
    nll = -(like.view(-1, group)[:, :, None] * better).sum() / N
    total = each.sum() / N + t["nll"] * nll
    gh, gl = torch.autograd.grad(total, (h, like))
    c = gh * t["beta"] * (per if length_mean else 1.0) + gl * per
    want = torch.zeros(n, dtype=torch.float64, device="cuda").index_copy_(0, at, c[s])
    assert int(pairs) == N
    close(scores, h.detach(), 1e2)
    assert bool(((omega.double() - want).abs() <= U * 1.001 * want.abs() + 2.0 ** -36 * c.abs().max()).all())
    close(stats, torch.stack([total, (gap > 0).double().mean(), gap.mean(), nll]).detach(), 1e2)


@pytest.mark.parametrize("off", ["1", "0"])
def test_small_calls_as_one_cluster_or_as_several_launches(off, monkeypatch):
    """Small policy losses are one cluster of CTAs: the same results, to the roundings of sums in another order, without it."""
    monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", off)
    for lengths in ([5], [300, 0, 17, 4000], [128] * 200, [32768], [32769]):
        cu, seq, mask, n, normal = ragged(5, lengths)
        S = len(lengths)
        for ratio, mean, per_token in ((0, 0, True), (0, 1, False), (1, 1, False)):
            x = policy_inputs(seq, n, S, normal, ratio, per_token)
            found = []
            for again in ("0", off):
                monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", again)
                found.append(policy_call(cu, mask, n, S, x, dict(ratio=ratio, mean=mean, kl=3), per_token, 99))
            (s0, o0), (s1, o1) = found
            assert bool(((o0 - o1).abs() <= 4 * U * o0.abs()).all()) and bool(((s0 - s1).abs() <= 8 * U * s0.abs().max()).all())
        R = normal(S)
        ws = torch.full((api.hilore_preference_loss_workspace_bytes(S, n),), 0xFF, dtype=torch.uint8, device="cuda")
        found = []
        for again in ("0", off):
            monkeypatch.setenv("HILORE_DISABLE_CLUSTER_LAUNCH", again)
            omega, stats, scores = torch.empty(n, device="cuda"), torch.empty(4, device="cuda"), torch.empty(S, device="cuda")
            api.hilore_preference_loss(x["logp"], x["ref"], mask, R, S, cu, S, n, api.make_preference_terms(length_mean=True), 0, None, None, scores, None,
                                       stats, omega, ws, ws.numel())
            found.append((omega, stats, scores))
        for a, b in zip(*found):
            assert bool(((a - b).abs() <= 4 * U * a.abs().max()).all())


@pytest.mark.parametrize("n,S", [(1, 1), (1024, 700), (1025, 3), (65537, 9), (910000, 900), (1300001, 2), (7400001, 4000), (23000001, 6)])
def test_nothing_is_written_behind_a_workspace(n, S):
    """Workspaces of just the size that is asked for, with bytes behind them that have to stay, and with any content."""
    cu = torch.linspace(0, n, S + 1, device="cuda", dtype=torch.float64).round().int()
    seq_input, x = torch.ones(S, device="cuda"), torch.zeros(n, device="cuda")
    R = torch.arange(S, device="cuda", dtype=torch.float32)
    out, more, few, per = (torch.zeros(m, device="cuda") for m in (n, n, 5, S))  # moments are two numbers, statistics four or five
    group = next(g for g in (7, 3, 2, 1) if S % g == 0)
    calls = {
        api.hilore_advantages_workspace_bytes(n): [
            lambda w, b: api.hilore_advantages(x, seq_input, x, api.F32, None, None, None, cu, S, n, 1.0, 0.9, out, more, few, w, b),
            lambda w, b: api.hilore_advantages_backward(x, x, x, x, None, cu, S, n, 1.0, 0.9, out, per, more, None, None, w, b)],
        api.hilore_policy_loss_workspace_bytes(S, n): [
            lambda w, b, r=r, m=m: api.hilore_policy_loss(x, x, x, x, None, seq_input, None, cu, S, n, api.make_policy_terms(ratio=r, mean=m), n, None, None, few,
                                                          out, w, b) for r in (0, 1) for m in (0, 1)],
        api.hilore_preference_loss_workspace_bytes(S, n) + 16: [  # a key of its own
            lambda w, b: api.hilore_preference_loss(x, x, None, R, group, cu, S, n, api.make_preference_terms(), 0, None, None, None, None, few, out, w, b - 16)]}
    for size, some in calls.items():
        buf = torch.full((size + 4096,), 0x7F, dtype=torch.uint8, device="cuda")
        for call in some:
            call(buf, size)
        torch.cuda.synchronize()
        assert bool((buf[size:] == 0x7F).all()) and bool(torch.isfinite(few[:4]).all())
    assert bool((buf[size - 16:] == 0x7F).all())


@pytest.mark.parametrize("T", [2000, 140000])
def test_tensors_of_more_than_two_to_the_31_bytes(T):
    """Rows at the end of a call whose tensors pass 2^31 bytes are what a call over these rows alone gives."""
    S = 560_000_000 // T
    n, few = S * T, 4
    tail = few * T
    g = torch.Generator(device="cuda").manual_seed(6)
    lp = torch.empty(n, device="cuda").normal_(-1.5, 0.7, generator=g)
    old = torch.empty(n, device="cuda").normal_(-1.5, 0.7, generator=g)
    mask = torch.empty(n, dtype=torch.uint8, device="cuda").random_(0, 4, generator=g)
    R = torch.empty(S, device="cuda").normal_(generator=g)

    def run(lp, old, mask, R, S, n):
        ws = torch.empty(max(api.hilore_advantages_workspace_bytes(n), api.hilore_policy_loss_workspace_bytes(S, n),
                             api.hilore_preference_loss_workspace_bytes(S, n)), dtype=torch.uint8, device="cuda")
        out, stats, found = torch.empty(n, device="cuda"), torch.empty(5, device="cuda"), []
        keep = lambda: found.append(out[-tail:].clone())  # noqa: E731
        api.hilore_advantages(lp, R, old, api.F32, None, None, mask, None, S, n, 1.0, 0.99, out, None, None, ws, ws.numel())
        keep()
        api.hilore_advantages_backward(lp, old, None, None, mask, None, S, n, 1.0, 0.99, None, None, out, None, None, ws, ws.numel())
        keep()
        for ratio, mean in ((0, 0), (0, 1), (1, 1)):
            api.hilore_policy_loss(lp, old, None, None, mask, R, None, None, S, n, api.make_policy_terms(ratio=ratio, mean=mean), 1000, None, None, stats, out,
                                   ws, ws.numel())
            keep()
        api.hilore_preference_loss(lp, old, mask, R, 2, None, S, n, api.make_preference_terms(length_mean=True), 1000, None, None, None, None, stats, out,
                                   ws, ws.numel())
        keep()
        return found

    for whole, part in zip(run(lp, old, mask, R, S, n), run(lp[-tail:].clone(), old[-tail:].clone(), mask[-tail:].clone(), R[-few:].clone(), few, tail)):
        assert bool((whole.double() - part.double()).abs().max() <= 4 * U * part.abs().max())
