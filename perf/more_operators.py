"""Cases of the objectives between rewards and the gradient of the log-probabilities: advantages and returns by a gated
recurrence over the tokens of a sequence with their backward pass, the clipped policy loss with a KL term, and the
preference loss on pairs of responses, both with their gradients.

`run` computes a case in its plain form (elementary torch operations) or, where `own` is true, through the library's entry
points.  `exact` is the definition in 64 bits, written apart from both.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    packed = dict(layout="packed")
    return [
        # one response of a streaming trainer: the latency of the call
        dict(name="advantages one response", kind="adv", seqs=1, tokens=700, prompt=0.2, holes=0.0, values="f32", trace=False, gamma=1.0, lam=0.95,
             moments=False, **packed),
        # a rollout batch, 2048 responses of up to some 4096 tokens, critic in bf16, tool outputs masked, whitening afterwards
        dict(name="advantages rollout batch", kind="adv", seqs=2048, tokens=4_325_377, prompt=0.15, holes=0.1, values="bf16", trace=False, gamma=1.0,
             lam=0.95, moments=True, **packed),
        # few long agent runs: the recurrence crosses a hundred thousand tokens, with a weight per token
        dict(name="advantages long runs", kind="adv", seqs=24, tokens=2_000_003, prompt=0.05, holes=0.3, values="f32", trace=True, gamma=0.9995, lam=1.0,
             moments=False, **packed),
        # the whole rollout of a large update, padded rows of 2048 slots
        dict(name="advantages padded update", kind="adv", seqs=32768, tokens=32768 * 2048, prompt=0.1, holes=0.0, values="f32", trace=False, gamma=1.0,
             lam=0.97, moments=True, layout="padded"),
        # gradients through the estimator for a microbatch, weights learned
        dict(name="advantages gradient microbatch", kind="adv_grad", seqs=12, tokens=24_001, prompt=0.2, holes=0.1, trace=True, gamma=0.99, lam=0.95,
             **packed),
        # the same for a whole rollout, weights fixed
        dict(name="advantages gradient rollout", kind="adv_grad", seqs=8000, tokens=16_000_001, prompt=0.2, holes=0.0, trace=False, gamma=1.0, lam=0.95,
             **packed),
        # a tiny step: 4 prompts x 8 responses x 256 slots
        dict(name="policy tiny step", kind="policy", seqs=32, tokens=8192, prompt=0.0, holes=0.0, ratio="token", mean="tokens", kl=0, dual=0.0,
             rollout=False, adv="sequence", white=False, layout="padded"),
        # a microbatch of 64 responses, KL to the reference, dual clip, corrected for the sampling engine, whitened advantages
        dict(name="policy microbatch", kind="policy", seqs=64, tokens=131_071, prompt=0.15, holes=0.1, ratio="token", mean="sequences", kl=3, dual=3.0,
             rollout=True, adv="token", white=True, **packed),
        # ratios of whole sequences over an update of 512 responses
        dict(name="policy sequence ratios", kind="policy", seqs=512, tokens=1_048_577, prompt=0.15, holes=0.0, ratio="sequence", mean="sequences", kl=2,
             dual=0.0, rollout=False, adv="sequence", white=False, **packed),
        # all tokens of a large update in one call
        dict(name="policy whole update", kind="policy", seqs=32768, tokens=60_000_001, prompt=0.1, holes=0.0, ratio="token", mean="tokens", kl=3, dual=0.0,
             rollout=False, adv="token", white=False, **packed),
        # pairs of a preference microbatch, chosen and rejected, half of each a prompt
        dict(name="preference microbatch", kind="pref", seqs=16, group=2, tokens=9_001, prompt=0.5, holes=0.0, loss="sigmoid", length=False, ref=True,
             nll=0.0, smoothing=0.0, **packed),
        # all pairs among 16 responses of each of 2048 prompts, likelihood term, label smoothing
        dict(name="preference groups", kind="pref", seqs=32768, group=16, tokens=50_000_001, prompt=0.15, holes=0.0, loss="sigmoid", length=True, ref=True,
             nll=0.1, smoothing=0.05, **packed),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adv", "adv", "adv_grad", "policy", "policy", "policy", "pref", "pref"])
    tokens = _log(rng, 100, {"adv": 60_000_000, "adv_grad": 16_000_000, "policy": 60_000_000, "pref": 50_000_000}[kind])
    # mean lengths from a few tokens to a hundred thousand, up to 40000 sequences
    seqs = max(1, min(40_000, tokens // _log(rng, 6, 100_000)))
    case = dict(kind=kind, seqs=seqs, tokens=tokens, prompt=rng.choice([0.0, 0.1, 0.5]), holes=rng.choice([0.0, 0.0, 0.2]),
                layout=rng.choice(["packed", "packed", "padded"]))
    if kind == "pref":
        group = rng.choice([2, 2, 4, 7, 16, 32])
        case["group"] = group = min(group, seqs)
        case["seqs"] = seqs = seqs // group * group
        case.update(loss=rng.choice(["sigmoid", "hinge", "square"]), length=rng.random() < 0.5, ref=rng.random() < 0.7, nll=rng.choice([0.0, 0.2]),
                    smoothing=rng.choice([0.0, 0.1]))
    elif kind == "policy":
        ratio = rng.choice(["token", "token", "sequence"])
        case.update(ratio=ratio, mean=rng.choice(["tokens", "sequences"]), kl=rng.choice([0, 1, 2, 3, 3]), dual=rng.choice([0.0, 2.0]),
                    rollout=rng.random() < 0.3, adv="sequence" if ratio == "sequence" else rng.choice(["token", "sequence"]), white=rng.random() < 0.3)
    else:
        case.update(trace=rng.random() < 0.4, gamma=rng.choice([1.0, 1.0, 0.99, 0.9999]), lam=rng.choice([1.0, 0.95, 0.9]))
        if kind == "adv":
            case.update(values=rng.choice(["f32", "f32", "bf16"]), moments=rng.random() < 0.5)
    if case["layout"] == "padded":
        case["tokens"] = max(1, tokens // seqs) * seqs
    return case


def work(case):
    """Each input read once, each output written once."""
    n, kind = case["tokens"], case["kind"]
    per_seq = 4 * case["seqs"] * (case["layout"] == "packed")
    if kind == "adv":
        per = 4 + (2 if case["values"] == "bf16" else 4) + 4 * case["trace"] + 1 + 8
        return {"bytes": n * per + per_seq + 8 * case["seqs"], "flops": n * (8 + 4 * case["moments"])}
    if kind == "adv_grad":
        return {"bytes": n * (8 + 1 + 8 + 12 * case["trace"]) + per_seq + 8 * case["seqs"], "flops": n * 8}
    if kind == "policy":
        per = 8 + 4 * (case["kl"] > 0) + 4 * case["rollout"] + 4 * (case["adv"] == "token") + 1 + 4
        return {"bytes": n * per + per_seq + 4 * case["seqs"], "flops": n * 20}
    return {"bytes": n * (4 + 4 * case["ref"] + 1 + 4) + per_seq + 8 * case["seqs"], "flops": n * 4 + case["seqs"] * case["group"] * 20}


# --------------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _sequences(case, g):
    """Lengths that add up to the case's tokens, the sequence of every token, and the mask of the generated tokens: a prompt, a
    response, tool outputs in it; padded rows end in slots without a token."""
    n, S = case["tokens"], case["seqs"]
    if case["layout"] == "padded":
        length = torch.full((S,), n // S, device="cuda", dtype=torch.int64)
    else:
        share = torch.rand(S, generator=g, device="cuda", dtype=torch.float64) + 0.05
        edge = torch.round(torch.cumsum(share, 0) / share.sum() * n).long()
        edge[-1] = n
        length = torch.diff(edge, prepend=edge.new_zeros(1))
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), length, output_size=n)
    begin = torch.cumsum(length, 0) - length
    place = torch.arange(n, device="cuda") - begin[seq]
    prompt = (length.double() * case["prompt"] * 2 * torch.rand(S, generator=g, device="cuda", dtype=torch.float64)).long()
    mask = place >= prompt[seq]
    if case["layout"] == "padded":
        end = (length.double() * (0.2 + 0.8 * torch.rand(S, generator=g, device="cuda", dtype=torch.float64))).long() + 1
        mask &= place < end[seq]
    if case["holes"]:
        mask &= (torch.rand(n // 150 + 1, generator=g, device="cuda") >= case["holes"])[torch.arange(n, device="cuda") // 150]
    cu = torch.cat([begin, begin.new_full((1,), n)]).int() if case["layout"] == "packed" else None
    return length, seq, mask.to(torch.uint8), cu


def prepare(case, seed):
    g = _generator(seed)
    n, S, kind = case["tokens"], case["seqs"], case["kind"]
    length, seq, mask, cu = _sequences(case, g)
    normal = lambda std=1.0, k=n: torch.empty(k, device="cuda").normal_(0.0, std, generator=g)  # noqa: E731
    s = {"case": dict(case), "mask": mask, "cu": cu, "length": length, "seq": seq}
    room = lambda *names: s.update({k: torch.zeros(n, device="cuda") for k in names})  # noqa: E731
    correct = (torch.rand(S, generator=g, device="cuda") < 0.5).float()
    if kind in ("adv", "adv_grad"):
        s["trace"] = torch.exp(normal(0.2)).clamp_(max=1.0) if case["trace"] else None
        if kind == "adv":
            s["rewards"] = normal(0.02)  # a penalty per token, and the verdict on the whole response
            s["outcome"] = correct
            s["values"] = normal(0.2).add_(0.5).to(torch.bfloat16 if case["values"] == "bf16" else torch.float32)
            s["bootstrap"] = torch.where(torch.rand(S, generator=g, device="cuda") < 0.1, 0.5, 0.0)  # responses cut short
            room("adv", "returns")
            s["moments"] = torch.zeros(2, device="cuda")
        else:
            s["grad_adv"], s["grad_returns"] = normal(), normal()
            s["adv"] = normal() * mask
            room("grad_rewards", "grad_values", "grad_trace")
            s["grad_outcome"], s["grad_bootstrap"] = torch.zeros(S, device="cuda"), torch.zeros(S, device="cuda")
    else:
        s["logp"] = -normal(1.2).abs_()
        s["omega"] = torch.zeros(n, device="cuda")
        if kind == "policy":
            s["old"] = s["logp"] + normal(0.08)
            s["ref"] = s["logp"] + normal(0.15) if case["kl"] else None
            s["rollout"] = s["old"] + normal(0.02) if case["rollout"] else None
            s["adv"] = normal(1.0, n if case["adv"] == "token" else S)
            s["white"] = torch.tensor([0.1, 0.8], device="cuda") if case["white"] else None
            s["stats"] = torch.zeros(5, device="cuda")
            s["norm"] = int(mask.sum(dtype=torch.int64)) if case["mean"] == "tokens" else S
            s["terms"] = dict(clip_low=0.2, clip_high=0.28, dual_clip=case["dual"], beta=1e-2 if case["kl"] else 0.0, rollout_cap=1.05, adv_eps=1e-6)
            s["norm"] = max(1, s["norm"])
            if case["ratio"] == "sequence":  # a sequence's mean moves less than its tokens
                s["terms"].update(clip_low=4e-3, clip_high=6e-3)
        else:
            s["ref"] = s["logp"] + normal(0.3) if case["ref"] else None
            s["rewards"] = torch.round(4 * torch.rand(S, generator=g, device="cuda")) / 4 if case["group"] > 2 else \
                torch.stack([correct, 1 - correct], 1).view(-1)[:S].contiguous()
            s["scores"], s["stats"] = torch.zeros(S, device="cuda"), torch.zeros(4, device="cuda")
            s["pairs"] = torch.zeros(1, dtype=torch.int64, device="cuda")
            s["terms"] = dict(beta=2.0 if case["length"] else 0.1, margin=0.2 if not case["ref"] else 0.0, margin_reward=0.1, nll=case["nll"],
                              smoothing=case["smoothing"] if case["loss"] == "sigmoid" else 0.0)
    if own:
        from paper_2609_33570_b200 import api
        s["api"] = api
        if kind == "policy":
            s["handle"] = api.make_policy_terms(**s["terms"], ratio=api.RATIO_SEQUENCE if case["ratio"] == "sequence" else api.RATIO_TOKEN,
                                                mean=api.MEAN_SEQUENCES if case["mean"] == "sequences" else api.MEAN_TOKENS, kl=case["kl"] or api.KL_K3,
                                                adv_per_token=case["adv"] == "token")
            size = api.hilore_policy_loss_workspace_bytes(S, n)
        elif kind == "pref":
            s["handle"] = api.make_preference_terms(**s["terms"], length_mean=case["length"],
                                                    loss={"sigmoid": api.PREF_SIGMOID, "hinge": api.PREF_HINGE, "square": api.PREF_SQUARE}[case["loss"]])
            size = api.hilore_preference_loss_workspace_bytes(S, n)
        else:
            size = api.hilore_advantages_workspace_bytes(n)
        s["workspace"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms
def _recurrence(gate, add, longest):
    """x_k = add_k + gate_k x_{k+1} from the last element on (64 bits: long sums), every element at once: after a round each
    element has taken in twice as many of its followers, so the rounds are the logarithm of the longest sequence."""
    step = 1
    while step < min(longest, add.numel()):
        head = add[:-step] + gate[:-step] * add[step:]
        add = torch.cat([head, add[-step:]])
        gate = torch.cat([gate[:-step] * gate[step:], torch.zeros_like(gate[-step:])])
        step *= 2
    return add


def _valid(s):
    """Places of the valid tokens, their sequences, and whether each is the last one of its sequence."""
    at = torch.nonzero(s["mask"])[:, 0]
    seq = s["seq"][at]
    last = torch.ones_like(seq, dtype=torch.bool)
    last[:-1] = seq[1:] != seq[:-1]
    return at, seq, last


def _next(x, last, end):
    """The following valid token's entry; `end` where there is none in the sequence."""
    y = torch.cat([x[1:], x[:1]])
    return torch.where(last, end, y)


def _spread(at, x, n, dtype=torch.float32):
    return torch.zeros(n, dtype=dtype, device=x.device).index_copy_(0, at, x.to(dtype))


def _plain_adv(s):
    case, n = s["case"], s["case"]["tokens"]
    at, seq, last = _valid(s)
    v = s["values"][at].double()
    r = s["rewards"][at].double() + torch.where(last, s["outcome"][seq].double(), 0.0)
    delta = r + case["gamma"] * _next(v, last, s["bootstrap"][seq].double()) - v
    gate = torch.full_like(v, case["gamma"] * case["lam"])
    if s["trace"] is not None:
        gate = gate * s["trace"][at].double()
    a = _recurrence(torch.where(last, 0.0, gate), delta, int(s["length"].max()))
    out = {"adv": _spread(at, a, n), "returns": _spread(at, a + v, n)}
    if case["moments"]:
        count = max(1, a.numel())
        mean = a.sum() / count
        out["moments"] = torch.stack([mean, ((a - mean).square().sum() / count).sqrt()]).float()
    return out


def _plain_adv_grad(s):
    case, n = s["case"], s["case"]["tokens"]
    at, seq, last = _valid(s)
    first = torch.cat([torch.ones_like(last[:1]), last[:-1]])
    weight = case["gamma"] * case["lam"]
    gate = torch.full_like(at, weight, dtype=torch.float64)
    if s["trace"] is not None:
        gate = gate * s["trace"][at].double()
    before = torch.where(first, 0.0, torch.cat([gate[:1], gate[:-1]]))
    g_ret = s["grad_returns"][at].double()
    back = lambda x: torch.flip(x, (0,))  # noqa: E731
    G = back(_recurrence(back(before), back(s["grad_adv"][at].double() + g_ret), int(s["length"].max())))
    G_before = torch.where(first, 0.0, torch.cat([G[:1], G[:-1]]))
    S = case["seqs"]
    final = _spread(seq[last], G[last], S, torch.float64)
    out = {"grad_rewards": _spread(at, G, n), "grad_values": _spread(at, g_ret - G + case["gamma"] * G_before, n), "grad_outcome": final.float(),
           "grad_bootstrap": (case["gamma"] * final).float()}
    if s["trace"] is not None:
        out["grad_trace"] = _spread(at, weight * _next(s["adv"][at].double(), last, 0.0) * G, n)
    return out


def _sum_by(seq, x, S):
    return torch.zeros(S, dtype=torch.float64, device=x.device).index_add_(0, seq, x.double())


def _plain_policy(s):
    case, p, n, S = s["case"], s["terms"], s["case"]["tokens"], s["case"]["seqs"]
    at, seq, _ = _valid(s)
    lp, old = s["logp"][at], s["old"][at]
    count = _sum_by(seq, torch.ones_like(lp), S).clamp(min=1)
    log_ratio = lp.double() - old.double()  # 64 bits: what lies next to a clip border is told apart
    if case["ratio"] == "sequence":
        log_ratio = (_sum_by(seq, log_ratio, S) / count)[seq]
    A = s["adv"][at] if case["adv"] == "token" else s["adv"][seq]
    if s["white"] is not None:
        A = (A - s["white"][0]) / (s["white"][1] + p["adv_eps"])
    up, low = math.log1p(p["clip_high"]), math.log1p(-p["clip_low"])
    most = math.log(p["dual_clip"]) if p["dual_clip"] else math.inf
    flat = torch.where(A >= 0, log_ratio > up, (log_ratio < low) | (log_ratio > most))
    held = torch.where(A >= 0, log_ratio.clamp(max=up), log_ratio.clamp(min=low, max=most)).float()
    w = torch.full_like(lp, 1.0 / s["norm"]) if case["mean"] == "tokens" else (1.0 / (s["norm"] * count)).float()[seq]
    weight = w
    if s["rollout"] is not None:
        gap = old - s["rollout"][at]
        if case["ratio"] == "sequence":
            gap = (_sum_by(seq, gap, S) / count)[seq].float()
        weight = w * torch.exp(gap).clamp(max=p["rollout_cap"])
    policy = -weight * A * torch.exp(held)
    omega = torch.where(flat, 0.0, -weight * A * torch.exp(log_ratio.float()))
    kl = torch.zeros_like(lp)
    if case["kl"]:
        e = (s["ref"][at].double() - lp.double())  # 64 bits: differences of nearly equal terms
        kl, slope = {1: (-e, torch.ones_like(e)), 2: (e * e / 2, -e), 3: (torch.expm1(e) - e, -torch.expm1(e))}[case["kl"]]
        omega = omega + p["beta"] * w * slope.float()
    wd = w.double()
    parts = [policy.double().sum(), (wd * kl).sum(), (wd * (flat & (A != 0))).sum(), (wd * (old.double() - lp.double())).sum()]
    return {"stats": torch.stack([parts[0] + p["beta"] * parts[1]] + parts).float(), "omega": _spread(at, omega, n)}


def _plain_pref(s):
    case, p, n, S, G = s["case"], s["terms"], s["case"]["tokens"], s["case"]["seqs"], s["case"]["group"]
    at, seq, _ = _valid(s)
    lp = s["logp"][at].double()
    count = _sum_by(seq, torch.ones_like(lp), S)
    size = count.clamp(min=1)
    own_sum = _sum_by(seq, lp, S)
    ratio = own_sum if s["ref"] is None else _sum_by(seq, lp - s["ref"][at].double(), S)
    per = 1.0 / size if case["length"] else torch.ones_like(size)
    h = p["beta"] * per * ratio
    R = s["rewards"].double().view(-1, G)
    real = (count > 0).view(-1, G)
    better = (R[:, :, None] > R[:, None, :]) & real[:, :, None] & real[:, None, :]  # [group, winner, loser]
    gap = h.view(-1, G)[:, :, None] - h.view(-1, G)[:, None, :]
    z = gap - p["margin"] - p["margin_reward"] * (R[:, :, None] - R[:, None, :])
    if case["loss"] == "sigmoid":
        e = p["smoothing"]
        far = torch.log1p(torch.exp(-z.abs()))
        loss = (1 - e) * (far + (-z).clamp(min=0)) + e * (far + z.clamp(min=0))
        slope = e - 1 / (1 + torch.exp(z))
    elif case["loss"] == "hinge":
        loss, slope = (1 - z).clamp(min=0), -(z < 1).double()
    else:
        loss, slope = ((z - 0.5) / p["beta"]) ** 2, 2 * (z - 0.5) / p["beta"] ** 2
    pairs = better.sum()
    unit = 1.0 / pairs.clamp(min=1)
    loss, slope = (torch.where(better, x, 0.0) * unit for x in (loss, slope))
    wins = better.sum(2).view(-1) * unit
    nll = -(own_sum / size * wins).sum()
    c = p["beta"] * per * (slope.sum(2) - slope.sum(1)).view(-1) - p["nll"] * wins / size
    stats = torch.stack([loss.sum() + p["nll"] * nll, (better & (gap > 0)).sum() * unit, torch.where(better, gap, 0.0).sum() * unit, nll])
    return {"stats": stats.float(), "omega": _spread(at, c[seq], n), "scores": h.float(), "pairs": pairs.view(1)}


# ------------------------------------------------------------------------------------------------------------------ run
def run(state):
    s, case = state, state["case"]
    kind, n, S = case["kind"], case["tokens"], case["seqs"]
    if not own:
        return {"adv": _plain_adv, "adv_grad": _plain_adv_grad, "policy": _plain_policy, "pref": _plain_pref}[kind](s)
    api, ws = s["api"], s["workspace"]
    if kind == "adv":
        api.hilore_advantages(s["rewards"], s["outcome"], s["values"], api.BF16 if case["values"] == "bf16" else api.F32, s["bootstrap"], s["trace"],
                              s["mask"], s["cu"], S, n, case["gamma"], case["lam"], s["adv"], s["returns"], s["moments"] if case["moments"] else None,
                              ws, ws.numel())
        return {k: s[k] for k in ["adv", "returns"] + ["moments"] * case["moments"]}
    if kind == "adv_grad":
        api.hilore_advantages_backward(s["grad_adv"], s["grad_returns"], s["adv"] if case["trace"] else None, s["trace"], s["mask"], s["cu"], S, n,
                                       case["gamma"], case["lam"], s["grad_rewards"], s["grad_outcome"], s["grad_values"], s["grad_bootstrap"],
                                       s["grad_trace"] if case["trace"] else None, ws, ws.numel())
        return {k: s[k] for k in ["grad_rewards", "grad_values", "grad_outcome", "grad_bootstrap"] + ["grad_trace"] * case["trace"]}
    if kind == "policy":
        api.hilore_policy_loss(s["logp"], s["old"], s["ref"], s["rollout"], s["mask"], s["adv"], s["white"], s["cu"], S, n, s["handle"], s["norm"], None,
                               None, s["stats"], s["omega"], ws, ws.numel())
        return {"stats": s["stats"], "omega": s["omega"]}
    api.hilore_preference_loss(s["logp"], s["ref"], s["mask"], s["rewards"], case["group"], s["cu"], S, n, s["handle"], 0, None, None, s["scores"],
                               s["pairs"], s["stats"], s["omega"], ws, ws.numel())
    return {k: s[k] for k in ("stats", "omega", "scores", "pairs")}


# ---------------------------------------------------------------------------------------------------------------- exact
def _rows(s, x, fill=0.0):
    """[sequence, place] in 64 bits of a value per token, and the way back."""
    length = s["length"]
    S, L = length.numel(), int(length.max())
    begin = torch.cumsum(length, 0) - length
    place = torch.arange(s["case"]["tokens"], device="cuda") - begin[s["seq"]]
    out = torch.full((S, L), fill, dtype=torch.float64, device="cuda")
    out[s["seq"], place] = x.double()
    return out, (s["seq"], place)


def exact(case, seed):
    s = prepare(case, seed)
    if int(s["length"].max()) * case["seqs"] > 600_000_000:  # one very long sequence among many: rows would not fit
        return None
    return {"adv": _exact_adv, "adv_grad": _exact_adv_grad, "policy": _exact_policy, "pref": _exact_pref}[case["kind"]](s)


def _exact_adv(s):
    """Token by token from the end, as the recurrence is written."""
    case = s["case"]
    m, back = _rows(s, s["mask"])
    if m.shape[1] > 200_000:
        return None
    m = (m > 0).t().contiguous()
    r, v = (_rows(s, s[k])[0].t().contiguous() for k in ("rewards", "values"))
    c = _rows(s, s["trace"])[0].t().contiguous() if case["trace"] else None
    x = torch.zeros(case["seqs"], dtype=torch.float64, device="cuda")
    q = s["outcome"].double() + case["gamma"] * s["bootstrap"].double()
    for k in range(m.shape[0] - 1, -1, -1):
        w = case["gamma"] * case["lam"] * (1.0 if c is None else c[k])
        new = r[k] + q - v[k] + w * x
        x = torch.where(m[k], new, x)
        q = torch.where(m[k], case["gamma"] * v[k], q)
        r[k] = torch.where(m[k], new, 0.0)
    a = r.t()[back]
    out = {"adv": a, "returns": torch.where(s["mask"] > 0, a + s["values"].double(), 0.0)}
    if case["moments"]:
        a = a[s["mask"] > 0]
        out["moments"] = torch.stack([a.mean(), a.std(correction=0)]) if a.numel() else torch.zeros(2, dtype=torch.float64)
    return out


def _exact_adv_grad(s):
    case, w = s["case"], s["case"]["gamma"] * s["case"]["lam"]
    m, back = _rows(s, s["mask"])
    if m.shape[1] > 140_000:
        return None
    m = (m > 0).t().contiguous()
    names = ["grad_adv", "grad_returns"] + (["trace", "adv"] if case["trace"] else [])
    t = {k: _rows(s, s[k])[0].t().contiguous() for k in names}
    G_last = torch.zeros(case["seqs"], dtype=torch.float64, device="cuda")
    at_last = torch.full((case["seqs"],), -1, device="cuda")
    c_last = torch.zeros_like(G_last)
    every = torch.arange(case["seqs"], device="cuda")
    by_trace = torch.zeros_like(t["grad_adv"]) if case["trace"] else None
    for k in range(m.shape[0]):
        G = t["grad_adv"][k] + t["grad_returns"][k] + w * c_last * G_last
        t["grad_adv"][k] = torch.where(m[k], G, 0.0)
        t["grad_returns"][k] = torch.where(m[k], t["grad_returns"][k] - G + case["gamma"] * G_last, 0.0)
        if case["trace"]:
            to = (at_last.clamp(min=0), every)
            by_trace[to] += torch.where(m[k] & (at_last >= 0), w * t["adv"][k] * G_last, 0.0)
        G_last = torch.where(m[k], G, G_last)
        c_last = torch.where(m[k], t["trace"][k] if case["trace"] else 1.0, c_last)
        at_last = torch.where(m[k], k, at_last)
    out = {"grad_rewards": t["grad_adv"].t()[back], "grad_values": t["grad_returns"].t()[back], "grad_outcome": G_last,
           "grad_bootstrap": case["gamma"] * G_last}
    if case["trace"]:
        out["grad_trace"] = by_trace.t()[back]
    return out


def _exact_policy(s):
    """The gradient is autograd's, of the loss in 64 bits over rows of sequences."""
    case, p = s["case"], s["terms"]
    m, back = _rows(s, s["mask"])
    m = m > 0
    lp, old = _rows(s, s["logp"])[0].requires_grad_(), _rows(s, s["old"])[0]
    size = m.sum(1, keepdim=True).clamp(min=1).double()
    mean = lambda x: torch.where(m, x, 0.0).sum(1, keepdim=True) / size  # noqa: E731
    A = _rows(s, s["adv"])[0] if case["adv"] == "token" else s["adv"].double()[:, None]
    if s["white"] is not None:
        A = (A - s["white"][0].double()) / (s["white"][1].double() + p["adv_eps"])
    rho = torch.exp(mean(lp - old) if case["ratio"] == "sequence" else lp - old)
    clipped = A * rho.clamp(1 - p["clip_low"], 1 + p["clip_high"])
    gain = torch.minimum(A * rho, clipped)
    if p["dual_clip"]:
        gain = torch.where(A < 0, torch.maximum(gain, p["dual_clip"] * A), gain)
        over = (A < 0) & (rho > p["dual_clip"])
    else:
        over = torch.zeros_like(gain, dtype=torch.bool)
    flat = (((A > 0) & (rho > 1 + p["clip_high"])) | ((A < 0) & (rho < 1 - p["clip_low"])) | over).expand_as(m)
    w = torch.where(m, 1.0, 0.0) / (s["norm"] if case["mean"] == "tokens" else s["norm"] * size)
    if s["rollout"] is not None:
        gap = old - _rows(s, s["rollout"])[0]
        gain = gain * torch.exp(mean(gap) if case["ratio"] == "sequence" else gap).clamp(max=p["rollout_cap"])
    policy = -(w * gain).sum()
    kl = torch.zeros((), dtype=torch.float64, device="cuda")
    if case["kl"]:
        e = _rows(s, s["ref"])[0] - lp
        kl = (w * {1: -e, 2: e.square() / 2, 3: torch.expm1(e) - e}[case["kl"]]).sum()
    loss = policy + p["beta"] * kl
    grad, = torch.autograd.grad(loss, lp)
    stats = torch.stack([loss, policy, kl, (w * flat).sum(), (w * (old - lp)).sum()]).detach()
    return {"stats": stats, "omega": torch.where(s["mask"] > 0, grad[back], 0.0)}


def _exact_pref(s):
    """Pairs by their two indexes; the gradient is autograd's."""
    case, p, G = s["case"], s["terms"], s["case"]["group"]
    m, back = _rows(s, s["mask"])
    m = m > 0
    lp = _rows(s, s["logp"])[0].requires_grad_()
    count = m.sum(1)
    own_sum = torch.where(m, lp, 0.0).sum(1)
    ratio = own_sum if s["ref"] is None else torch.where(m, lp - _rows(s, s["ref"])[0], 0.0).sum(1)
    h = p["beta"] * (ratio / count.clamp(min=1) if case["length"] else ratio)
    R = s["rewards"].double()
    i = torch.arange(case["seqs"], device="cuda")[:, None].expand(-1, G)
    j = (torch.arange(case["seqs"], device="cuda") // G * G)[:, None] + torch.arange(G, device="cuda")
    pick = (R[i] > R[j]) & (count[i] > 0) & (count[j] > 0)
    i, j = i[pick], j[pick]
    N = max(1, i.numel())
    gap = h[i] - h[j]
    z = gap - p["margin"] - p["margin_reward"] * (R[i] - R[j])
    if case["loss"] == "sigmoid":
        f = torch.nn.functional.logsigmoid
        each = -(1 - p["smoothing"]) * f(z) - p["smoothing"] * f(-z)
    elif case["loss"] == "hinge":
        each = torch.relu(1 - z)
    else:
        each = ((z - 0.5) / p["beta"]) ** 2
    nll = (-own_sum[i] / count[i]).sum() / N
    loss = each.sum() / N + p["nll"] * nll
    grad, = torch.autograd.grad(loss, lp)
    stats = torch.stack([loss, (gap > 0).sum() / N, gap.sum() / N, nll]).detach()
    return {"stats": stats, "omega": torch.where(s["mask"] > 0, grad[back], 0.0), "scores": h.detach(), "pairs": None}
