"""Cases of the two ends of an actor update that touch the model: rules on logits (penalties for repeated tokens, biases,
grammar masks, temperature), log-probabilities of sampled tokens with their gradient, and the AdamW step with states in
32 or in 8 bits.

`run` computes a case in its plain form (elementary torch operations, 32 bits inside, rounded once at the end) or, where
`own` is true, through the library's entry points.  `exact` is the definition in 64 bits, written apart from both.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 64  # elements that share one scale of an 8-bit state


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one sequence at a decoding step, short history: the latency of the call
        dict(name="rules one row", kind="rules", rows=1, vocab=32064, extra=0, dtype="bf16", history=700, prefix=False, bias=16, grammar=0.0),
        # a decoding batch in fp32 logits: histories up to 16 K tokens, a grammar on half of the rows, user biases
        dict(name="rules decode batch", kind="rules", rows=96, vocab=151936, extra=0, dtype="f32", history=16384, prefix=False, bias=48,
             grammar=0.5),
        # gradients back through the rules for the rows of one training microbatch: every row's history is a prefix
        dict(name="rules gradient prefixes", kind="rules_grad", rows=2048, vocab=128256, extra=0, dtype="bf16", history=1536, prefix=True,
             bias=0, grammar=0.0),
        # log-probabilities of the newest token of eight responses
        dict(name="logp eight tokens", kind="logp", rows=8, vocab=151936, extra=0, dtype="bf16", entropy=False, pad=0.0, rules=False),
        # scoring pass (old or reference policy) of a 1.5B-shaped microbatch: 4 responses x 2048 slots, a quarter of them padding
        dict(name="logp microbatch", kind="logp", rows=8192, vocab=151936, extra=0, dtype="bf16", entropy=True, pad=0.25, rules=False),
        # odd vocabulary, padded leading dimension, fp32 logits, scored under the rules they were sampled with
        dict(name="logp ragged under rules", kind="logp", rows=1021, vocab=50001, extra=7, dtype="f32", entropy=True, pad=0.1, rules=True,
             history=900, prefix=True, bias=24, grammar=0.3),
        # backward of the policy loss from its coefficients: 2 responses x 2048 slots
        dict(name="logp gradient", kind="logp_grad", rows=4096, vocab=151936, extra=0, dtype="bf16", pad=0.25, rules=False),
        # the same under rules, odd vocabulary
        dict(name="logp gradient under rules", kind="logp_grad", rows=1500, vocab=32063, extra=0, dtype="bf16", pad=0.0, rules=True,
             history=1200, prefix=True, bias=0, grammar=0.0),
        # a few odd-sized tensors with 8-bit states: the latency of the call
        dict(name="adamw few small 8 bit", kind="adamw", tensors=9, total=120_001, param="bf16", grad="bf16", master=False, state=8, clip=True),
        # low-rank adapters of a 7B-shaped actor: 28 layers x 7 projections x 2 factors, all fp32
        dict(name="adamw adapters", kind="adamw", tensors=392, total=40_370_176, param="f32", grad="f32", master=False, state=32, clip=True),
        # full-parameter shard: bf16 weights with an fp32 master copy and 32-bit states
        dict(name="adamw master 32 bit", kind="adamw", tensors=146, total=400_000_007, param="bf16", grad="bf16", master=True, state=32,
             clip=False),
        # a full 0.9B shard with 8-bit states, global norm and clipping
        dict(name="adamw shard 8 bit", kind="adamw", tensors=219, total=900_000_001, param="bf16", grad="bf16", master=False, state=8,
             clip=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rules", "rules", "rules_grad", "logp", "logp", "logp_grad", "logp_grad", "adamw", "adamw", "adamw"])
    if kind == "adamw":
        state = rng.choice([8, 32])
        param = rng.choice(["bf16", "f32"])
        master = param == "bf16" and state == 32 and rng.random() < 0.5
        total = _log(rng, 5_000, 400_000_000)
        return dict(kind=kind, tensors=min(_log(rng, 1, 600), max(1, total // 500)), total=total, param=param,
                    grad=rng.choice(["bf16", param]), master=master, state=state, clip=rng.random() < 0.6)
    vocab = _log(rng, 1000, 152000)
    rows = _log(rng, 1, 4096)
    rows = max(1, min(rows, 400_000_000 // vocab))
    case = dict(kind=kind, rows=rows, vocab=vocab, extra=rng.choice([0, 0, 1, 8, 37]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    ruled = True
    if kind in ("logp", "logp_grad"):
        ruled = rng.random() < 0.5
        case.update(pad=rng.choice([0.0, 0.2, 0.5]), rules=ruled)
        if kind == "logp":
            case["entropy"] = rng.random() < 0.5
    if ruled:
        prefix = kind != "rules"
        longest = 2048 if prefix else min(131072, 40_000_000 // rows)
        case.update(history=_log(rng, 1, longest), prefix=prefix, bias=rng.choice([0, 0, 5, 100]), grammar=rng.choice([0.0, 0.0, 0.4, 1.0]))
    return case


def _active(case):
    """Rows that carry a token: the others are padding slots."""
    return case["rows"] - int(case["rows"] * case.get("pad", 0.0))


def _sizes(case):
    """Sizes of the tensors of an adamw case: odd ones, a few large and many small."""
    k, total = case["tensors"], case["total"]
    w = [1.0 / (1 + (7 * i) % k) for i in range(k)]
    sizes = [max(1, int((total - k) * x / sum(w))) for x in w]
    sizes[0] += total - sum(sizes)
    return sizes


def work(case):
    if case["kind"] == "adamw":
        n = case["total"]
        size = {"bf16": 2, "f32": 4}
        per = size[case["grad"]] + size[case["param"]] * (1 if case["master"] else 2) + (8 if case["master"] else 0)
        per += 16 if case["state"] == 32 else 4 + 16.0 / BLOCK
        return {"bytes": n * per, "flops": n * (16 + (2 if case["clip"] else 0))}
    rows, V = case["rows"], case["vocab"]
    es = 2 if case["dtype"] == "bf16" else 4
    act = _active(case)
    side = 0
    if case.get("rules", True):
        side = rows * case["history"] * (0.5 if not case["prefix"] else 0.0) * 4 + rows * case["bias"] * 8 + rows * case["grammar"] * V / 8 + rows * 40
    if case["kind"] == "rules":
        return {"bytes": 2 * rows * V * es + side, "flops": 3 * rows * V}
    if case["kind"] == "rules_grad":
        return {"bytes": 2 * rows * V * es + side, "flops": rows * V}
    if case["kind"] == "logp":
        return {"bytes": act * V * es + side + rows * 16, "flops": act * V * (6 if case["entropy"] else 4)}
    return {"bytes": (act + rows) * V * es + side + rows * 12, "flops": act * V * 5}


# --------------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _rules_inputs(case, g):
    """Histories (prompt, then what was generated), penalties, biases, grammar bits and temperatures of every row."""
    rows, V, H = case["rows"], case["vocab"], case["history"]
    r = {}
    if case["prefix"]:  # rows are the slots of sequences of H tokens: slot t has seen the tokens before t
        prompt = H // 4
        seqs = -(-rows // max(1, H))
        row = torch.arange(rows, device="cuda")
        begin = row // H * H
        r["hist_begin"] = begin
        r["hist_end"] = row
        r["resp_begin"] = torch.minimum(begin + prompt, row)
        n_tokens = seqs * H
    else:
        length = (_uniform(g, rows) * H).long() + 1
        length[0] = H
        end = torch.cumsum(length, 0)
        r["hist_end"] = end
        r["hist_begin"] = end - length
        r["resp_begin"] = end - (length.float() * _uniform(g, rows)).long()
        n_tokens = int(length.sum())
    u = _uniform(g, n_tokens)
    r["tokens"] = (u.pow(3) * V).int().clamp_(max=V - 1)  # few tokens carry most of a text
    flip = _uniform(g, rows) < 0.8
    one = torch.ones(rows, device="cuda")
    r["repetition"] = torch.where(flip, 1.0 + 0.3 * _uniform(g, rows), one)
    r["frequency"] = torch.where(flip, 0.4 * _uniform(g, rows), 0 * one)
    r["presence"] = torch.where(flip, 0.6 * _uniform(g, rows), 0 * one)
    r["temperature"] = 0.6 + 0.6 * _uniform(g, rows)
    if case["bias"]:
        k = min(case["bias"], V)
        stride = V // k  # k different tokens of each row
        r["bias_tokens"] = (torch.arange(k, device="cuda") * stride + (_uniform(g, rows, k) * stride).long()).int().reshape(-1)
        r["bias_values"] = 4.0 * torch.randn(rows * k, generator=g, device="cuda")
        r["bias_offsets"] = torch.arange(rows + 1, device="cuda") * k
    if case["grammar"] > 0:
        words = -(-V // 32)
        bits = torch.randint(-2**31, 2**31 - 1, (rows, words), generator=g, device="cuda", dtype=torch.int64)
        bits &= torch.randint(-2**31, 2**31 - 1, (rows, words), generator=g, device="cuda", dtype=torch.int64)
        r["allow"] = bits.int()
        has = _uniform(g, rows) < case["grammar"]
        has[0] = True
        r["allow_row"] = torch.where(has, torch.arange(rows, device="cuda"), -1).int()
    return r


def _logits(case, g):
    rows, V, ld = case["rows"], case["vocab"], case["vocab"] + case["extra"]
    x = torch.empty(rows, ld, dtype=DTYPES[case["dtype"]], device="cuda")
    return x.normal_(0.0, 3.0, generator=g)[:, :V]


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"] == "adamw":
        return _prepare_adamw(case, g)
    rows, V = case["rows"], case["vocab"]
    s = {"case": dict(case), "logits": _logits(case, g), "rules": _rules_inputs(case, g) if case.get("rules", True) else None}
    x = s["logits"]
    if case["kind"] == "rules":
        s["out"] = torch.empty_like(x)
    elif case["kind"] == "rules_grad":
        s["grad_out"] = torch.randn(rows, V, generator=g, device="cuda").mul_(1e-3).to(x.dtype)
        s["grad"] = torch.empty(rows, V, dtype=x.dtype, device="cuda")
    else:
        t = (_uniform(g, rows) * V).long().clamp_(max=V - 1)
        x[torch.arange(rows, device="cuda"), t] += 12.0  # a sampled token is a likely one
        if s["rules"] and "allow" in s["rules"]:  # and one that the grammar allows
            words = s["rules"]["allow"]
            at = (torch.arange(rows, device="cuda"), t // 32)
            bit = torch.bitwise_left_shift(torch.ones_like(t), t % 32)
            word = words[at].long() & 0xFFFFFFFF | bit
            words[at] = torch.where(word >= 2**31, word - 2**32, word).int()
        idle = torch.randperm(rows, generator=g, device="cuda")[_active(case):]
        t[idle] = -1
        s["targets"] = t.int()
        for name in ("logp", "lse", "entropy"):
            s[name] = torch.zeros(rows, device="cuda")
        if case["kind"] == "logp_grad":
            s["omega"] = torch.randn(rows, generator=g, device="cuda") / rows
            s["omega"][idle] = 0.0
            s["grad"] = torch.empty(rows, V, dtype=x.dtype, device="cuda")
            for a in range(0, rows, 512):  # what the forward pass left behind
                part = {k: v[a:a + 512] for k, v in s.items() if k in ("logits", "targets")}
                s["lse"][a:a + 512] = torch.logsumexp(_plain_rules(part["logits"].float(), _rows_of(s["rules"], a, a + 512)), 1)
            s["lse"][idle] = 0.0
    if own:
        from paper_2609_33570_b200 import api
        s["api"] = api
        s["dtype"] = api.BF16 if x.dtype == torch.bfloat16 else api.F32
        s["handle"] = api.make_logit_rules(**s["rules"]) if s["rules"] else None
    return s


def _prepare_adamw(case, g):
    sizes = _sizes(case)
    # every tensor starts on a 64-element boundary of one flat buffer, as a sharded trainer keeps them; the gaps hold zeros
    room = [-(-n // BLOCK) * BLOCK for n in sizes]
    starts = [0]
    for n in room:
        starts.append(starts[-1] + n)
    total = starts[-1]
    edge = torch.zeros(total + 1, dtype=torch.int8, device="cuda")
    at = torch.tensor(starts[:-1], device="cuda")
    edge.index_add_(0, at, torch.ones(len(sizes), dtype=torch.int8, device="cuda"))
    edge.index_add_(0, at + torch.tensor(sizes, device="cuda"), -torch.ones(len(sizes), dtype=torch.int8, device="cuda"))
    used = torch.cumsum(edge[:total], 0, dtype=torch.int8) > 0
    del edge
    s = {"case": dict(case), "step": 7, "lr": 5e-4, "betas": (0.9, 0.99), "eps": 1e-8, "decay": 0.05, "max_norm": 1.0}
    w = torch.empty(total, device="cuda").normal_(0.0, 0.02, generator=g).mul_(used)
    s["param"] = w.to(DTYPES[case["param"]])
    s["master"] = w if case["master"] else None
    # gradients and moments differ in size from one block of weights to the next
    size = torch.exp(torch.randn(total // BLOCK, generator=g, device="cuda")).mul_(2e-5).repeat_interleave(BLOCK).mul_(used)
    s["grad"] = torch.empty(total, device="cuda").normal_(generator=g).mul_(size).to(DTYPES[case["grad"]])
    m = torch.empty(total, device="cuda").normal_(generator=g).mul_(size).mul_(0.3)
    r = torch.empty(total, device="cuda").normal_(generator=g).abs_().add_(0.2).mul_(size)
    if case["state"] == 8:
        for name, x in (("m", m), ("v", r)):
            amax = x.view(-1, BLOCK).abs().amax(1)
            scale = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
            s[name] = (x.view(-1, BLOCK) / scale[:, None]).view(-1).to(torch.float8_e4m3fn)
            s[name + "_scale"] = scale
    else:
        s["m"], s["v"] = m, r.square()
    s["norm"], s["scale"] = torch.zeros(1, device="cuda"), torch.ones(1, device="cuda")
    if own:
        from paper_2609_33570_b200 import api
        s["api"] = api
        entries = []
        for n, a in zip(sizes, starts):
            e = dict(p=s["param"][a:a + n], g=s["grad"][a:a + n], m=s["m"][a:a + n], v=s["v"][a:a + n], weight_decay=s["decay"])
            if case["master"]:
                e["master"] = s["master"][a:a + n]
            if case["state"] == 8:
                e["m_scale"], e["v_scale"] = (s[k][a // BLOCK:(a + n + BLOCK - 1) // BLOCK] for k in ("m_scale", "v_scale"))
            entries.append(e)
        s["table"] = api.make_param_table(entries)
        s["workspace"] = torch.zeros(api.hilore_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")
    return s


def _rows_of(r, a, b):
    """The rules of rows [a, b)."""
    if r is None:
        return None
    return {k: v if k in ("tokens", "allow", "bias_tokens", "bias_values") else v[a:b + 1] if k == "bias_offsets" else v[a:b] for k, v in r.items()}


# ---------------------------------------------------------------------------------------------------------- plain forms
def _pairs(begin, end):
    """Row and place of every element of the ranges [begin, end)."""
    n = end - begin
    row = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n)
    first = torch.cumsum(n, 0) - n
    return row, torch.arange(row.numel(), device="cuda") - first[row] + begin[row]


def _counts(r, rows, V, begin):
    row, at = _pairs(r[begin], r["hist_end"])
    c = torch.zeros(rows * V, device="cuda")
    return c.scatter_add_(0, row * V + r["tokens"][at].long(), torch.ones(row.numel(), device="cuda")).view(rows, V)


def _allowed(r, V):
    words = r["allow"][r["allow_row"].clamp(min=0).long()]
    bit = (words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return (bit.view(words.shape[0], -1)[:, :V] > 0) | (r["allow_row"] < 0)[:, None]


def _plain_rules(x, r):
    if r is None:
        return x
    rows, V = x.shape
    rep, freq, pres = r["repetition"][:, None], r["frequency"][:, None], r["presence"][:, None]
    z = torch.where(_counts(r, rows, V, "hist_begin") > 0, torch.where(x > 0, x / rep, x * rep), x)
    out = _counts(r, rows, V, "resp_begin")
    z = z - freq * out - pres * (out > 0)
    if "bias_tokens" in r:
        row, at = _pairs(r["bias_offsets"][:-1], r["bias_offsets"][1:])
        z[row, r["bias_tokens"][at].long()] += r["bias_values"][at]
    z = z / r["temperature"][:, None]
    if "allow" in r:
        z = torch.where(_allowed(r, V), z, -math.inf)
    return z


def _plain_slope(x, r):
    """What a processed logit changes by, per change of the logit itself."""
    rows, V = x.shape
    rep = r["repetition"][:, None]
    k = torch.where(_counts(r, rows, V, "hist_begin") > 0, torch.where(x > 0, 1 / rep, rep), torch.ones_like(x)) / r["temperature"][:, None]
    if "allow" in r:
        k = torch.where(_allowed(r, V), k, 0.0)
    return k


def _plain_logits(s):
    x = s["logits"].float()
    kind = s["case"]["kind"]
    if kind == "rules":
        return _plain_rules(x, s["rules"]).to(s["logits"].dtype)
    if kind == "rules_grad":
        return (s["grad_out"].float() * _plain_slope(x, s["rules"])).to(s["logits"].dtype)
    t = s["targets"].long()
    real = t >= 0
    z = _plain_rules(x, s["rules"])
    if kind == "logp":
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1)
        lse = top[:, 0] + torch.log(total)
        logp = z.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse
        res = [torch.where(real, v, 0.0) for v in (logp, lse)]
        if s["case"]["entropy"]:
            mean = torch.where(e > 0, e * (z - top), 0.0).sum(1) / total
            res.append(torch.where(real, torch.log(total) - mean, 0.0))
        return res
    d = -s["omega"][:, None] * torch.exp(z - s["lse"][:, None])
    d.scatter_add_(1, t.clamp(min=0)[:, None], s["omega"][:, None])
    if s["rules"] is not None:
        d = d * _plain_slope(x, s["rules"])
    return torch.where(real[:, None], d, 0.0).to(s["logits"].dtype)


def _pack(x):
    """Codes and scales of blocks of 64 (E4M3FN, largest magnitude to 448); a positive value of v never becomes zero."""
    x = x.view(-1, BLOCK)
    amax = x.abs().amax(1, keepdim=True)
    scale = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
    q = x * torch.where(amax > 0, 448 / amax, torch.ones_like(amax))
    return q, scale


def _plain_adamw(s):
    case = s["case"]
    b1, b2 = s["betas"]
    g = s["grad"].float()
    if case["clip"]:
        norm = g.square().sum(dtype=torch.float64).sqrt()
        s["norm"].copy_(norm)
        s["scale"].copy_(torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0))
        g = g * s["scale"]
    if case["state"] == 8:
        m, v = ((s[k].float().view(-1, BLOCK) * s[k + "_scale"][:, None]).view(-1) for k in ("m", "v"))
        v = v * v
    else:
        m, v = s["m"], s["v"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    root = torch.sqrt(v)
    p = s["master"] if case["master"] else s["param"].float()
    p = p - s["lr"] * (s["decay"] * p + m / (1 - b1 ** s["step"]) / (root / math.sqrt(1 - b2 ** s["step"]) + s["eps"]))
    if case["master"]:
        s["master"].copy_(p)
    s["param"].copy_(p)
    if case["state"] == 8:
        q, scale = _pack(m)
        s["m"].copy_(q.view(-1))
        s["m_scale"].copy_(scale[:, 0])
        q, scale = _pack(root)
        s["v"].copy_(torch.where(q > 0, q.clamp(min=2.0 ** -9), q).view(-1))
        s["v_scale"].copy_(scale[:, 0])
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _updated(s)


def _updated(s):
    """The state after a step: codes of 8-bit states as the E4M3FN values they are, beside their scales."""
    names = ["param", "m", "v"] + (["master"] if s["case"]["master"] else []) + (["m_scale", "v_scale"] if s["case"]["state"] == 8 else [])
    return {k: s[k] for k in names + (["norm", "scale"] if s["case"]["clip"] else [])}


# ------------------------------------------------------------------------------------------------------------------ run
def run(state):
    s, case = state, state["case"]
    if not own:
        return _plain_adamw(s) if case["kind"] == "adamw" else _plain_logits(s)
    api, kind = s["api"], case["kind"]
    if kind == "adamw":
        dev, host = s["table"]
        k = case["tensors"]
        if case["clip"]:
            api.hilore_grad_norm(dev, host, k, s["max_norm"], s["norm"], s["scale"], s["workspace"], s["workspace"].numel())
        api.hilore_adamw_step(dev, host, k, s["lr"], None, s["betas"][0], s["betas"][1], s["eps"], s["step"], None,
                              s["scale"] if case["clip"] else None)
        return _updated(s)
    x, rows, V = s["logits"], case["rows"], case["vocab"]
    ld = V + case["extra"]
    if kind == "rules":
        api.hilore_logits_apply(x, s["dtype"], rows, V, ld, s["handle"], s["out"], s["out"].stride(0))
        return s["out"]
    if kind == "rules_grad":
        api.hilore_logits_apply_backward(x, s["dtype"], rows, V, ld, s["handle"], s["grad_out"], V, s["grad"], V)
        return s["grad"]
    if kind == "logp":
        api.hilore_token_logp(x, s["dtype"], rows, V, ld, s["handle"], s["targets"], s["logp"], s["lse"], s["entropy"] if case["entropy"] else None)
        return [s["logp"], s["lse"]] + ([s["entropy"]] if case["entropy"] else [])
    api.hilore_token_logp_backward(x, s["dtype"], rows, V, ld, s["handle"], s["targets"], s["lse"], s["omega"], s["grad"], V)
    return s["grad"]


# ---------------------------------------------------------------------------------------------------------------- exact
def _exact_row(z, r, i):
    """Processed logits of row i and their derivative, in 64 bits, from the definition."""
    V = z.numel()
    slope = torch.ones_like(z)
    if r is None:
        return z, slope
    tokens = r["tokens"]
    b, m, e = (int(r["spans"][i][k]) for k in range(3))
    rep, freq, pres, temp = (float(x) for x in r["levels"][i])
    z = z.clone()
    if e > b:
        seen = torch.unique(tokens[b:e].long())
        factor = torch.where(z[seen] > 0, 1.0 / rep, rep).double()
        slope[seen] = factor
        z[seen] = z[seen] * factor
    if e > m:
        tok, count = torch.unique(tokens[m:e].long(), return_counts=True)
        z[tok] -= freq * count.double() + pres
    if "bias_tokens" in r:
        k = r["bias_tokens"].numel() // (r["bias_offsets"].numel() - 1)
        z[r["bias_tokens"][i * k:(i + 1) * k].long()] += r["bias_values"][i * k:(i + 1) * k].double()
    z, slope = z / temp, slope / temp
    if "allow" in r and r["rows_of_allow"][i] >= 0:
        word = r["allow"][r["rows_of_allow"][i]].long()
        v = torch.arange(V, device="cuda")
        no = torch.bitwise_right_shift(word[v // 32] & 0xFFFFFFFF, v % 32) % 2 == 0
        z[no] = -math.inf
        slope[no] = 0.0
    return z, slope


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    r = s["rules"]
    if r is not None:
        r["spans"] = torch.stack([r["hist_begin"], r["resp_begin"], r["hist_end"]], 1).tolist()
        r["levels"] = torch.stack([r[k].double() for k in ("repetition", "frequency", "presence", "temperature")], 1).tolist()
        if "allow" in r:
            r["rows_of_allow"] = r["allow_row"].tolist()
    rows, V, kind = case["rows"], case["vocab"], case["kind"]
    targets = s["targets"].tolist() if "targets" in s else None
    whole = torch.zeros(rows, V, dtype=torch.float64, device="cuda") if kind not in ("logp",) else None
    cols = [torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(3)]
    for i in range(rows):
        if targets is not None and targets[i] < 0:
            continue
        z, slope = _exact_row(s["logits"][i].double(), r, i)
        if kind == "rules":
            whole[i] = z
        elif kind == "rules_grad":
            whole[i] = s["grad_out"][i].double() * slope
        else:
            lse = torch.logsumexp(z, 0)
            p = torch.exp(z - lse)
            if kind == "logp":
                cols[0][i] = z[targets[i]] - lse
                cols[1][i] = lse
                if case["entropy"]:
                    cols[2][i] = -torch.xlogy(p, p).sum()
            else:
                p.neg_()
                p[targets[i]] += 1
                whole[i] = s["omega"][i].double() * p * slope
    if kind == "logp":
        return cols if case["entropy"] else cols[:2]
    return whole


def _exact_adamw(s):
    case, (b1, b2), t = s["case"], s["betas"], s["step"]
    g = s["grad"].double()
    res = {}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        scale = min(1.0, s["max_norm"] / (float(norm) + 1e-6))
        res["norm"], res["scale"] = norm.reshape(1), torch.tensor([scale], dtype=torch.float64)
        g = g * scale
    m, v = s["m"].double(), s["v"].double()
    if case["state"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = m + (1 - b1) * (g - m)
    v = v + (1 - b2) * (g * g - v)
    p = (s["master"] if case["master"] else s["param"]).double()
    p = (1 - s["lr"] * s["decay"]) * p - s["lr"] * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + s["eps"])
    res["param"] = p
    if case["master"]:
        res["master"] = p
    if case["state"] == 8:  # the values that the codes round, in units of their block's scale
        for name, x in (("m", m), ("v", torch.sqrt(v))):
            x = x.view(-1, BLOCK)
            top = x.abs().amax(1, keepdim=True)
            unit = torch.where(top > 0, top / 448, torch.ones_like(top))
            res[name], res[name + "_scale"] = (x / unit).view(-1), unit[:, 0]
    else:
        res["m"], res["v"] = m, v
    return res
