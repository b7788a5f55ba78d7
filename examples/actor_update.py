"""A small actor trained by the library's calls from end to end: sampling under rules, rewards, log-probabilities under the
same rules, GRPO coefficients, the gradient of the logits, and a clipped AdamW step with 8-bit moments.

    python examples/actor_update.py [iterations]

The actor knows the previous token alone: logits = emb[previous] @ head + bias.  A response earns the share of its tokens
that are even.  PyTorch does the two products of the actor and draws the samples; the rest are calls of the C ABI.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_33570_b200 import api  # noqa: E402

V, D = 1000, 64              # vocabulary, width
PROMPTS, G, P, T = 8, 8, 4, 16   # groups, responses of a group, prompt tokens, response slots
L = P + T
ROWS = PROMPTS * G
EOS = 2                      # ends a response; the slots behind it hold no token


class Actor:
    """Parameters in bf16 with fp32 master copies and 8-bit moments; the bias in fp32 with fp32 moments."""

    def __init__(self, gen, dev):
        f = lambda *s: torch.randn(*s, generator=gen, device=dev) * 0.1
        self.w = dict(emb=f(V, D).to(torch.bfloat16), head=f(D, V).to(torch.bfloat16), bias=torch.zeros(V, device=dev))
        self.g = {k: torch.zeros_like(t) for k, t in self.w.items()}
        entries = []
        for k, t in self.w.items():
            n = t.numel()
            blocks = -(-n // api.BLOCK)
            z = lambda m, dt: torch.zeros(m, dtype=dt, device=dev)
            if t.dtype == torch.bfloat16:
                entries.append(dict(p=t, g=self.g[k], master=t.float(), m=z(n, torch.uint8), v=z(n, torch.uint8),
                                    m_scale=z(blocks, torch.float32), v_scale=z(blocks, torch.float32), weight_decay=0.01))
            else:
                entries.append(dict(p=t, g=self.g[k], m=z(n, torch.float32), v=z(n, torch.float32)))
        self.n = len(entries)
        self.table = api.make_param_table(entries, dev)
        self.norm, self.scale = torch.zeros(1, device=dev), torch.zeros(1, device=dev)
        self.ws = torch.empty(api.hilore_grad_norm_workspace_bytes(), dtype=torch.uint8, device=dev)

    def logits(self, previous):
        h = self.w["emb"][previous]
        return h, (h @ self.w["head"]).float().add_(self.w["bias"]).to(torch.bfloat16)

    def backward(self, previous, h, dlogits):
        self.g["head"].copy_(h.t() @ dlogits)
        self.g["bias"].copy_(dlogits.float().sum(0))
        self.g["emb"].zero_().index_add_(0, previous, dlogits @ self.w["head"].t())

    def step(self, t, lr):
        """The norm over all gradients, then one launch for all tensors; neither result visits the host."""
        dev, host = self.table
        api.hilore_grad_norm(dev, host, self.n, 1.0, self.norm, self.scale, self.ws, self.ws.numel())
        api.hilore_adamw_step(dev, host, self.n, lr, None, 0.9, 0.99, 1e-8, t, None, self.scale)


def rules(tokens, begin, middle, end, allow, dev):
    """Rules of rows whose histories are tokens[begin .. end), generated from `middle` on."""
    n = begin.numel()
    full = lambda v: torch.full((n,), v, device=dev)
    return api.make_logit_rules(temperature=full(0.9), repetition=full(1.2), frequency=full(0.1), presence=full(0.1), tokens=tokens,
                                hist_begin=begin, resp_begin=middle, hist_end=end, allow=allow,
                                allow_row=torch.zeros(n, dtype=torch.int32, device=dev))


def rollout(actor, gen, allow, dev):
    """Token by token: logits, rules in place, a draw.  Returns the packed sequences and the mask of the response slots."""
    seq = torch.full((ROWS, L), -1, dtype=torch.int32, device=dev)               # -1: no token yet, counts nowhere
    seq[:, :P] = torch.randint(3, V, (PROMPTS, P), generator=gen, device=dev, dtype=torch.int32).repeat_interleave(G, 0)
    mask = torch.zeros(ROWS, T, dtype=torch.uint8, device=dev)
    live = torch.ones(ROWS, dtype=torch.bool, device=dev)
    begin = torch.arange(ROWS, device=dev) * L
    for t in range(T):
        _, x = actor.logits(seq[:, P + t - 1].clamp_min(0).long())
        r = rules(seq.view(-1), begin, begin + P, begin + P + t, allow, dev)
        api.hilore_logits_apply(x, api.BF16, ROWS, V, V, r, x, V)
        noise = -torch.log(-torch.log(torch.rand(ROWS, V, generator=gen, device=dev).clamp_min(1e-20)))
        token = (x.float() + noise).argmax(1).int()
        seq[:, P + t] = torch.where(live, token, -1)
        mask[:, t] = live.to(torch.uint8)
        live &= token != EOS
    return seq, mask


def train(iterations=40, epochs=2, lr=0.02, seed=0):
    """Returns the mean reward of each iteration's responses, and the last gradient norm."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    actor = Actor(gen, dev)
    allow = torch.full((1, -(-V // 32)), -1, dtype=torch.int32, device=dev)
    allow[0, 0] = ~0b11                                                          # tokens 0 and 1 are never sampled
    begin = (torch.arange(ROWS, device=dev) * L).repeat_interleave(T)
    end = begin + P + torch.arange(T, device=dev).repeat(ROWS)
    n = ROWS * T
    logp, lse, entropy = (torch.empty(n, device=dev) for _ in range(3))
    omega = torch.empty(ROWS, T, device=dev)
    dlogits = torch.empty(n, V, dtype=torch.bfloat16, device=dev)
    valid = torch.zeros(1, dtype=torch.int64, device=dev)
    rewards, t = [], 0
    for _ in range(iterations):
        seq, mask = rollout(actor, gen, allow, dev)
        token = seq[:, P:]
        reward = (((token % 2 == 0) & (token >= 0)).sum(1) / (token >= 0).sum(1)).float()
        rewards.append(float(reward.mean()))
        r = rules(seq.view(-1), begin, begin + P, end, allow, dev)               # row (i, t): prefixes of sequence i
        targets = token.reshape(-1).contiguous()                                 # -1: a slot without a token
        previous = seq[:, P - 1:-1].reshape(-1).clamp_min(0).long()
        api.hilore_mask_count(mask, n, valid)
        old = None
        for _ in range(epochs):
            h, x = actor.logits(previous)
            api.hilore_token_logp(x, api.BF16, n, V, V, r, targets, logp, lse, entropy)
            if old is None:
                old = logp.clone()
            api.hilore_grpo_coeffs(reward, ROWS, G, 0, ROWS, T, logp.view(ROWS, T), old.view(ROWS, T), None, mask, 0, valid, 0.2, 0.0,
                                   1e-6, None, omega, None, None)
            api.hilore_token_logp_backward(x, api.BF16, n, V, V, r, targets, lse, omega, dlogits, V)
            actor.backward(previous, h, dlogits)
            t += 1
            actor.step(t, lr)
    return rewards, float(actor.norm)


if __name__ == "__main__":
    got, norm = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    for i, r in enumerate(got):
        print(f"iteration {i:3d}  mean reward {r:.3f}")
    print(f"last gradient norm {norm:.4f}")
