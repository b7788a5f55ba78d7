"""The example of an actor update with the policy and the preference loss: it runs, and its gradients are those of the losses as torch
differentiates them in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "actor_update.py")


def example():
    spec = importlib.util.spec_from_file_location("actor_update", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def policy(s, v, valid):
    """Whitened advantages of the step, the clipped ratio with its bound for large ones, K3 to the reference, means of sequences."""
    loss, t = v["loss"], v["loss"].policy
    A = (loss.adv.double() - loss.moments[0].double()) / (loss.moments[1].double() + t.adv_eps)
    rho = (s - v["old"].double().view_as(s)).exp()
    held = torch.where(A >= 0, rho.clamp(max=1 + t.clip_high), rho.clamp(1 - t.clip_low, t.dual_clip))
    e = v["ref"].double().view_as(s) - s
    each = -A * held + t.beta * (torch.expm1(e) - e)
    size = valid.sum(1, keepdim=True)
    return torch.where(valid, each / (len(s) * size), 0.0).sum()


def preference(s, v, valid, group):
    t = v["loss"].preference
    zero = torch.zeros_like(s)
    size = valid.sum(1).clamp(min=1)
    h = t.beta * torch.where(valid, s - v["ref"].double().view_as(s), zero).sum(1)
    mean = torch.where(valid, s, zero).sum(1) / size
    r, h, mean = (x.view(-1, group) for x in (v["reward"], h, mean))
    better = r[:, :, None] > r[:, None, :]
    z = (h[:, :, None] - h[:, None, :])[better]
    won = mean[:, :, None].expand_as(better)[better]
    return (-torch.nn.functional.logsigmoid(z) - t.nll * won).mean()


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_losses_of_the_example(kind):
    mod = example()
    seen = []

    def watch(v):
        valid = v["mask"] > 0
        s = torch.where(valid, v["logp"].view(valid.shape).double(), 0.0).requires_grad_()
        value = policy(s, v, valid) if kind == "policy" else preference(s, v, valid, mod.G)
        want, = torch.autograd.grad(value, s)
        value = value.detach()
        got, bits = v["omega"].double(), 2.0 ** -24
        # some twenty roundings of a token's terms, each no larger than the largest weight times the largest advantage or score
        scale = want.abs().max(1, keepdim=True).values.clamp(min=float(want.abs().max()) * 1e-2)
        assert bool(((got - want).abs() <= 64 * bits * scale).all()), float(((got - want).abs() / scale).max() / bits)
        assert not bool(got[~valid].any())
        assert abs(float(v["loss"].stats[0]) - float(value)) <= 64 * bits * max(1.0, abs(float(value)))
        # masked slots have no gradient of the logits
        assert bool(torch.isfinite(v["dlogits"].float()).all()) and not bool(v["dlogits"].view(*valid.shape, -1)[~valid].any())
        seen.append(value)

    rewards, norm = mod.train(3, kind=kind, watch=watch)
    assert len(rewards) == 3 and len(seen) == 6 and np.isfinite(rewards).all() and np.isfinite(norm) and norm > 0
