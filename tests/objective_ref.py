"""Plain NumPy definitions in 64 bits of the advantages with their backward pass, the policy loss and the preference loss, and the
error bounds that the GPU tests hold the kernels to.

u = 2^-24 is the unit roundoff of fp32, e = 2^-53 that of fp64.  The bounds count roundings; none was fitted to a result.
"""
from __future__ import annotations

import numpy as np

U, E = 2.0 ** -24, 2.0 ** -53
RATIO_TOKEN, RATIO_SEQUENCE, MEAN_TOKENS, MEAN_SEQUENCES = 0, 1, 0, 1


def valid_places(mask, bounds):
    """Places of the valid tokens of each sequence."""
    return [np.array([t for t in range(a, b) if mask is None or mask[t]], np.int64) for a, b in zip(bounds[:-1], bounds[1:])]


def f64(x, n):
    return np.zeros(n) if x is None else np.asarray(x, np.float64)


# ----------------------------------------------------------------------------------------------------------- advantages
def advantages(rewards, outcome, values, bootstrap, trace, mask, bounds, n_tok, gamma, lam):
    """-> adv, returns, (mean, std), bound of adv and returns.  Every A is a sum of products of what precedes it in the recurrence; a
    length of n tokens gives at most 4 n roundings of fp64 relative to the sum of the terms' sizes, and one to fp32."""
    S = len(bounds) - 1
    r, v, o, b = f64(rewards, n_tok), f64(values, n_tok), f64(outcome, S), f64(bootstrap, S)
    c = np.ones(n_tok) if trace is None else np.asarray(trace, np.float64)
    adv, ret, size = np.zeros(n_tok), np.zeros(n_tok), np.zeros(n_tok)
    with np.errstate(invalid="ignore", over="ignore"):
        for s, at in enumerate(valid_places(mask, bounds)):
            A, q, big, q_big = 0.0, o[s] + gamma * b[s], 0.0, abs(o[s]) + abs(gamma * b[s])
            for t in at[::-1]:
                w = gamma * lam * c[t]
                A, big = r[t] + q - v[t] + w * A, abs(r[t]) + abs(v[t]) + q_big + abs(w) * big
                q, q_big = gamma * v[t], abs(gamma * v[t])
                adv[t], ret[t], size[t] = A, A + v[t], big + abs(v[t])
    at = np.concatenate(valid_places(mask, bounds)) if S else np.zeros(0, np.int64)
    a = adv[at]
    with np.errstate(invalid="ignore"):
        moments = (a.mean(), a.std()) if a.size else (0.0, 0.0)
    return adv, ret, moments, 4 * max(8, n_tok) * E * size


def advantages_backward(grad_adv, grad_returns, adv, trace, mask, bounds, n_tok, gamma, lam):
    S = len(bounds) - 1
    ga, gr, A = f64(grad_adv, n_tok), f64(grad_returns, n_tok), f64(adv, n_tok)
    c = np.ones(n_tok) if trace is None else np.asarray(trace, np.float64)
    out = dict(rewards=np.zeros(n_tok), values=np.zeros(n_tok), trace=np.zeros(n_tok), outcome=np.zeros(S), bootstrap=np.zeros(S))
    slack = {k: np.zeros_like(x) for k, x in out.items()}
    few = 4 * max(8, n_tok) * E
    for s, at in enumerate(valid_places(mask, bounds)):
        G, y, big, last = 0.0, 0.0, 0.0, -1
        y_big = 0.0
        for t in at:
            g_before, b_before = G, big
            G, big = ga[t] + gr[t] + y, abs(ga[t]) + abs(gr[t]) + y_big
            out["rewards"][t], slack["rewards"][t] = G, few * big
            out["values"][t] = gr[t] - G + gamma * g_before
            slack["values"][t] = few * (abs(gr[t]) + big + gamma * b_before)
            if last >= 0:
                out["trace"][last] = gamma * lam * A[t] * g_before
                slack["trace"][last] = few * abs(gamma * lam * A[t]) * b_before
            y, y_big, last = gamma * lam * c[t] * G, abs(gamma * lam * c[t]) * big, t
        if at.size:
            out["outcome"][s], out["bootstrap"][s] = G, gamma * G
            slack["outcome"][s], slack["bootstrap"][s] = few * big, few * big
    return out, slack


# ---------------------------------------------------------------------------------------------------------- policy loss
def policy(logp, old, ref, rollout, mask, adv, moments, bounds, t, N, grad_loss=1.0):
    """t: dict of the terms.  -> stats, omega, bounds of both.  Bounds per token, in units of u: the exponentials are 2 ulp = 4 u off
    and move by |x| u with the rounding of their argument x; at most eight products and weights are rounded beside them.  The
    KL term's derivative for |e| <= 1 is a series of relative error 12 u at an argument that is |e| u off."""
    n = len(logp)
    lp, lo = np.asarray(logp, np.float64), np.asarray(old, np.float64)
    lr, lb = (None if x is None else np.asarray(x, np.float64) for x in (ref, rollout))
    omega, tol = np.zeros(n), np.zeros(n)
    stats, slack = np.zeros(5), np.zeros(5)
    white = lambda a: a if moments is None else (a - float(moments[0])) / (float(moments[1]) + t["adv_eps"])
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        up, low = np.log1p(t["clip_high"]), np.log1p(-t["clip_low"])
        most = np.log(t["dual_clip"]) if t["dual_clip"] else np.inf
        for s, at in enumerate(valid_places(mask, bounds)):
            if not at.size or not N > 0:
                continue
            w = 1.0 / N if t["mean"] == MEAN_TOKENS else 1.0 / (N * at.size)
            d = lp[at] - lo[at]
            gap = np.zeros(at.size) if lb is None else lo[at] - lb[at]
            if t["ratio"] == RATIO_SEQUENCE:
                d, gap = np.full(at.size, d.mean()), np.full(at.size, gap.mean())
            A = white(np.asarray(adv, np.float64)[at] if t["adv_per_token"] else np.full(at.size, float(adv[s])))
            rho, i = np.exp(d), np.where(np.exp(gap) > t["rollout_cap"], t["rollout_cap"], np.exp(gap))
            flat = np.where(A >= 0, d > up, (d < low) | (d > most))
            u = np.where(~flat, rho, np.where(A >= 0, 1 + t["clip_high"], np.where(d < low, 1 - t["clip_low"], t["dual_clip"])))
            term = -w * i * A * u
            g = np.where(flat, 0.0, -w * i * A * rho)
            near = (16 + np.abs(d) + np.abs(gap)) * U
            g_tol = near * np.abs(g)
            stats[1] += term.sum()
            slack[1] += (near * np.abs(term)).sum() + 8 * U * np.abs(term).sum()
            stats[3] += (w * (flat & (A != 0))).sum()
            slack[3] += 10 * U * w * at.size
            drift = w * (lo[at] - lp[at])
            stats[4] += drift.sum()
            slack[4] += 12 * U * np.abs(drift).sum()
            if lr is not None:
                e = lr[at] - lp[at]
                kl, slope = {1: (-e, np.ones_like(e)), 2: (e * e / 2, -e), 3: (np.expm1(e) - e, -np.expm1(e))}[t["kl"]]
                stats[2] += w * kl.sum()
                kl_tol = w * U * np.where(np.abs(e) <= 1, 16 * np.abs(kl) + e * e, (8 + np.abs(e)) * (np.exp(e) + 1 + np.abs(e)))
                slack[2] += (kl_tol + 8 * U * w * np.abs(kl)).sum()
                if t["beta"]:
                    g = g + t["beta"] * w * slope
                    s_tol = np.where(np.abs(e) <= 1, np.abs(e) * np.exp(e) + 16 * np.abs(slope), (8 + np.abs(e)) * (np.exp(e) + 1)) * U
                    g_tol = g_tol + abs(t["beta"]) * w * (s_tol + 6 * U * np.abs(slope)) + U * np.abs(g)
            omega[at], tol[at] = g * grad_loss, (g_tol + 2 * U * np.abs(g)) * abs(grad_loss)
    stats[0] = stats[1] + (t["beta"] * stats[2] if t["beta"] else 0.0)
    slack[0] = slack[1] + abs(t["beta"]) * slack[2]
    return stats, omega, slack + U * np.abs(stats), tol


# ------------------------------------------------------------------------------------------------------ preference loss
def preference(logp, ref, mask, rewards, G, bounds, t, N=0, grad_loss=1.0):
    """t: dict of the terms; N = 0: the pairs of the call, None: a device count that is not positive.  -> stats, omega, scores, pairs,
    and the bounds of omega and stats: a score of n tokens is n e off relative to the sum of its terms' sizes, a slope as much as its
    two scores times its steepest change; then one rounding to fp32."""
    n, S = len(logp), len(rewards)
    lp = np.asarray(logp, np.float64)
    lr = np.zeros(n) if ref is None else np.asarray(ref, np.float64)
    R = np.asarray(rewards, np.float64)
    at = valid_places(mask, bounds)
    size = np.array([a.size for a in at])
    like = np.array([lp[a].sum() for a in at])
    h = np.array([t["beta"] * (lp[a] - lr[a]).sum() for a in at])
    off = np.array([t["beta"] * (a.size + 40) * E * (np.abs(lp[a]) + np.abs(lr[a])).sum() for a in at])
    per = np.where(size > 0, 1.0 / np.maximum(size, 1), 0.0)
    if t["length_mean"]:
        h, off = h * per, off * per
    c, tol = np.zeros(S), np.zeros(S)
    sums, pairs, slack = np.zeros(4), 0, np.zeros(4)
    for i in range(S):
        for j in range(i // G * G, i // G * G + G):
            if not R[i] > R[j] or not size[i] or not size[j]:
                continue
            gap = h[i] - h[j]
            z = gap - t["margin"] - (t["margin_reward"] * (R[i] - R[j]) if t["margin_reward"] else 0.0)
            if t["loss"] == 0:
                sm = t["smoothing"]
                lose, win = np.logaddexp(0.0, -z), np.logaddexp(0.0, z)
                value, slope, steep = (1 - sm) * lose + (sm * win if sm else 0.0), sm - 1 / (1 + np.exp(z)), 0.25
            elif t["loss"] == 1:
                value, slope, steep = max(0.0, 1 - z), -1.0 if z < 1 else 0.0, 0.0
            else:
                value, slope, steep = ((z - 0.5) / t["beta"]) ** 2, 2 * (z - 0.5) / t["beta"] ** 2, 2 / t["beta"] ** 2
            mean = t["beta"] * (per if t["length_mean"] else np.ones(S))
            c[i] += mean[i] * slope - t["nll"] * per[i]
            c[j] -= mean[j] * slope
            e = steep * (off[i] + off[j] + 8 * E * (abs(h[i]) + abs(h[j]) + 1)) + 16 * E * abs(slope)
            tol[i] += mean[i] * e + 8 * E * t["nll"] * per[i]
            tol[j] += mean[j] * e
            pairs += 1
            sums += (value, gap > 0, gap, -like[i] * per[i])
            slack += (abs(slope) * (off[i] + off[j]) + e, 0, off[i] + off[j], off[i] / t["beta"] * (1 if t["length_mean"] else per[i]) + E * abs(like[i] * per[i]))
    N = pairs if N == 0 else (0 if N is None else N)
    stats, omega, o_tol = np.zeros(4), np.zeros(n), np.zeros(n)
    if N and pairs:
        sums[0] += t["nll"] * sums[3]
        slack[0] += abs(t["nll"]) * slack[3]
        stats = sums / N
        for s in range(S):
            omega[at[s]] = c[s] / N * grad_loss
            o_tol[at[s]] = (tol[s] / N + 8 * E * abs(c[s]) / N) * abs(grad_loss)
        slack = slack / N + (pairs + 8) * E * np.abs(stats)
    return stats, omega, h, pairs, o_tol + U * np.abs(omega), slack + U * np.abs(stats), off + U * np.abs(h)
