"""Plain NumPy definitions in 64 bits of the logit rules, the token log-probabilities with their gradient, the gradient
norm and the AdamW step, and the error bounds that the GPU tests hold the fp32 kernels to.

u = 2^-24 is the unit roundoff of fp32.  The bounds count roundings; none of them was fitted to a result.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
BF16_HALF = 2.0 ** -8          # relative size of a rounding to bf16 (8 significant bits: half of 2^-7)
LOG2E = 1.4426950408889634


# ---------------------------------------------------------------------------------------------------------------- rules
def rules_row(x, r, i):
    """Row i of fp64 logits -> (z, dz/dx, bound of the fp32 error of z)."""
    x = np.asarray(x, np.float64)
    V = x.size
    z, k, size = x.copy(), np.ones(V), np.abs(x)
    get = lambda name, default: float(r[name][i]) if r.get(name) is not None else default
    rep, freq, pres = get("repetition", 1.0), get("frequency", 0.0), get("presence", 0.0)
    T = get("temperature", 1.0)
    T = T if T > 0 else 1.0
    if r.get("tokens") is not None and any(r.get(n) is not None for n in ("repetition", "frequency", "presence")):
        n = len(r["tokens"])
        b, mid, e = max(0, int(r["hist_begin"][i])), int(r["resp_begin"][i]), min(n, int(r["hist_end"][i]))
        hist = np.asarray(r["tokens"][b:e], np.int64)
        gen = hist[max(0, mid - b):] if mid < e else hist[:0]
        hist, gen = hist[(hist >= 0) & (hist < V)], gen[(gen >= 0) & (gen < V)]
        seen, c = np.bincount(hist, minlength=V) > 0, np.bincount(gen, minlength=V)
        with np.errstate(invalid="ignore"):
            f = np.where(x > 0, 1.0 / rep, rep)
        k = np.where(seen, f, k)
        z = np.where(seen, x * f, z)
        z = np.where(c > 0, z - freq * c - pres, z)
        size = np.abs(x) * max(rep, 1 / rep) + abs(freq) * c + abs(pres)
    if r.get("bias_tokens") is not None:
        last = {}
        for j in range(int(r["bias_offsets"][i]), int(r["bias_offsets"][i + 1])):
            v = int(r["bias_tokens"][j])
            if 0 <= v < V:
                last[v] = float(r["bias_values"][j])
        for v, b in last.items():
            z[v] += b
            size[v] += abs(b)
    z, k, size = z / T, k / T, size / T
    free = allowed_row(r, i, V)
    z, k = np.where(free, z, -np.inf), np.where(free, k, 0.0)
    return z, k, 8 * U * size   # at most eight roundings, each relative to a term of `size`


def allowed_row(r, i, V):
    if r.get("allow") is None:
        return np.ones(V, bool)
    a = int(r["allow_row"][i]) if r.get("allow_row") is not None else i
    if not 0 <= a < r["allow"].shape[0]:
        return np.ones(V, bool)
    w = r["allow"][a].view(np.uint32)
    v = np.arange(V)
    return (w[v // 32] >> (v % 32).astype(np.uint32) & 1).astype(bool)


def logp_row(z, a):
    """(logp, lse, entropy) of token a under fp64 logits z; the stated values at the edges."""
    if not 0 <= a < z.size:
        return 0.0, 0.0, 0.0
    if np.isnan(z).any():
        return np.nan, np.nan, np.nan
    top = z.max()
    if top == -np.inf:
        return -np.inf, -np.inf, 0.0
    if top == np.inf:
        return (np.nan if z[a] == np.inf else -np.inf), np.inf, np.nan
    e = np.exp(z - top)
    s = e.sum()
    d = np.where(e > 0, z - top, 0.0)
    return z[a] - top - np.log(s), top + np.log(s), np.log(s) - (e * d).sum() / s


def logp_bound(z, zerr, V):
    """Bound of the fp32 error of logp, lse and entropy: the logits' own error (twice: token and sum), the exponent
    (3 u |z - m| averaged over p, at most 3 u (ln V + 1)), ex2.approx (2^-22), the additions in sequence in a thread (two
    chains over its share of the row) and across them, logarithm and joins; the entropy multiplies them by ln V + 1."""
    finite = np.isfinite(z)
    ez = zerr[finite].max() if finite.any() else 0.0
    zmax = np.abs(z[finite]).max() if finite.any() else 0.0
    adds = V / 256 + 40
    lnv = np.log(V) + 1
    err = 2 * ez + 3 * U * lnv + 2.0 ** -22 + adds * U
    return err, err + 4 * U * zmax, err * lnv + 4 * U * lnv


def grad_row(z, k, a, omega, lse):
    """omega (1[v = a] - p_v) k_v; zeros for rows that the definition leaves out."""
    if not 0 <= a < z.size or omega == 0 or lse <= -1e30 or z[a] == -np.inf and k[a] == 0:
        return np.zeros(z.size)
    p = np.exp(z - lse)
    d = -p
    d[a] += 1
    return np.where(k == 0, 0.0, omega * d * k)


def grad_bound(z, zerr, k, omega, lse, lse_err):
    """|omega| k (p (error of the exponent + 2^-22) + 6 roundings of terms up to 1)."""
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(np.isfinite(z), np.exp(np.minimum(z - lse, 80.0)), 0.0)
        exponent = np.where(np.isfinite(z), zerr + 3 * U * (np.abs(z) + abs(lse)), 0.0) + lse_err + 2.0 ** -22
    return abs(omega) * k * (p * exponent + 6 * U)


# ------------------------------------------------------------------------------------------------------------ AdamW step
def e4m3_values():
    c = np.arange(256)
    s, e, f = np.where(c & 128, -1.0, 1.0), (c >> 3) & 15, (c & 7).astype(np.float64)
    v = np.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * 2.0 ** (e.astype(float) - 7)) * s
    v[(c & 127) == 127] = np.nan
    return v


E4M3 = e4m3_values()


def decode(codes, scales):
    """Values of block-scaled codes (n elements, ceil(n / 64) scales)."""
    return E4M3[codes] * np.repeat(scales.astype(np.float64), 64)[:codes.size]


def e4m3_round(q):
    """Nearest E4M3FN value to q (ties to even), saturating at +-448."""
    a = np.minimum(np.abs(q), 448.0)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -20))), -6.0)
    step = 2.0 ** (e - 3)
    return np.copysign(np.minimum(np.rint(a / step) * step, 448.0), q)


def tie_distance(q):
    """Distance of |q| to the nearest point halfway between two values, relative to their spacing."""
    a = np.minimum(np.abs(q), 448.0)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -20))), -6.0)
    t = a / 2.0 ** (e - 3)
    return np.abs(t - np.floor(t) - 0.5)


def block_scales(x):
    n = x.size
    pad = np.zeros(-(-n // 64) * 64)
    pad[:n] = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = pad.reshape(-1, 64).max(1)
    tiny = ~(amax * (3.4e38 / 448) > 1)          # 448 / amax is not an fp32 number
    return np.where(tiny, 1.0, amax / 448), tiny


def adamw(p, g, m, v, *, lr, b1, b2, eps, t, wd, scale=1.0):
    """fp64 step: (p, m, v) and bounds of their fp32 errors."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * scale
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    mh, den = m1 / (1 - b1 ** t), np.sqrt(v1 / (1 - b2 ** t)) + eps
    d = lr * (wd * p + mh / den)
    em = 5 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    ev = 8 * U * v1                                # sums of positive terms; m, v of the state count as exact
    ep = 2 * U * np.abs(p) + 20 * U * (np.abs(lr * wd * p) + np.abs(lr * mh / den)) + np.abs(lr) * em / (1 - b1 ** t) / den
    return p - d, m1, v1, ep, em, ev
