"""Float64 models of the operators round the cache: residual norms, 4-bit products, rotary rows, sampling.

Every model takes arrays of float64 that hold the inputs' exact values and returns the definition's value, with a bound
on how far an fp32 computation of it may be off before its output is rounded."""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
F32 = 2.0**-24          # half a step of fp32, relative
ROUND = {"bf16": 2.0**-8, "f32": 2.0**-24}


def norm(r, o, gain, post_gain=None, gate=None, scale=1.0, eps=1e-5):
    """(r', bound, y, bound).  A sum of squares is right to (terms in a chain + tree) F32 < 2^-18; the factors add a few."""
    mag = np.abs(r)
    new = r
    if o is not None:
        p = o
        if post_gain is not None:
            p = p / np.sqrt((p * p).mean(-1, keepdims=True) + eps) * post_gain
        if gate is not None:
            p = p * gate
        new = r + scale * p
        mag = mag + np.abs(scale * p)
    inv = 1 / np.sqrt((new * new).mean(-1, keepdims=True) + eps)
    y = new * inv * gain
    return new, 2.0**-18 * mag, y, 2.0**-17 * mag * inv * np.abs(gain)


def weights(codes, scales):
    """Values of codes uint8 [n][k/2] and scale bytes [n][k/32] (bytes up to 252)."""
    n, half = codes.shape
    c = np.stack([codes & 15, codes >> 4], -1).reshape(n, 2 * half)
    return np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7] * np.exp2(scales.astype(np.float64) - 127).repeat(32, 1)


def silu(x):
    with np.errstate(over="ignore"):
        return x / (1 + np.exp(-x))


def product(a, w, gated=False):
    """(out, bound).  A product takes part in at most k/32 sums of one chain and 40 more where chains are joined, each
    off by at most 2 F32 of the sum of magnitudes."""
    k = w.shape[1]
    out = a @ w.T
    bound = (k / 32 + 40) * 2 * F32 * (np.abs(a) @ np.abs(w).T)
    if gated:
        f = w.shape[0] // 2
        g, u, dg, du = out[:, :f], out[:, f:], bound[:, :f], bound[:, f:]
        out = silu(g) * u                                     # |silu'| <= 1.1
        bound = 1.1 * dg * (np.abs(u) + du) + np.abs(silu(g)) * du + 8 * F32 * np.abs(out)
    return out, bound


def frequencies(rot, theta, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=8192):
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        h = np.clip((original_len * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = f * ((1 - h) / factor + h)
    return f


def rotate(x, pos, freq, interleaved=False, mscale=1.0):
    """(rows, bound): x [rows][heads][hd].  cos and sin are right to 2^-21."""
    rot = 2 * len(freq)
    ang = np.asarray(pos, np.float64)[:, None, None] * freq
    c, s = mscale * np.cos(ang), mscale * np.sin(ang)
    y, bound = x.copy(), np.zeros_like(x)
    i = np.arange(rot // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y[..., p] = x[..., p] * c - x[..., q] * s
    y[..., q] = x[..., q] * c + x[..., p] * s
    bound[..., p] = bound[..., q] = 2.0**-20 * abs(mscale) * (np.abs(x[..., p]) + np.abs(x[..., q]))
    return y, bound


def sample(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, logprob) of one row of logits."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    best = int(np.argmax(x))
    if x[best] == -np.inf:
        return -1, -math.inf
    if not temperature > 0:
        return best, 0.0
    ids = np.lexsort((np.arange(len(x)), -x))
    if 0 < top_k < len(x):
        ids = ids[:top_k]
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(x[ids] == x[best], 0.0, x[ids] - x[best])
        w = np.where(np.isneginf(z), 0.0, np.exp(z / temperature))
    if top_p < 1:
        before = np.cumsum(w) - w
        n = max(1, int((before < max(top_p, 0.0) * w.sum()).sum()))
        ids, w = ids[:n], w[:n]
    low = min(min_p, 1.0) if min_p > 0 else 0.0
    ids, w = ids[w >= low], w[w >= low]
    order = np.argsort(ids)
    ids, w = ids[order], w[order]
    u = min(max(u, 0.0), 1 - 2.0**-53) if u == u else 0.0
    run = np.cumsum(w)
    j = int((run <= u * run[-1]).sum())
    if j >= len(ids):
        j = int(np.nonzero(w)[0][-1])
    return int(ids[j]), math.log(w[j] / run[-1])
