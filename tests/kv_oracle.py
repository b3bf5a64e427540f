"""Float64 model of the paged KV cache in 8 bits and of windowed attention over it, for the tests.

Pages are held plainly, [blocks][heads][16][hd], as code values (8 bits) or
values (bf16); the pools' layouts are converted here with tensor indexing.
"""
from __future__ import annotations

import numpy as np
import torch

MIN_EXP, MAX_EXP = -100, 120


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """float64 of magnitude <= 464 to the nearest e4m3 value, ties to even (steps 2^(exponent - 3), at least 2^-9)."""
    step = np.exp2(np.maximum(np.frexp(x)[1] - 4, -9).astype(np.float64))
    return np.rint(x / step) * step


def block_exponent(x: np.ndarray) -> int:
    """max(-100, least e with |x| <= 448 2^e over the finite values)."""
    fin = np.abs(x[np.isfinite(x)])
    top = fin.max() if fin.size else 0.0
    e = MIN_EXP
    while top > 448 * 2.0 ** e:
        e += 1
    return e


def append_block(codes, e_old: int, t0: int, rows: np.ndarray):
    """Append rows [n][hd] from token t0 on to codes [16][hd] (values of the codes); returns the block's exponent."""
    e = block_exponent(rows)
    if t0 > 0:
        e = max(e, e_old)
        if e > e_old:
            codes[:t0] = round_e4m3(codes[:t0] * 2.0 ** (e_old - e))
    lim = 240.0 if e >= MAX_EXP else 448.0
    with np.errstate(invalid="ignore"):
        new = round_e4m3(np.clip(np.where(np.isfinite(rows), rows, 0.0) * 2.0 ** -e, -lim, lim))
    codes[t0:t0 + len(rows)] = np.where(np.isfinite(rows), new, np.nan)
    return e


def pages(pool: torch.Tensor, is_k: bool) -> np.ndarray:
    """A layer's pool as float64 [blocks][heads][16][hd]: K pages are slabs of dims, V pages dim-major."""
    x = pool.float().cpu()
    x = x.transpose(2, 3) if not is_k else x.permute(0, 1, 3, 2, 4).reshape(x.shape[0], x.shape[1], 16, -1)
    return x.double().numpy().copy()


def visible(pos: int, n_keys: int, window: int, sinks: int) -> np.ndarray:
    t = np.arange(n_keys)
    ok = t <= pos
    if window > 0:
        ok &= (t > pos - window) | (t < sinks)
    return ok


def attend(q, k, v, pos, window, sinks):
    """q [rows][hq][hd] at positions pos, k, v [keys][hkv][hd], float64: (out, bound), the outputs and how far a
    correct result may be off.

    The bound, per output: P is rounded to bf16 (half a step: 2^-8 of it) in the sum of p v and, where the row sum
    adds the same rounded P, in the normaliser; each score is a sum of hd products in fp32, off by at most
    hd 2^-24 sum|q k| (scaled), which moves p by that ratio, twice (numerator and normaliser), with the exponential's
    own few 2^-22; the sums of p v over n keys in fp32 add (n / 16 + 16) 2^-24 of sum p |v| (a matrix instruction sums
    up to 32 products, partial sums are joined); the result is rounded to bf16 (half a step)."""
    rows, hq, hd = q.shape
    hkv = k.shape[1]
    out = np.zeros_like(q)
    bound = np.zeros_like(q)
    for r in range(rows):
        ok = visible(int(pos[r]), len(k), window, sinks)
        for h in range(hq):
            kk, vv = k[ok, h * hkv // hq], v[ok, h * hkv // hq]
            with np.errstate(invalid="ignore", over="ignore"):
                s = kk @ q[r, h] / np.sqrt(hd)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[r, h] = p @ vv
                spread = float((np.abs(kk) @ np.abs(q[r, h])).max()) / np.sqrt(hd)
                rel = 2 * 2.0 ** -8 + 2 * (hd * 2.0 ** -24 * spread + 2.0 ** -20) + (ok.sum() / 16 + 16) * 2.0 ** -24
                bound[r, h] = rel * (p @ np.abs(vv)) + 2.0 ** -8 * np.abs(out[r, h]) + 1e-30
    return out, bound


def check_rows(got, want, bound, what=""):
    """Outputs within the bound; infinities and NaN where the definition has them."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN at other places"
    assert np.array_equal(got[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)]), f"{what}: infinities"
    fin = ~odd
    off = np.abs(got[fin] - want[fin])
    worst = float(np.max(off / bound[fin])) if off.size else 0.0
    assert worst <= 1.0, f"{what}: off by {worst:.3f} of the bound"
    return worst
