"""Plain 64-bit reference of the paged key/value cache and its attention (torch on the CPU)."""

from __future__ import annotations

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # unit roundoff
HELD = {torch.bfloat16: 1.875 * 2.0 ** 127, torch.float16: 61440.0}


def e4m3_values():
    """The 256 codes' values, from the format: 4 exponent bits (bias 7), 3 fraction bits."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    v[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -v, v)


def quantise(x, dtype):
    """(values held, exponent byte) of rows x [..., d] of dtype in an e4m3 cache."""
    x = x.double().numpy()
    fin = np.isfinite(x)
    y = np.clip(np.where(fin, x, 0.0), -HELD[dtype], HELD[dtype])
    amax = np.abs(y).max(-1)
    k = np.zeros(amax.shape, np.int64) - 9
    for i, a in np.ndenumerate(amax):
        if a > 0:
            k[i] = -200
            while a > 448.0 * 2.0 ** float(k[i]):
                k[i] += 1
    k = np.clip(k, -100, 120)
    scale = 2.0 ** k.astype(np.float64)[..., None]
    z = np.abs(y) / scale
    step = 2.0 ** (np.floor(np.log2(np.maximum(z, 2.0 ** -6))) - 3)
    held = np.copysign(np.rint(z / step) * step, y) * scale   # rint: ties to even
    held[~fin] = np.nan
    return torch.from_numpy(held), torch.from_numpy((k + 127).astype(np.uint8))


def sees(n, ctx, window=0, sinks=0):
    """[n, ctx] which keys each of the last n tokens sees."""
    p = torch.arange(ctx - n, ctx)[:, None]
    j = torch.arange(ctx)[None]
    m = j <= p
    if window:
        m &= (j > p - window) | (j < sinks)
    return m


def attend(q, k, v, mask, scale):
    """One sequence: q [n, hq, d], k, v [ctx, hkv, d] (64 bits), mask [n, ctx].  Returns out,
    lse, and per value sum_j w_j |v_j| and per row max_j sum |q_i k_ij|, from which bounds follow.  Keys
    outside a row's mask have no part in it."""
    n, hq, d = q.shape
    G = hq // k.shape[1]
    out = torch.zeros(n, hq, d, dtype=torch.float64)
    mag = torch.zeros(n, hq, d, dtype=torch.float64)
    lse = torch.full((n, hq), -np.inf, dtype=torch.float64)
    big = torch.zeros(n, hq, dtype=torch.float64)
    for r in range(n):
        j = mask[r].nonzero()[:, 0]
        if not len(j):
            continue
        for h in range(hq):
            kk, vv = k[j, h // G], v[j, h // G]
            s = (kk @ q[r, h]) * scale
            w = torch.softmax(s, 0)
            out[r, h] = w @ vv
            mag[r, h] = w @ vv.abs()
            lse[r, h] = torch.logsumexp(s, 0)
            big[r, h] = (kk.abs() @ q[r, h].abs()).max() * scale
    return out, lse, mag, big


def attend_fast(q, k, v, mask, scale):
    """attend() with the rows at once, for finite inputs."""
    n, hq, d = q.shape
    G = hq // k.shape[1]
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    lse, big = torch.full_like(q[..., 0], -np.inf), torch.zeros_like(q[..., 0])
    some = mask.any(1)
    for h in range(hq):
        kk, vv = k[:, h // G], v[:, h // G]
        s = (q[:, h] @ kk.T) * scale
        s[~mask] = -np.inf
        z = torch.logsumexp(s, 1)
        w = torch.exp(s - torch.where(some, z, torch.zeros_like(z))[:, None])
        out[:, h], mag[:, h], lse[:, h] = w @ vv, w @ vv.abs(), z
        big[:, h] = (q[:, h].abs() @ kk.abs().T).amax(1) * scale
    return out, lse, mag, big


def bounds(dtype, mag, big, lse, d, keys, vmax):
    """How far out and lse may be off.  Scores are sums of d products in 32 bits: an error of
    (d + 2) 2^-24 of the sum of magnitudes, and as much relative error of the exponential
    (and twice 2^-21 for exp2 and its argument).  Exponentials are rounded to dtype: u; below
    its normal range (f16) by at most 2^-25 each.  The result is rounded to dtype: u."""
    u = U[dtype]
    ds = (d + 2) * 2.0 ** -24 * big
    rel = 2 * u + 2 * torch.expm1(ds) + 2.0 ** -18
    tiny = keys * 2.0 ** -25 * vmax + 2.0 ** -24 if dtype == torch.float16 else 1e-37
    return rel[..., None] * mag * 1.01 + tiny, ds + 2.0 ** -20 * (1 + lse.abs())
