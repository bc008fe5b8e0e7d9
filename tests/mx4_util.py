"""Plain 64-bit forms of microscaled 4-bit matrices and of a cache in this form, on the CPU, for the tests."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def quantize(x):
    """codes uint8 [..., K'] and scale bytes uint8 [..., K' / 32] of fp64 rows, K' = the length rounded up to 32."""
    x = np.asarray(x, np.float64)
    k = -(-x.shape[-1] // 32) * 32
    padded = np.zeros((*x.shape[:-1], k))
    padded[..., :x.shape[-1]] = x
    b = padded.reshape(*x.shape[:-1], k // 32, 32)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(b).all(-1)
    safe = np.where(bad | (top == 0), 1.0, top)
    exponent = np.floor(np.log2(safe)).astype(int)
    exponent -= 2.0 ** exponent > safe          # log2 may round up to the next whole number
    e = np.where(top == 0, -127, np.maximum(exponent - 2, -127))
    y = np.where(bad[..., None], 0.0, b) / np.exp2(e.astype(float))[..., None]
    size = np.abs(y)
    # the nearest value, ties to the even code: the sum of the borders passed, a border itself passed where that leads to an even code
    codes = np.zeros(size.shape, np.uint8)
    for i, border in enumerate([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]):
        codes += (size >= border) if i % 2 else (size > border)
    codes += 8 * np.signbit(y).astype(np.uint8)
    codes[bad] = 0
    return codes.reshape(*x.shape[:-1], k), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales):
    """fp64 values of codes (one a byte) under scale bytes."""
    v = VALUES[codes].reshape(*codes.shape[:-1], -1, 32)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(float) - 127.0))
    return (v * s[..., None]).reshape(codes.shape)


def pairs(codes):
    """Two codes a byte, the first in the low half."""
    return codes[..., 0::2] | codes[..., 1::2] << 4


def packed(codes, scales, rows, cols):
    """The library's layout of a matrix, all bytes of it."""
    tiles, chunks = -(-rows // 16), -(-cols // 128)
    c = np.zeros((tiles * 16, chunks * 128), np.uint8)
    c[:rows, :codes.shape[1]] = codes
    s = np.zeros((tiles * 16, -(-chunks // 4) * 16), np.uint8)
    s[:rows, :scales.shape[1]] = scales
    c = pairs(c).reshape(tiles, 16, chunks, 4, 16).transpose(0, 2, 3, 1, 4).reshape(tiles, -1)
    s = s.reshape(tiles, 16, -1, 4, 4).transpose(0, 2, 4, 1, 3).reshape(tiles, -1)      # tile, group, block, row, chunk of the group
    return np.concatenate([c, s], 1).reshape(-1)


def k_pages(codes, scales):
    """The cache's bytes [pages, heads, 17, d / 32, page] of keys given as [pages, place, head, column]."""
    p, page, h, d = codes.shape
    c = pairs(codes).reshape(p, page, h, d // 32, 16).transpose(0, 2, 3, 1, 4).reshape(p, h, -1)
    s = scales.transpose(0, 2, 3, 1).reshape(p, h, -1)
    return np.ascontiguousarray(np.concatenate([c, s], -1).reshape(p, h, 17, d // 32, page))


def v_pages(codes, scales):
    """The cache's bytes [pages, heads, 17, page / 4, d / 8] of values given as [pages, place, head, column]."""
    p, page, h, d = codes.shape
    c = pairs(codes).reshape(p, page // 4, 4, h, d // 8, 4).transpose(0, 3, 1, 4, 2, 5).reshape(p, h, -1)
    s = scales.reshape(p, page // 4, 4, h, d // 32).transpose(0, 3, 1, 4, 2).reshape(p, h, -1)
    return np.ascontiguousarray(np.concatenate([c, s], -1).reshape(p, h, 17, page // 4, d // 8))


def scored_attention(q, k, v, table, lens, scale, cap=0.0, slopes=None, q_exact=True):
    """q [B, H, d], k and v [pages, place, kv head, d], fp64; pages outside the pool drop their tokens.  Returns the context, per
    element a bound sum_j p_j |v_j| and per row a bound on a score's error in fp32: its sum of d terms and scaling (each
    rounding 2^-23, rounded or cut), for a cache in 4 bits what splitting q leaves out (2^-21 of the largest of 32 columns, q_exact False),
    the tanh (2^-20 of the cap up to 64, beyond 2^-19 of its result) and the roundings of the scaled score, the slope's product and their sum."""
    batch, heads, d = q.shape
    pages, page, kv, _ = k.shape
    out, mag, err = np.zeros_like(q), np.zeros_like(q), np.zeros((batch, heads, 1))
    for b in range(batch):
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        pos = np.arange(n)
        ids = table[b][pos // page]
        keep = (ids >= 0) & (ids < pages)
        if not keep.any():
            continue
        kk, vv = (x[ids[keep], pos[keep] % page] for x in (k, v))
        for h in range(heads):
            g = h // (heads // kv)
            s = kk[:, g] @ q[b, h] * scale
            e = (d + 2) * 2.0 ** -23 * (np.abs(kk[:, g]) @ np.abs(q[b, h]) * abs(scale)).max()
            if not q_exact:
                top = np.abs(q[b, h]).reshape(-1, 32).max(1)
                e += 2.0 ** -21 * (np.abs(kk[:, g]).reshape(len(kk), -1, 32).sum(2) @ top * abs(scale)).max()
            if cap:
                s = cap * np.tanh(s / cap)
                e += 2.0 ** -20 * cap if cap <= 64 else 2.0 ** -19 * np.abs(s).max()
            if slopes is not None:
                bias = slopes[h] * (n - 1 - pos[keep])
                s = s - bias
                e += 2.0 ** -22 * np.abs(bias).max()
            err[b, h] = e + 2.0 ** -22 * np.abs(s).max()
            p = np.exp(s - s.max())
            p /= p.sum()
            out[b, h] = p @ vv[:, g]
            mag[b, h] = p @ np.abs(vv[:, g])
    return out, mag, err


def scored_tolerance(ref, mag, err, n):
    """Half a bf16 step of the result, and on sum p |v|: the probabilities' 16 bits, exp2 and the rescalings (2^-20), the
    score's error (each p and their sum change by it) and the fp32 sums over the keys."""
    return 2.0 ** -8 * np.abs(ref) + 2 * (2.0 ** -16 + 2.0 ** -20 + np.expm1(np.minimum(err, 1.0)) + (n + 64) * 2.0 ** -24) * mag


def product_tolerance(a, w, y, k, f32):
    """Exact terms, summed in fp32: 128 at a time (each addition off by at most 2^-23 of what it adds up, rounded or cut),
    then the chunks and the waves, the bias; the result's own rounding."""
    chunks = -(-k // 128)
    e = 2.0 ** -23 * (128 + chunks + 12) * (np.abs(a) @ np.abs(w).T) + 2.0 ** -22 * np.abs(y)
    return e if f32 else e + 2.0 ** -8 * np.abs(y)
