"""Plain 64-bit implementations of the paged cache's operators and of the 4-bit product, on the CPU, for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch


def to_pages(x: torch.Tensor, kind: str, piece: int) -> torch.Tensor:
    """[pages, place, head, column] -> the cache's K ("k": pieces of `piece` columns) or V ("v") layout."""
    p, page, h, d = x.shape
    if kind == "k":
        return x.reshape(p, page, h, d // piece, piece).permute(0, 2, 3, 1, 4).contiguous()
    return x.reshape(p, page // 4, 4, h, d).permute(0, 3, 1, 4, 2).contiguous()


def from_pages(x: torch.Tensor, kind: str) -> torch.Tensor:
    """The inverse of to_pages."""
    if kind == "k":
        p, h, n, page, piece = x.shape
        return x.permute(0, 3, 1, 2, 4).reshape(p, page, h, n * piece)
    p, h, q, d, _ = x.shape
    return x.permute(0, 2, 4, 1, 3).reshape(p, 4 * q, h, d)


def attention(q, k, v, table, lens, scale):
    """q [B, H, d], k and v [pages, place, kv head, d], all fp64 numpy; pages outside the pool drop their tokens.
    Returns the context and a bound on each element's magnitude sum_j p_j |v_j| and the rows' largest sum_i |q_i k_i|."""
    batch, heads, d = q.shape
    pages, page, kv, _ = k.shape
    out, mag, dots = np.zeros_like(q), np.zeros_like(q), np.zeros((batch, heads, 1))
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
            p = np.exp(s - s.max())
            p /= p.sum()
            out[b, h] = p @ vv[:, g]
            mag[b, h] = p @ np.abs(vv[:, g])
            dots[b, h] = (np.abs(kk[:, g]) @ np.abs(q[b, h])).max()
    return out, mag, dots


def attention_tolerance(ref, mag, dots, n, d, scale):
    """Half a bf16 step (2^-8 of the value) for the result, and on sum p |v|: the probabilities' rounding to a bf16
    and its bf16 rest (2^-16), exp2 and the rescalings (2^-20), the score's fp32 sum of d terms and its scaling
    (each p changes by the score's error, and so does their sum), and the fp32 sums over the n keys."""
    score = (d + 2) * 2.0 ** -24 * dots * abs(scale)
    return 2.0 ** -8 * np.abs(ref) + 2 * (2.0 ** -16 + 2.0 ** -20 + score + (n + 64) * 2.0 ** -24) * mag


def plan(page, lens, new, table, ring, counters, room):
    """The planning call, one request after the other; returns the outputs by name."""
    table, ring_out, size = table.copy(), ring.copy(), len(ring)
    cap = table.shape[1] * page
    head, tail = int(counters[0]), int(counters[1])
    sane = head >= 0 and 0 <= tail - head <= size
    avail, space = (tail - head, size - (tail - head)) if sane else (0, 0)
    slots, starts = np.full(room, -1, np.int64), np.zeros(len(lens) + 1, np.int32)
    lens_out = lens.copy()
    tokens = wanted = back = taken = given = refused = 0
    for b, (o, n) in enumerate(zip(lens.tolist(), new.tolist())):
        starts[b] = min(tokens, room)
        if not (0 <= o <= cap and 0 <= n <= cap):
            refused += 1
            continue
        held, want = -(-o // page), -(-n // page)
        more, need, give = max(0, n - o), max(0, want - held), max(0, held - want)
        first = tokens
        tokens, wanted, back = tokens + more, wanted + need, back + give
        if (need and wanted > avail) or (more and tokens > room) or (give and back > space):
            refused += 1
            continue
        for j in range(need):
            table[b, held + j] = ring[(head + taken + j) % size]
        for j in range(give):
            ring_out[(tail + given + j) % size] = table[b, want + j]
        taken, given = taken + need, given + give
        for i in range(more):
            pos = o + i
            e = int(table[b, pos // page])
            slots[first + i] = e * page + pos % page if 0 <= e < size else -1
        lens_out[b] = n
    starts[-1] = min(tokens, room)
    return dict(table=table, ring=ring_out, counters_out=np.array([head + taken, tail + given], np.int64),
                lens_out=lens_out, slots=slots, starts=starts, refused=np.array([refused], np.int32))


def gelu(x):
    return 0.5 * x * (1.0 + np.vectorize(math.erf)(x / math.sqrt(2.0)))


def q4_weight(codes, scales, zeros):
    """fp64 [N, K] of the 4-bit form (numpy codes [N, K / 2], scales fp64 [N, G], zeros [N, G] or None)."""
    n, half = codes.shape
    c = np.stack([codes & 15, codes >> 4], -1).reshape(n, scales.shape[1], -1).astype(np.float64)
    z = 8.0 if zeros is None else zeros[..., None].astype(np.float64)
    return ((c - z) * scales[..., None]).reshape(n, 2 * half)
