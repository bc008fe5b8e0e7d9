"""Slopes of every size and sign in the paged attention, over few keys and over a million, against a plain 64-bit form."""
import pytest
import torch

import paper_2503_05130_amd as ie
from tests.gpu_util import DEV, sync

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
SLOPES = [-1.0, -0.01, 0.3, 0.0, 3e38, -3e38, 1e30, -1e30, 2.4e38, -2.0 ** -20, 1e-40, -7.0]
PAGE, POOL = 256, 64


def _plain(q, k, v, slope, cap, mx4):
    """One head in fp64: the context, and what it may be off by: half a bf16 step of it, and what its probabilities p are off by, on p |v|
    and in their sum on the whole: their 16 bits, exp2 and the rescalings (2^-16 + 2^-20), and the error of their score.  That is
    its d terms and scaling (2^-23 each), what splitting q for 4-bit keys leaves out (2^-21 of the largest of 32 columns), the tanh (2^-20
    of the cap) and the roundings of the score, the product with the slope and the difference from the largest.  The slope counts from
    the end that it favours: the scores from the other end differ by the same for all keys.  In the fp32 sums a term changes a sum by at
    most 2^-23 of it or itself."""
    key = torch.arange(len(k), device=DEV)
    low = abs(slope) * (key if slope < 0 else len(k) - 1 - key).double()
    keep = low <= 1000.0      # beyond, p is 0: q . k / sqrt(d) is far below 100
    k, v, low = k[keep], v[keep], low[keep]
    n, d = k.shape
    s = k @ q * d ** -0.5
    e = (d + 2) * 2.0 ** -23 * (k.abs() @ q.abs()) * d ** -0.5
    if mx4:
        e += 2.0 ** -21 * (k.abs().view(n, -1, 32).sum(2) @ q.abs().view(-1, 32).amax(1)) * d ** -0.5
    if cap:
        s = cap * torch.tanh(s / cap)
        e += 2.0 ** -20 * cap
    t = s - low
    t = t - t.max()
    p = torch.exp(t)
    p /= p.sum()
    e = torch.where(p > 0, e + 2.0 ** -22 * (s.abs() + low - t), 0.0)
    off = p * (2.0 ** -16 + 2.0 ** -20 + torch.expm1(e))
    sums = 2.0 ** -23 * (float((p > 2.0 ** -60).sum()) + 64) + 2.0 ** -60 * n
    ctx, mag = p @ v, p @ v.abs()
    return ctx, 2.0 ** -8 * ctx.abs() + off @ v.abs() + (off.sum() + 2 * sums) * mag


@pytest.mark.parametrize("n", [1, 300, 5000, (1 << 20) + 5])
@pytest.mark.parametrize("kind", ["mx4", "bf16", "e4m3"])
@pytest.mark.parametrize("heads,dim,cap", [(12, 64, 0.0), (4, 128, 30.0), (8, 64, 0.0)])
def test_slopes_of_every_size_and_sign(kind, n, heads, dim, cap):
    g = torch.Generator().manual_seed(n + heads)
    scales = [torch.tensor([s], device=DEV) for s in (0.02, 0.03)] if kind == "e4m3" else [None, None]
    c = ie.PagedCache.empty(POOL, PAGE, 1, dim, *scales, mx4=kind == "mx4")
    rows = [torch.randn(POOL * PAGE, 1, dim, generator=g).to(BF).to(DEV) for _ in range(2)]
    c.append(*rows, torch.arange(POOL * PAGE, device=DEV))
    cols = -(-n // PAGE)
    table = torch.randint(POOL, (1, cols), generator=g, dtype=torch.int32).to(DEV)      # pages may come again
    q = torch.randn(1, heads, dim, generator=g).to(BF).to(DEV)
    slopes = torch.tensor(SLOPES[-heads:], device=DEV)
    out = torch.empty(1, heads, dim, dtype=BF, device=DEV)
    c.attention(q, table, torch.tensor([n], dtype=torch.int32, device=DEV), out, c.workspace(1, heads, cols), cap=cap, slopes=slopes)
    pos = torch.arange(n, device=DEV)
    slots = table[0, pos // PAGE].long() * PAGE + pos % PAGE
    if kind == "e4m3":      # the values themselves: reading back rounds them to bf16
        kk, vv = ((r / s).clamp(-448, 448).to(torch.float8_e4m3fn).double() * s.double() for r, s in zip([x.float() for x in rows], scales))
    else:
        kk, vv = (torch.empty_like(r) for r in rows)
        c.read(torch.arange(POOL * PAGE, device=DEV), kk, vv)
    sync()
    k, v = (x[slots, 0].double() for x in (kk, vv))
    for h in range(heads):
        ctx, tol = _plain(q[0, h].double(), k, v, float(slopes[h]), cap, kind == "mx4")
        off = (out[0, h].double() - ctx).abs()
        assert (off <= tol).all(), (SLOPES[-heads:][h], float((off / tol).max()), out[0, h, :4], ctx[:4])


def test_huge_slopes_where_the_newest_key_is_gone():
    """A page outside the pool drops its keys: the nearest of the others takes all, as under any other large slope."""
    c = ie.PagedCache.empty(4, 16, 1, 64, mx4=False)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(64, 1, 64, generator=g).to(BF).to(DEV) for _ in range(2))
    c.append(k, v, torch.arange(64, device=DEV))
    q = torch.randn(1, 2, 64, generator=g).to(BF).to(DEV)
    out = torch.empty_like(q)
    table = torch.tensor([[-1, 1, 2, -1]], dtype=torch.int32, device=DEV)
    c.attention(q, table, torch.tensor([60], dtype=torch.int32, device=DEV), out, c.workspace(1, 2, 4),
                slopes=torch.tensor([3e38, -3e38], device=DEV))
    sync()
    assert torch.equal(out[0, 0], v[47, 0]) and torch.equal(out[0, 1], v[16, 0])
