"""Every variant of the paged attention kernels: workgroups of 8, 4 and 2 waves (by batch x key-value heads x tiles of 16 heads),
heads a key-value head, plain and changed scores, pages read as usual and past the last cache (by the table's width and the
pool's size), against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import mx4_util as X
from tests.gpu_util import DEV, f64
from tests.test_gpu_paged_mx4 import _attend, _case

pytestmark = pytest.mark.gpu

STREAM = 96 << 20      # bytes of pages from which they are read past the last cache


def _lengths(batch):
    """Mostly short requests, one of several parts, one of two, one without keys."""
    lens = [(i * 37) % 61 for i in range(batch)]
    lens[1], lens[batch // 2], lens[-1] = 2600, 700, 1100
    return lens


def _widened(ops):
    """The same pages at the front of a pool, and the table at the left of one, that count as a cache of more than STREAM bytes."""
    c, table = ops["cache"], ops["table"]
    per_page = 2 * c.k[0].numel() * c.k.element_size()
    pages = max(-(-STREAM // per_page), len(c.k))
    bytes_of = [torch.full((pages, *x.shape[1:]), 255, dtype=torch.uint8, device=DEV) if x.element_size() == 1 else
                torch.full((pages, *x.shape[1:]), float("nan"), dtype=x.dtype, device=DEV) for x in (c.k, c.v)]
    k, v = (new.view(old.dtype) for new, old in zip(bytes_of, (c.k, c.v)))
    for new, old in ((k, c.k), (v, c.v)):
        new.view(torch.uint8)[:len(old)] = old.view(torch.uint8)
    scales = [] if c.k_scale is None else [c.k_scale, c.v_scale]
    wide = torch.full((len(table), max(-(-pages // len(table)), table.shape[1])), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    assert min(pages, wide.numel()) * per_page >= STREAM
    return dict(ops, cache=ie.PagedCache(k, v, *scales), table=wide)


def _all_forms(kind, batch, heads, kv, dim):
    lens = _lengths(batch)
    ops, (q, k, v, table, _) = _case(kind, batch, heads, kv, dim, 32, lens, batch + heads + dim)
    slopes = 0.3 * 2.0 ** -torch.linspace(0, 8, heads)
    for cap, low in ((0.0, None), (20.0, slopes)):
        ref, mag, err = X.scored_attention(q, k, v, table, lens, dim ** -0.5, cap, None if low is None else f64(low), kind != "mx4")
        tol = X.scored_tolerance(ref, mag, err, max(lens))
        for stream in (False, True):
            given = dict(_widened(ops) if stream else ops)
            given["out"] = torch.full_like(ops["out"], 5.0)
            got = f64(_attend(given, cap=cap, slopes=None if low is None else low.to(DEV)))
            bad = np.abs(got - ref) > tol
            assert not bad.any(), (cap, stream, np.argwhere(bad)[:5], (np.abs(got - ref) / tol).max())


@pytest.mark.parametrize("rows", [40, 260, 2060])      # 8, 4 and 2 waves
@pytest.mark.parametrize("heads,kv", [(16, 4), (28, 4), (32, 2), (40, 2)])      # 4, 7, 16 and 20 heads a key-value head
@pytest.mark.parametrize("dim", [64, 128])
def test_cache_in_4_bits(rows, heads, kv, dim):
    tiles = -(-(heads // kv) // 16)
    _all_forms("mx4", -(-rows // (kv * tiles)), heads, kv, dim)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [40, 4100])           # 8 and 2 waves
@pytest.mark.parametrize("dim", [64, 128])
def test_cache_in_16_and_8_bits(kind, rows, dim):
    _all_forms(kind, rows // 4, 12, 4, dim)
