"""Infinite elements of the cache's values: what the definition gives, in every column and row that they reach and no other."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import paged_util as P
from tests.gpu_util import DEV, f64, sync

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,heads,kv", [(64, 4, 2), (128, 20, 1)])
@pytest.mark.parametrize("lens", [[1], [33, 300, 0], [3000, 513, 40]])
def test_infinite_values(lens, dim, heads, kv):
    page, batch, scale = 16, len(lens), 0.1
    g = torch.Generator().manual_seed(dim + max(lens))
    held = [-(-n // page) for n in lens]
    pages = sum(held) + 1
    c = ie.PagedCache.empty(pages, page, kv, dim)
    k, v = (torch.randn(pages, page, kv, dim, generator=g).bfloat16() for _ in range(2))
    table = torch.zeros(batch, max(held), dtype=torch.int32)
    order = torch.randperm(pages, generator=g).int()
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    touched = torch.zeros(batch, kv, dim, dtype=torch.bool)
    for b, n in enumerate(lens):
        for head in range(kv) if n else ():
            # a key of every kind of place: the first, the last, one in the middle; +inf, -inf, both signs (NaN)
            for j, (key, x) in enumerate([(0, "inf"), (n - 1, "-inf"), (n // 2, "inf"), (n // 3, "-inf")]):
                v[table[b, key // page], key % page, head, 5 * j + head] = float(x)
                touched[b, head, 5 * j + head] = True
            for key, x in ((0, "inf"), (n - 1, "-inf")):
                if n > 1:
                    v[table[b, key // page], key % page, head, 50] = float(x)
                    touched[b, head, 50] = True
    q = torch.randn(batch, heads, dim, generator=g).bfloat16()
    c.k.copy_(P.to_pages(k, "k", 8).to(DEV))
    c.v.copy_(P.to_pages(v, "v", 8).to(DEV))
    out = torch.empty(batch, heads, dim, dtype=torch.bfloat16, device=DEV)
    c.attention(q.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out,
                c.workspace(batch, heads, table.shape[1]), scale)
    sync()
    with np.errstate(invalid="ignore"):
        ref, _, _ = P.attention(f64(q), f64(k), f64(v), table.numpy(), np.array(lens), scale)
    got = f64(out)
    special = touched.repeat_interleave(heads // kv, 1).numpy()
    assert (np.isfinite(ref) == ~special).all()
    assert np.array_equal(got[special], ref[special], equal_nan=True)
    # and the columns beside them as if there were none
    clean = torch.where(torch.isfinite(v.float()), v.float(), torch.zeros(())).bfloat16()
    want, mag, dots = P.attention(f64(q), f64(k), f64(clean), table.numpy(), np.array(lens), scale)
    tol = P.attention_tolerance(want, mag, dots, max(lens), dim, scale)
    assert (np.abs(got - want)[~special] <= tol[~special]).all()
