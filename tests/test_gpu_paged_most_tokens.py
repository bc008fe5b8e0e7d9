"""Append to a cache in 4 bits and reading back, with as many tokens as the calls take (2^28 a call and head)."""
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import mx4_util as X
from tests.gpu_util import DEV, f64, sync

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def test_most_tokens():
    """All but a few tokens are outside the pool: skipped, and read as zeros.  68.7 GB of rows, for keys and values alike."""
    tokens, dim, page = 1 << 28, 128, 16
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GiB of GPU memory")
    c = ie.PagedCache.empty(2, page, 1, dim, mx4=True)
    rows = torch.empty(tokens, 1, dim, dtype=BF, device=DEV)
    at = torch.tensor([0, 1, 15, 16, (1 << 27) - 1, 1 << 27, (1 << 27) + 1, tokens - 17, tokens - 1], device=DEV)
    x = torch.randn(len(at), 1, dim, generator=torch.Generator().manual_seed(1)).to(BF)
    rows[at] = x.to(DEV)
    slots = torch.full((tokens,), -1, device=DEV)
    slots[at] = torch.arange(len(at), device=DEV) * 3
    c.append(rows, rows, slots)
    sync()
    rows.fill_(7.0)
    c.read(slots, rows, rows)      # keys and values are equal
    sync()
    want = X.values(*X.quantize(f64(x)))
    assert (f64(rows[at]) == want).all()
    rows[at] = 0
    assert not any(bool(p.view(torch.int64).any()) for p in rows.view(-1).split(1 << 30))
    del rows, slots
    torch.cuda.empty_cache()
