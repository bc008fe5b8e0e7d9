"""One workspace, made for the largest batch, through calls of every smaller one: the same bits as with one of their own."""
import pytest
import torch

import paper_2503_05130_amd as ie
from tests.gpu_util import DEV, sync

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _answers(x, tokens, n, ws):
    rows = len(x)
    lp, h, top = (torch.full(s, 7.0, device=DEV) for s in ((rows,), (rows,), (rows, n)))
    ids = torch.full((rows, n), 7, dtype=torch.int32, device=DEV)
    ie.token_logprobs(x, tokens, lp, ws, entropy=h, top_ids=ids, top_logprobs=top)
    return lp, h, ids, top


@pytest.mark.parametrize("dtype", [BF, F32])
def test_log_probabilities(dtype):
    vocab, n = 20001, 5
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1300, vocab, generator=g, device=DEV).to(dtype)
    tokens = torch.randint(vocab, (1300,), generator=g, device=DEV)
    ws = ie.token_logprobs_workspace(1300, vocab, n)
    for rows in (1300, 1025, 1024, 683, 682, 48, 1):
        got = _answers(x[:rows], tokens[:rows], n, ws)
        want = _answers(x[:rows], tokens[:rows], n, torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device=DEV))
        sync()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), rows
        top = torch.topk(x[:rows].float(), n, dim=1).values
        assert torch.equal(x[:rows].gather(1, got[2].long()).float(), top)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("keys", [1024, 2048])
def test_paged_attention(mx4, keys):
    heads, kv, dim, page, batch = 16, 4, 64, 32, 70
    g = torch.Generator(device=DEV).manual_seed(2)
    pages = 150
    c = ie.PagedCache.empty(pages, page, kv, dim, mx4=mx4)
    c.append(*(torch.randn(pages * page, kv, dim, generator=g, device=DEV).to(BF) for _ in range(2)), torch.arange(pages * page, device=DEV))
    q = torch.randn(batch, heads, dim, generator=g, device=DEV).to(BF)
    table = torch.randint(pages, (batch, keys // page), generator=g, device=DEV).int()
    lens = torch.randint(keys // 2, keys + 1, (batch,), generator=g, device=DEV).int()
    ws = c.workspace(batch, heads, keys // page)
    for b in (70, 64, 33, 32, 16, 5, 1):
        out = torch.full((2, b, heads, dim), 7.0, dtype=BF, device=DEV)
        for i, space in enumerate((ws, torch.full((1 << 23,), 0xFF, dtype=torch.uint8, device=DEV))):
            c.attention(q[:b], table[:b], lens[:b], out[i], space)
        sync()
        assert torch.equal(out[0], out[1]) and not (out[0] == 7.0).any()
