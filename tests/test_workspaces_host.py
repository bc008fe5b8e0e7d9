"""A workspace that is made for the largest batch serves every smaller one (no GPU needed)."""
import ctypes

import pytest

import paper_2503_05130_amd as ie

ROWS = [1, 2, 3, 7, 31, 32, 33, 48, 64, 65, 100, 127, 128, 200, 256, 300, 512, 600, 682, 683, 1000, 1024, 1025, 2000, 2048, 2049, 4096,
        5000]


def _logprobs_bytes(rows, vocab, n):
    b = ctypes.c_size_t()
    assert ie.lib().iefwd_token_logprobs_workspace(rows, vocab, n, ctypes.byref(b)) == ie.OK
    return b.value


@pytest.mark.parametrize("vocab", [100, 8192, 8193, 20001, 50000, 131072, 600000, 1 << 24])
@pytest.mark.parametrize("n", [0, 5, 32])
def test_log_probabilities(vocab, n):
    need = {r: _logprobs_bytes(r, vocab, n) for r in ROWS if r * vocab <= 1 << 35}
    for r in need:
        # the documented bound
        assert need[r] <= min(64 * r, 2048) * (12 + 8 * n)
        given = ie.token_logprobs_workspace(r, vocab, n, device="cpu").numel()
        assert given >= max(need[s] for s in need if s <= r)
        assert given <= min(64 * r, 2048) * (12 + 8 * n) and (given > 0) == (vocab > 8192)


@pytest.mark.parametrize("kind", [ie.KV_BF16, ie.KV_MX4])
@pytest.mark.parametrize("heads,kv,dim", [(32, 8, 128), (12, 12, 64), (16, 1, 128), (40, 2, 128), (64, 1, 64)])
@pytest.mark.parametrize("pages", [1, 40, 64, 65, 128, 300, 5000])
def test_paged_attention(kind, heads, kv, dim, pages):
    desc = ie.PagedCacheDesc(ie.ABI_VERSION, kind, 100, 16, kv, dim, 1 << 20, 1 << 20, None, None)
    cache = ie.PagedCache.__new__(ie.PagedCache)      # the sizes alone: making one takes memory on a GPU
    cache.desc, cache._ref, cache.device = desc, ctypes.byref(desc), "cpu"
    cache.n_kv_heads, cache.head_dim, cache.page_size = kv, dim, 16
    most = 0
    for batch in range(1, 520):
        b = ctypes.c_size_t()
        assert ie.lib().iefwd_paged_attention_workspace(cache._ref, batch, heads, pages, ctypes.byref(b)) == ie.OK
        most = max(most, b.value)
        assert cache.workspace(batch, heads, pages).numel() == most
