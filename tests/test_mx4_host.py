"""What the entry points of microscaled 4-bit matrices refuse before any device work, and their sizes (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_2503_05130_amd as ie
from tests import mx4_util as X

P = 1 << 20          # stands for an aligned device address; nothing here reads it


def _bytes(rows, k):
    n = ctypes.c_size_t(7)
    status = ie.lib().iefwd_mx4_bytes(rows, k, ctypes.byref(n))
    return status, n.value


@pytest.mark.parametrize("rows,k", [(1, 1), (16, 128), (17, 129), (100, 512), (3, 513), (1 << 24, 4096), (1 << 16, 1 << 20)])
def test_bytes(rows, k):
    tiles, chunks = -(-rows // 16), -(-k // 128)
    assert _bytes(rows, k) == (ie.OK, tiles * (chunks * 1024 + -(-chunks // 4) * 256))


@pytest.mark.parametrize("rows,k", [(0, 5), (5, 0), ((1 << 24) + 1, 1), (1, (1 << 20) + 1), (1 << 17, 1 << 20)])
def test_bad_sizes_are_refused(rows, k):
    assert _bytes(rows, k) == (ie.EINVAL, 7)
    lib = ie.lib()
    assert lib.iefwd_mx4_quantize(ie.BF16, P, 1 << 21, P, rows, k, None) == ie.EINVAL and ie.last_error()
    assert lib.iefwd_mx4_values(P, ie.BF16, P, 1 << 21, rows, k, None) == ie.EINVAL
    assert lib.iefwd_mx4_pack(P, P, P, rows, k, None) == ie.EINVAL
    assert lib.iefwd_mx4_gemm(0, P, P, None, None, P, 1, rows, k, None) == ie.EINVAL
    assert lib.iefwd_mx4_gemm(0, P, P, None, None, P, rows, 1, k, None) == ie.EINVAL


def test_null_bytes():
    assert ie.lib().iefwd_mx4_bytes(1, 1, None) == ie.EINVAL


@pytest.mark.parametrize("bad", [dict(kind=2), dict(x=None), dict(x=P + 1), dict(kind=1, x=P + 2), dict(stride=99), dict(stride=(1 << 40) + 1),
                                 dict(dst=None), dict(dst=P + 8)])
def test_conversions_refuse(bad):
    d = dict(kind=0, x=P, stride=100, dst=P) | bad
    lib = ie.lib()
    assert lib.iefwd_mx4_quantize(d["kind"], d["x"], d["stride"], d["dst"], 5, 100, None) == ie.EINVAL
    assert lib.iefwd_mx4_values(d["dst"], d["kind"], d["x"], d["stride"], 5, 100, None) == ie.EINVAL


def test_pack_refuses():
    for codes, scales, dst, k in ((None, P, P, 64), (P + 8, P, P, 64), (P, None, P, 64), (P, P, None, 64), (P, P, P + 4, 64), (P, P, P, 48)):
        assert ie.lib().iefwd_mx4_pack(codes, scales, dst, 5, k, None) == ie.EINVAL


@pytest.mark.parametrize("bad", [dict(epi=3), dict(a=None), dict(a=P + 8), dict(w=None), dict(w=P + 2), dict(out=None), dict(out=P + 2),
                                 dict(epi=2), dict(epi=2, resid=P + 4), dict(m=0), dict(n=0), dict(k=0)])
def test_products_refuse(bad):
    d = dict(epi=0, a=P, w=P, bias=None, resid=None, out=P, m=3, n=5, k=64) | bad
    assert ie.lib().iefwd_mx4_gemm(*d.values(), None) == ie.EINVAL and ie.last_error()
    assert ie.lib().iefwd_mx4_gemm_bf16(*d.values(), None) == ie.EINVAL
    few = d | dict(bad or {}, m=17)
    assert ie.lib().iefwd_mx4_gemm_bf16(*few.values(), None) == ie.EINVAL


def test_bf16_products_refuse_more_rows_and_odd_lengths():
    assert ie.lib().iefwd_mx4_gemm_bf16(0, P, P, None, None, P, 17, 5, 64, None) == ie.EINVAL
    assert ie.lib().iefwd_mx4_gemm_bf16(0, P, P, None, None, P, 16, 5, 60, None) == ie.EINVAL
    assert ie.lib().iefwd_mx4_gemm(0, P, P, None, None, P, 1 << 24, 1 << 24, 64, None) == ie.EINVAL      # M N past 2^36


def test_plain_form():
    """The tests' own quantisation, against the nearest of the listed values."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 96)) * np.exp(rng.standard_normal((50, 1)))
    codes, scales = X.quantize(x)
    v = X.values(codes, scales)
    unit = np.exp2(scales.astype(float) - 127).repeat(32, 1)
    best = np.abs(np.clip(x / unit, -6, 6)[..., None] - X.VALUES).min(-1)
    assert np.allclose(np.abs(np.clip(x / unit, -6, 6) - v / unit), best, atol=1e-12)
    top = np.abs(x.reshape(50, 3, 32)).max(-1)
    assert ((top / np.exp2(scales.astype(float) - 127) >= 4) & (top / np.exp2(scales.astype(float) - 127) < 8)).all()


# ------------------------------------------------------------------------------------ a cache in this form
def _desc(**kw):
    d = dict(abi_version=ie.ABI_VERSION, kv_type=ie.KV_MX4, n_pages=10, page_size=16, n_kv_heads=4, head_dim=64, k=P, v=2 * P)
    d.update(kw)
    return ie.PagedCacheDesc(**d)


def _read(cache, k=P, v=P, slots=P, n=5, ks=256, vs=256):
    return ie.lib().iefwd_paged_read(None if cache is None else ctypes.byref(cache), slots, k, v, n, ks, vs, None)


def _scored(cache, cap=0.0, slopes=None, scale=1.0, ctx=P, heads=8):
    return ie.lib().iefwd_paged_attention_scored(None if cache is None else ctypes.byref(cache), P, 512, heads, P, 200, 200, P, 3, scale,
                                                 cap, slopes, ctx, P, 1 << 30, None)


@pytest.mark.parametrize("bad", [dict(kv_type=2), dict(kv_type=4), dict(n_pages=0), dict(page_size=8), dict(head_dim=96), dict(k=None), dict(v=P + 8),
                                 dict(n_kv_heads=0)])
def test_bad_caches_are_refused(bad):
    c = _desc(**bad)
    assert _read(c) == ie.EINVAL and ie.last_error()
    assert _scored(c) == ie.EINVAL
    assert ie.lib().iefwd_paged_append(ctypes.byref(c), P, P, P, 5, 256, 256, None) == ie.EINVAL


def test_reads_and_scores_refuse():
    c = _desc()
    assert _read(None) == ie.EINVAL and _scored(None) == ie.EINVAL
    assert _read(_desc(abi_version=9)) == ie.EVERSION
    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(k=P + 8), dict(ks=255), dict(vs=252), dict(ks=(1 << 40) + 8),
               dict(n=(1 << 26) + 1)):
        assert _read(c, **kw) == ie.EINVAL, kw
    assert _read(c, n=0) == ie.OK
    for kw in (dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-19), dict(cap=2e18), dict(scale=float("inf")),
               dict(ctx=None), dict(heads=6)):
        assert _scored(c, **kw) == ie.EINVAL, kw


def test_workspace_of_a_4_bit_cache():
    sizes = []
    for kind in (ie.KV_BF16, ie.KV_MX4):
        n = ctypes.c_size_t()
        assert ie.lib().iefwd_paged_attention_workspace(ctypes.byref(_desc(kv_type=kind)), 3, 8, 200, ctypes.byref(n)) == ie.OK
        sizes.append(n.value)
    assert sizes[0] >= sizes[1] > 0


@pytest.mark.parametrize("rows,k", [((1 << 32) + 5, 32), (5, (1 << 32) + 32), (-1, 32), (1 << 40, 1 << 40)])
def test_sizes_beyond_32_bits_are_refused_by_the_binding(rows, k):
    with pytest.raises(ValueError, match="rows"):
        ie.Mx4Matrix(rows, k)
