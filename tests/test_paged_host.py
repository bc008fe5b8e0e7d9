"""What the paged cache's and the 4-bit product's entry points refuse before any device work, their sizes and the
descriptor's layout (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2503_05130_amd as ie

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20          # stands for an aligned device address; nothing here reads it


def _desc(**kw):
    d = dict(abi_version=ie.ABI_VERSION, kv_type=ie.KV_BF16, n_pages=10, page_size=16, n_kv_heads=4, head_dim=64, k=P, v=2 * P)
    d.update(kw)
    return ie.PagedCacheDesc(**d)


def test_descriptor_layout_matches_c(tmp_path):
    fields = [f for f, _ in ie.PagedCacheDesc._fields_]
    prog = tmp_path / "layout.c"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"iefwd.h\"\nint main(void) {\n"
                    '  printf("size %zu\\n", sizeof(iefwd_paged_cache));\n' +
                    "".join(f'  printf("{f} %zu\\n", offsetof(iefwd_paged_cache, {f}));\n' for f in fields) + "  return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{ROOT}/include", str(prog), "-o", str(exe)], check=True)
    out = dict(line.split() for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(out.pop("size")) == ctypes.sizeof(ie.PagedCacheDesc)
    assert {f: int(o) for f, o in out.items()} == {f: getattr(ie.PagedCacheDesc, f).offset for f in fields}


BAD_CACHES = [dict(kv_type=2), dict(n_pages=0), dict(n_pages=2 ** 31), dict(page_size=8), dict(page_size=24), dict(page_size=512),
              dict(page_size=0), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=32), dict(head_dim=96),
              dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(kv_type=ie.KV_E4M3),
              dict(kv_type=ie.KV_E4M3, k_scale=P)]


def _append(cache, k=P, v=P, slots=P, n=5, ks=256, vs=256):
    return ie.lib().iefwd_paged_append(None if cache is None else ctypes.byref(cache), k, v, slots, n, ks, vs, None)


def _attention(cache, q=P, qs=512, heads=8, table=P, stride=200, pages=200, lens=P, batch=3, scale=1.0, ctx=P, ws=P, bytes_=1 << 30):
    return ie.lib().iefwd_paged_attention(None if cache is None else ctypes.byref(cache), q, qs, heads, table, stride, pages, lens,
                                          batch, scale, ctx, ws, bytes_, None)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches_are_refused(bad):
    c = _desc(**bad)
    n = ctypes.c_size_t(7)
    assert _append(c) == ie.EINVAL and ie.last_error()
    assert _attention(c) == ie.EINVAL
    assert ie.lib().iefwd_paged_attention_workspace(ctypes.byref(c), 1, 4, 10, ctypes.byref(n)) == ie.EINVAL
    assert n.value == 7


def test_null_cache_and_versions():
    assert _append(None) == ie.EINVAL and _attention(None) == ie.EINVAL
    assert _append(_desc(abi_version=9)) == ie.EVERSION and _attention(_desc(abi_version=0)) == ie.EVERSION


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(slots=None), dict(k=P + 2), dict(v=P + 8), dict(ks=255),
                                 dict(vs=248), dict(ks=260), dict(ks=2 ** 41), dict(n=2 ** 26 + 1)])
def test_append_refuses(bad):
    assert _append(_desc(), **bad) == ie.EINVAL and ie.last_error()


def test_append_of_nothing_is_fine():
    assert _append(_desc(), k=None, v=None, slots=None, n=0) == ie.OK


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=P + 4), dict(qs=511), dict(qs=516), dict(heads=0), dict(heads=6),
                                 dict(heads=1028), dict(table=None), dict(lens=None), dict(ctx=None), dict(ctx=P + 2), dict(stride=199),
                                 dict(pages=0), dict(stride=2 ** 31), dict(stride=2 ** 27, pages=2 ** 27), dict(batch=0),
                                 dict(batch=65536), dict(batch=5000, heads=1024, qs=65536), dict(scale=float("inf")), dict(scale=float("nan")), dict(ws=None),
                                 dict(ws=P + 4), dict(bytes_=100)])      # 3200 keys: more than a part
def test_attention_refuses(bad):
    assert _attention(_desc(), **bad) == ie.EINVAL and ie.last_error()


@pytest.mark.parametrize("batch,heads,kv", [(1, 4, 4), (1, 1, 1), (3, 32, 8), (16, 16, 16), (20, 16, 16), (1, 40, 2), (300, 64, 1),
                                            (64, 32, 8)])
def test_workspace_holds_the_parts_of_every_length(batch, heads, kv):
    """The count of parts falls where a part doubles, so the longest request need not have the most."""
    most, last, rng = 1, 0, list(range(0, 9000)) + list(range(9000, 300000, 37)) + [2 ** k + d for k in range(14, 20) for d in (0, 1)]
    lengths = iter(sorted(rng))
    seen = next(lengths)
    for pages in (1, 2, 16, 17, 63, 64, 65, 128, 129, 500, 512, 513, 514, 1000, 5000, 16000, 18000):
        while seen is not None and seen <= 16 * pages:
            keys = ie.test_paged_split(batch, heads, kv, seen)
            assert (keys >= last or last == 512) and keys & (keys - 1) == 0
            last, most = keys, max(most, -(-seen // keys))
            seen = next(lengths, None)
        n = ctypes.c_size_t()
        assert ie.lib().iefwd_paged_attention_workspace(ctypes.byref(_desc(n_kv_heads=kv, head_dim=128)), batch, heads, pages,
                                                        ctypes.byref(n)) == ie.OK
        parts = n.value // (batch * heads * (128 + 2) * 4)
        assert n.value == parts * batch * heads * (128 + 2) * 4
        assert parts == 0 and most == 1 or parts >= most and parts <= most + 1      # the sample may miss the very most
        assert parts <= 128


@pytest.mark.parametrize("bad", [(0, 4, 4, 1), (65536, 4, 4, 1), (1, 0, 1, 1), (1, 6, 4, 1), (1, 4, 0, 1), (1, 1028, 1, 1),
                                 (1, 4, 4, 2 ** 30 + 1)])
def test_split_refuses(bad):
    with pytest.raises(ie.IefwdError) as e:
        ie.test_paged_split(*bad)
    assert e.value.status == ie.EINVAL


def _plan(batch=4, page=16, lens=P, new=2 * P, table=P, stride=10, pages=10, ring=P, size=50, counters=P, lens_out=3 * P,
          counters_out=2 * P, slots=P, room=9, starts=P, refused=P):
    return ie.lib().iefwd_paged_plan(batch, page, lens, new, table, stride, pages, ring, size, counters, lens_out, counters_out,
                                     slots, room, starts, refused, None)


@pytest.mark.parametrize("bad", [dict(batch=0), dict(batch=4097), dict(page=15), dict(page=0), dict(lens=None), dict(new=None),
                                 dict(table=None), dict(ring=None), dict(counters=None), dict(lens_out=None),
                                 dict(counters_out=None), dict(slots=None), dict(starts=None), dict(refused=None), dict(stride=9),
                                 dict(pages=0), dict(stride=2 ** 27, pages=2 ** 27), dict(size=0), dict(size=2 ** 31),
                                 dict(room=2 ** 31), dict(lens_out=P), dict(lens_out=2 * P), dict(counters_out=P)])
def test_plan_refuses(bad):
    assert _plan(**bad) == ie.EINVAL and ie.last_error()


SHAPES = [dict(N=0), dict(N=24), dict(K=0), dict(K=96), dict(group=16), dict(group=256), dict(group=0), dict(N=2 ** 20, K=2 ** 12), dict(N=16, K=2 ** 24 + 128)]


def _bytes(N=32, K=128, group=64):
    n = ctypes.c_size_t()
    return ie.lib().iefwd_q4_packed_bytes(N, K, group, ctypes.byref(n)), n.value


@pytest.mark.parametrize("bad", SHAPES)
def test_q4_shapes_are_refused(bad):
    s = dict(N=32, K=128, group=64)
    s.update(bad)
    assert _bytes(**s)[0] == ie.EINVAL and ie.last_error()
    assert ie.lib().iefwd_q4_pack(P, P, None, P, s["N"], s["K"], s["group"], None) == ie.EINVAL
    assert ie.lib().iefwd_q4_gemm(0, P, P, None, None, P, 1, s["N"], s["K"], s["group"], None) == ie.EINVAL


def test_q4_sizes():
    assert _bytes() == (ie.OK, 32 * 64 + 32 * 2 * 4)
    assert _bytes(16, 160, 32) == (ie.OK, 16 * 128 + 16 * 8 * 4)      # K rounded up to 256


@pytest.mark.parametrize("args", [(None, P, P), (P, None, P), (P, P, None), (P, P, P + 4)])
def test_q4_pack_refuses(args):
    codes, scales, dst = args
    assert ie.lib().iefwd_q4_pack(codes, scales, None, dst, 32, 128, 64, None) == ie.EINVAL


@pytest.mark.parametrize("bad", [dict(epi=3), dict(epi=2), dict(a=None), dict(packed=None), dict(out=None), dict(M=0), dict(M=17),
                                 dict(a=P + 8), dict(packed=P + 4)])
def test_q4_gemm_refuses(bad):
    d = dict(epi=0, a=P, packed=P, out=P, M=3)
    d.update(bad)
    assert ie.lib().iefwd_q4_gemm(d["epi"], d["a"], d["packed"], None, None, d["out"], d["M"], 32, 128, 64, None) == ie.EINVAL


def test_binding_refuses_what_is_not_on_the_gpu():
    t = torch.zeros(10, 4, 8, 16, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        ie.PagedCache(t, t)
    with pytest.raises(ValueError, match="GPU"):
        ie.Q4Weight(torch.zeros(16, 64, dtype=torch.uint8), torch.zeros(16, 1, dtype=torch.bfloat16))
    z = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        ie.paged_plan(16, z, z, z, z, z, z, z, z, z, z)
