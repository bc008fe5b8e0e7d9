"""The paged cache's operators at the ends of their range: scales of every size in an 8-bit cache, streams with a CU quota, tables
and pools much larger than the requests in them."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
import workloads as W
from tests import paged_util as P
from tests.gpu_util import DEV, f64, instance_config, run_instance, sync

pytestmark = pytest.mark.gpu

SCALES = [2.0 ** -61, 2.0 ** 61, 3e-30, 7e25, -0.03, -5e-25, 1e-39, 3e38, 0.0, float("inf"), float("-inf"), float("nan"), 0.017]


def test_append_divides_by_scales_of_every_size():
    heads, dim, page, tokens = len(SCALES), 64, 16, 75
    g = torch.Generator().manual_seed(1)
    ks, vs = torch.tensor(SCALES), torch.tensor(SCALES[::-1])
    c = ie.PagedCache.empty(6, page, heads, dim, ks.to(DEV), vs.to(DEV))
    slots = torch.cat([torch.arange(70), torch.tensor([90, 75, 83, 95, 72])])
    rows = []
    for scale in (ks, vs):      # quotients from far below to far above e4m3's range, and single infinities, NaN and zeros
        unit = torch.where(torch.isfinite(scale) & (scale != 0), scale.abs(), torch.ones(())).double()
        x = unit.view(1, -1, 1) * torch.randn(tokens, heads, dim, generator=g) * 2.0 ** torch.randint(-12, 11, (tokens, heads, dim), generator=g)
        x = x.clamp(-3e38, 3e38).float().bfloat16()
        x[::7, :, ::9], x[1::7, :, 1::9], x[2::7, :, 2::9], x[3::7, :, 3::9] = float("inf"), float("-inf"), float("nan"), 0.0
        rows.append(x)
    c.append(rows[0].to(DEV), rows[1].to(DEV), slots.to(DEV))
    sync()
    for t, kind, x, scale in ((c.k, "k", rows[0], ks), (c.v, "v", rows[1], vs)):
        got = P.from_pages(t.view(torch.uint8).cpu(), kind).view(-1, heads, dim)[slots].view(torch.float8_e4m3fn).float()
        want = (x.float() / scale.view(1, -1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def _requests(lens, heads, kv, dim, page, seed, columns=None, pages=None):
    """A cache with the requests' tokens in it and the calls' operands."""
    g = torch.Generator().manual_seed(seed)
    held = [-(-n // page) for n in lens]
    pages = pages or sum(held) + 2
    c = ie.PagedCache.empty(pages, page, kv, dim)
    table = torch.zeros(len(lens), columns or max(held), dtype=torch.int32)
    free, slots = torch.randperm(pages, generator=g).int(), []
    at = 0
    for b, n in enumerate(lens):
        table[b, :held[b]] = free[at:at + held[b]]
        at += held[b]
        pos = torch.arange(n)
        slots.append(table[b, pos // page].long() * page + pos % page)
    k, v = (torch.randn(sum(lens), kv, dim, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(len(lens), heads, dim, generator=g).bfloat16()
    return c, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), torch.cat(slots).to(DEV), q.to(DEV), k.to(DEV), v.to(DEV)


@pytest.mark.parametrize("quota", [8, 64])
def test_every_call_on_a_stream_with_a_quota(quota):
    """Results are the same on a few CUs as on all, bit for bit."""
    lens, heads, kv, dim, page = [700, 3, 0, 5000, 256, 900], 8, 2, 128, 16
    c, table, tokens, slots, q, k, v = _requests(lens, heads, kv, dim, page, 2)
    g = torch.Generator(device=DEV).manual_seed(3)
    codes = torch.randint(0, 256, (1040, heads * dim // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.rand(1040, heads * dim // 64, generator=g, device=DEV).bfloat16()
    zeros, new = torch.zeros_like(tokens), torch.arange(len(lens), dtype=torch.int32, device=DEV) * 20
    results = []
    shape = W.model_shape("encoder_l1_d128_s32_b2")
    with ie.Instance(**instance_config(shape, 1, 32)) as inst:
        inst.set_quota(quota)
        run_instance(inst, W.make_input(1, 1, 32, 128))     # applies the mask
        for stream in (None, inst.stream_handle()):
            c.k.zero_()
            c.v.zero_()
            out = torch.empty(len(lens), heads, dim, dtype=torch.bfloat16, device=DEV)
            y = torch.empty(len(lens), 1040, dtype=torch.bfloat16, device=DEV)
            ws = c.workspace(len(lens), heads, table.shape[1])
            plan = [torch.full((len(lens), 7), -1, dtype=torch.int32, device=DEV), torch.arange(40, dtype=torch.int32, device=DEV),
                    torch.tensor([3, 40], device=DEV), torch.empty_like(tokens), torch.empty(2, dtype=torch.int64, device=DEV),
                    torch.empty(300, dtype=torch.int64, device=DEV), torch.empty(len(lens) + 1, dtype=torch.int32, device=DEV),
                    torch.empty(1, dtype=torch.int32, device=DEV)]
            sync()
            weight = ie.Q4Weight(codes, scales, stream=stream)
            ie.paged_plan(page, zeros, new, *plan, stream=stream)
            c.append(k, v, slots, stream=stream)
            c.attention(q, table, tokens, out, ws, stream=stream)
            weight.product(out.view(len(lens), -1), y, stream=stream)
            sync()
            results.append([out, y, c.k.clone(), c.v.clone(), *plan])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    got, o = f64(results[1][0]), 0
    for b, n in enumerate(lens):      # and they are right
        if n:
            ref, mag, dots = P.attention(f64(q[b:b + 1]), f64(k[o:o + n])[None], f64(v[o:o + n])[None], np.zeros((1, 1), int), [n], dim ** -0.5)
            assert (np.abs(got[b:b + 1] - ref) <= P.attention_tolerance(ref, mag, dots, n, dim, dim ** -0.5)).all()
            o += n
    # 300 slots for 0 + 20 + ... + 100 new tokens, 37 free pages: all are served
    assert int(results[1][-1]) == 0 and results[1][8].tolist() == [40 - 37 + 2 + 3 + 4 + 5 + 7, 40]


def test_a_table_and_a_pool_as_wide_as_a_server_s():
    """Short requests under a table of 1024 columns and a pool of 400 MB: the same bits as under a narrow one."""
    lens, heads, kv, dim, page = [300, 1, 0, 77, 512], 16, 4, 128, 16
    a = _requests(lens, heads, kv, dim, page, 4)
    b = _requests(lens, heads, kv, dim, page, 5, columns=1024, pages=12500)
    outs = []
    for c, table, tokens, slots, _, _, _ in (a, b):
        c.append(a[5], a[6], slots)
        out = torch.empty(len(lens), heads, dim, dtype=torch.bfloat16, device=DEV)
        c.attention(a[4], table, tokens, out, c.workspace(len(lens), heads, table.shape[1]))
        sync()
        outs.append(out)
    assert torch.equal(*outs)
