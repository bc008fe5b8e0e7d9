"""The decode-step product with 4-bit weights on the GPU against a plain 64-bit implementation."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import paged_util as P
from tests.gpu_util import DEV, f64, sync, to_dev

pytestmark = pytest.mark.gpu


def _case(n, k, group, zeros, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8)
    scales = (0.01 * (1 + spread * torch.rand(n, k // group, generator=g))).bfloat16()
    scales[::5, ::3] *= -1
    z = torch.randint(0, 16, (n, k // group), generator=g, dtype=torch.uint8) if zeros else None
    w = P.q4_weight(codes.numpy(), f64(scales), None if z is None else z.numpy())
    return codes, scales, z, w


def _tolerance(a, scales, group, y, f32, extra=0.0):
    """fp32 sums: per group the 16 + code products and their correction, each term at most 31 |a s| and each sum of up to
    `group` terms rounded as often, then the groups' sum and the epilogue; and half a step of a bf16 result."""
    mag = np.abs(a).reshape(len(a), -1, group).sum(-1) @ np.abs(scales).T          # sum |a s|
    e = 2.0 ** -24 * (62 * (group + 4) + 16 * scales.shape[1]) * mag + extra + 2.0 ** -23 * np.abs(y)
    return e if f32 else e + 2.0 ** -8 * np.abs(y)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 3, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("n,k", [(16, 128), (48, 384), (768, 768), (1040, 2176), (8192, 256), (16400, 128)])
def test_product(m, n, k, group):
    codes, scales, z, w = _case(n, k, group, (m + n // 16) % 2 == 0, m * n + k)
    g = torch.Generator().manual_seed(m)
    a, bias = torch.randn(m, k, generator=g).bfloat16(), torch.randn(n, generator=g).bfloat16()
    q = ie.Q4Weight(to_dev(codes), to_dev(scales), None if z is None else to_dev(z))
    out = torch.full((m + 1, n), 7.0, dtype=torch.bfloat16, device=DEV)
    q.product(to_dev(a), out[:m], bias=to_dev(bias))
    sync()
    y = f64(a) @ w.T + f64(bias)
    assert (np.abs(f64(out[:m]) - y) <= _tolerance(f64(a), f64(scales), group, y, False)).all()
    assert (out[m:] == 7.0).all()


@pytest.mark.parametrize("k,group", [(32, 32), (64, 32), (160, 32), (192, 64), (704, 64), (8224, 32), (16384, 128)])
@pytest.mark.parametrize("m", [1, 7, 16])
def test_epilogues_and_odd_lengths(m, k, group):
    n = 80
    codes, scales, z, w = _case(n, k, group, True, k + m)
    g = torch.Generator().manual_seed(k)
    a, bias = torch.randn(m, k, generator=g).bfloat16(), torch.randn(n, generator=g).bfloat16()
    resid = torch.randn(m, n, generator=g)
    q = ie.Q4Weight(to_dev(codes), to_dev(scales), to_dev(z))
    plain = f64(a) @ w.T
    y = plain + f64(bias)
    out = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    q.product(to_dev(a), out)
    sync()
    assert (np.abs(f64(out) - plain) <= _tolerance(f64(a), f64(scales), group, plain, False)).all()
    q.product(to_dev(a), out, ie.EPI_BIAS_GELU_BF16, bias=to_dev(bias))
    sync()
    # GELU's slope is below 1.13; its own error is 1.5e-7 of erfc, times |y| / 2, and some fp32 steps
    tol = _tolerance(f64(a), f64(scales), group, y, True) * 1.13 + (1e-7 + 2.0 ** -21) * np.abs(y) + 2.0 ** -8 * np.abs(P.gelu(y))
    assert (np.abs(f64(out) - P.gelu(y)) <= tol).all()
    res = to_dev(resid)
    q.product(to_dev(a), res, ie.EPI_BIAS_RESID_F32, bias=to_dev(bias), resid=res)     # in place
    sync()
    want = y + f64(resid)
    assert (np.abs(f64(res) - want) <= _tolerance(f64(a), f64(scales), group, want, True, 2.0 ** -23 * np.abs(y))).all()


def test_every_code_and_zero():
    # 16 zeros x 16 codes: feature z, group of 32 weights with code c each; activations of ones
    codes = torch.arange(16).repeat_interleave(16).repeat(16, 1).to(torch.uint8) * 17
    scales = torch.ones(16, 16).bfloat16()
    zeros = torch.arange(16, dtype=torch.uint8)[:, None].repeat(1, 16).contiguous()
    for c in range(16):
        a = torch.zeros(1, 512)
        a[0, 32 * c:32 * c + 32] = 1
        for z, want in ((zeros, 32.0 * (c - torch.arange(16.0))), (None, torch.full((16,), 32.0 * (c - 8)))):
            out = torch.empty(1, 16, dtype=torch.float32, device=DEV)
            q = ie.Q4Weight(to_dev(codes), to_dev(scales), None if z is None else to_dev(z))
            q.product(to_dev(a.bfloat16()), out, ie.EPI_BIAS_RESID_F32, resid=torch.zeros_like(out))
            sync()
            assert torch.equal(out.cpu()[0], want)


def test_a_row_depends_on_no_other():
    codes, scales, z, _ = _case(1040, 1056, 32, True, 5)
    q = ie.Q4Weight(to_dev(codes), to_dev(scales), to_dev(z))
    a = to_dev(torch.randn(16, 1056).bfloat16())
    full = torch.empty(16, 1040, dtype=torch.bfloat16, device=DEV)
    q.product(a, full)
    a[1, 5] = float("nan")
    for m in (1, 4, 5, 8, 9, 16):
        out = torch.empty(m, 1040, dtype=torch.bfloat16, device=DEV)
        q.product(a[:m], out)
        sync()
        rows = [r for r in range(m) if r != 1]
        assert torch.equal(out[rows], full[rows])
        assert m == 1 or torch.isnan(out[1]).all()


def test_captured_product():
    codes, scales, z, _ = _case(256, 512, 64, True, 6)
    q = ie.Q4Weight(to_dev(codes), to_dev(scales), to_dev(z))
    a = to_dev(torch.randn(2, 512).bfloat16())
    out = [torch.empty(2, 256, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.product(a, out[0])
    for i in range(4):
        a.copy_(torch.randn(2, 512).bfloat16())
        graph.replay()
        q.product(a, out[1])
        sync()
        assert torch.equal(out[0], out[1])
