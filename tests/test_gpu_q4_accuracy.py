"""The 4-bit product where a form that sums codes and offsets apart loses bits: weights that equal their zero point,
activations of one sign, one large activation, infinities.  Tolerances count fp32 roundings of the terms
a s (code - zero) alone."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import paged_util as P
from tests.gpu_util import DEV, f64, sync, to_dev

pytestmark = pytest.mark.gpu


def _pack(codes):
    """uint8 [N, K] codes -> [N, K / 2] bytes."""
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def _product(a, codes, scales, zeros, resid):
    q = ie.Q4Weight(to_dev(_pack(codes)), to_dev(scales), None if zeros is None else to_dev(zeros))
    out = torch.empty_like(resid, device=DEV)
    q.product(to_dev(a), out, ie.EPI_BIAS_RESID_F32, resid=to_dev(resid))
    sync()
    return out


def _near_zero_weights(n, k, group, zeros, every, g):
    """Codes equal to their zero points but for each `every`-th weight of a feature."""
    z = torch.randint(0, 16, (n, k // group), generator=g, dtype=torch.uint8) if zeros else None
    codes = (torch.full((n, k // group), 8, dtype=torch.uint8) if z is None else z).repeat_interleave(group, 1)
    at = torch.arange(3, k, every)
    codes[:, at] = torch.randint(0, 16, (n, len(at)), generator=g, dtype=torch.uint8)
    return codes, z


@pytest.mark.parametrize("zeros", [True, False])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 6, 16])
def test_weights_at_their_zero_point_add_nothing(m, group, zeros):
    """Zero weights (of a pruned or padded feature) give zero, whatever the activations."""
    g = torch.Generator().manual_seed(m + group)
    n, k = 48, 4096
    codes, z = _near_zero_weights(n, k, group, zeros, 2 * k, g)
    codes[:, 3] = 8 if z is None else z[:, 0]
    scales = (0.01 + torch.rand(n, k // group, generator=g)).bfloat16()
    for a in (torch.randn(m, k, generator=g).abs(), torch.randn(m, k, generator=g), 1e30 * torch.rand(m, k, generator=g)):
        resid = torch.randn(m, n, generator=g)
        assert torch.equal(_product(a.bfloat16(), codes, scales, z, resid).cpu(), resid)


@pytest.mark.parametrize("zeros", [True, False])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(1, 48, 4096), (7, 1040, 4096), (16, 8208, 2048), (16, 80, 16384)])
def test_few_weights_beside_the_zero_point(m, n, k, group, zeros):
    """One weight in 512 differs from its zero point, the activations are of one sign: a sum has at most k / 512 terms that
    are not zero, each rounded at most once in every one of the sums it passes through (its own K steps' k / 512, the
    16 waves', the residual's)."""
    g = torch.Generator().manual_seed(m + n + k + group)
    codes, z = _near_zero_weights(n, k, group, zeros, 512, g)
    scales = (0.01 + 0.01 * torch.rand(n, k // group, generator=g)).bfloat16()
    a, resid = torch.randn(m, k, generator=g).abs().bfloat16(), torch.zeros(m, n)
    w = P.q4_weight(_pack(codes).numpy(), f64(scales), None if z is None else z.numpy())
    y, mag = f64(a) @ w.T, np.abs(f64(a)) @ np.abs(w).T
    tol = 2.0 ** -23 * (k // 512 + 20) * mag
    assert (np.abs(f64(_product(a, codes, scales, z, resid)) - y) <= tol).all()


@pytest.mark.parametrize("group", [32, 128])
def test_a_large_activation_at_zero_weights_hides_nothing(group):
    """Whole numbers whose sums fit 24 bits come out exactly, whatever stands at weights that are zero."""
    g = torch.Generator().manual_seed(group)
    m, n, k = 5, 64, 1024
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    z = torch.randint(0, 16, (n, k // group), generator=g, dtype=torch.uint8)
    a = torch.randint(0, 256, (m, k), generator=g).float()
    large = torch.arange(5, k, 16)
    a[:, large] = 2.0 ** 24 * torch.randint(1, 256, (m, len(large)), generator=g).float()
    codes[:, large] = z.repeat_interleave(group, 1)[:, large]
    a = a.bfloat16()
    scales = torch.full((n, k // group), 2.0).bfloat16()
    want = f64(a) @ P.q4_weight(_pack(codes).numpy(), f64(scales), z.numpy()).T
    assert np.abs(want).max() < 2 ** 24      # 2 x 255 x 15 x 1024 at most, in units of 2
    assert np.array_equal(f64(_product(a, codes, scales, z, torch.zeros(m, n))), want)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("k", [512, 8192])
@pytest.mark.parametrize("shape", ["one_sign", "after_gelu", "one_channel"])
def test_activations_that_do_not_cancel(shape, k, group):
    """fp32 sums of the terms a s (code - zero): a rounding for each of a group's terms, each group and each wave."""
    g = torch.Generator().manual_seed(k + group)
    m, n = 9, 272
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    z = torch.randint(0, 16, (n, k // group), generator=g, dtype=torch.uint8)
    scales = (0.01 * (1 + torch.rand(n, k // group, generator=g))).bfloat16()
    a = torch.randn(m, k, generator=g)
    a = a.abs() if shape == "one_sign" else torch.nn.functional.gelu(a) if shape == "after_gelu" else a
    if shape == "one_channel":
        a[:, k // 3] = 3000.0
    a, resid = a.bfloat16(), torch.randn(m, n, generator=g)
    w = P.q4_weight(_pack(codes).numpy(), f64(scales), z.numpy())
    y, mag = f64(a) @ w.T, np.abs(f64(a)) @ np.abs(w).T
    tol = 2.0 ** -23 * (group + k // group + 16) * mag + 2.0 ** -23 * (np.abs(y) + np.abs(f64(resid)))
    assert (np.abs(f64(_product(a, codes, scales, z, resid)) - y - f64(resid)) <= tol).all()


def test_infinite_and_nan_activations():
    """inf times a weight is an infinity of its sign, times a weight of zero NaN; the other rows do not see it."""
    g = torch.Generator().manual_seed(1)
    m, n, k, group = 4, 64, 256, 32
    codes = torch.randint(0, 16, (n, k), generator=g, dtype=torch.uint8)
    z = torch.randint(0, 16, (n, k // group), generator=g, dtype=torch.uint8)
    scales = (0.01 + torch.rand(n, k // group, generator=g)).bfloat16()
    scales[1::2] *= -1
    a, resid = torch.randn(m, k, generator=g).bfloat16(), torch.zeros(m, n)
    plain = _product(a, codes, scales, z, resid)
    a[1, 77], a[2, 130], a[3, 9] = float("inf"), float("-inf"), float("nan")
    got = _product(a, codes, scales, z, resid).cpu()
    assert torch.equal(got[0], plain[0].cpu())
    w = torch.from_numpy(P.q4_weight(_pack(codes).numpy(), f64(scales), z.numpy())).float()
    for row, at in ((1, 77), (2, 130)):
        want = a[row, at].float() * w[:, at]                 # +-inf, or NaN where the weight is zero
        assert torch.isnan(want).any() and (want == float("inf")).any() and (want == float("-inf")).any()
        assert torch.equal(torch.isnan(got[row]), torch.isnan(want))
        assert torch.equal(got[row][~torch.isnan(want)], want[~torch.isnan(want)])
    assert torch.isnan(got[3]).all()
