"""Products of many rows in microscaled 4 bits: every tile (64, 128 and 256 rows, with outputs kept near and sent past the last
cache) with GELU, and with the residual in the output's place."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests.gpu_util import DEV, f64, sync, to_dev
from tests.test_gpu_mx4 import _given, _weight

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.mark.parametrize("m,n,k", [(700, 600, 416), (700, 604, 2100), (701, 601, 288),                    # 64 rows
                                   (1500, 1600, 640), (1500, 1604, 1060), (1501, 1603, 384),              # 128
                                   (3501, 3600, 384), (3500, 3604, 128), (3500, 3603, 1700),              # 256
                                   (4100, 4400, 96), (4096, 4404, 700), (4100, 4401, 160)])               # 256, more than 32 MiB
def test_gelu_and_residual_in_place(m, n, k):
    w, wv = _weight(n, k, n + k)
    x, av = _given(m, k, m)
    g = torch.Generator().manual_seed(m)
    bias, resid = torch.randn(n, generator=g).to(BF), torch.randn(m, n, generator=g)
    y = torch.from_numpy(av) @ torch.from_numpy(wv).T + bias.double()
    # exact terms, summed in fp32: 128 at a time, then the chunks and the waves, and the bias
    tol = 2.0 ** -23 * (128 + -(-k // 128) + 12) * (torch.from_numpy(np.abs(av)) @ torch.from_numpy(np.abs(wv)).T) + 2.0 ** -21 * y.abs()
    a = ie.Mx4Matrix(m, k)
    a.quantize(to_dev(x))
    out = torch.full((m + 1, n), 7.0, dtype=BF, device=DEV)
    w.product(a, out[:m], ie.EPI_BIAS_GELU_BF16, bias=to_dev(bias))
    rd = torch.full((m + 1, n), 7.0, device=DEV)
    rd[:m] = resid.to(DEV)
    w.product(a, rd[:m], ie.EPI_BIAS_RESID_F32, bias=to_dev(bias), resid=rd[:m])
    sync()
    assert (out[m:] == 7.0).all() and (rd[m:] == 7.0).all()
    act = 0.5 * y * (1.0 + torch.erf(y * 0.5 ** 0.5))
    # the GELU's slope is at most 1.13; its erf is good to 1.5e-7 and its exponential to 2^-20
    off = (torch.from_numpy(f64(out[:m])) - act).abs() - (1.13 * tol + 2.0 ** -19 * y.abs() + 2.0 ** -8 * act.abs())
    assert off.max() <= 0
    z = y + resid.double()
    assert ((torch.from_numpy(f64(rd[:m])) - z).abs() <= tol + 2.0 ** -21 * (z.abs() + resid.double().abs())).all()
