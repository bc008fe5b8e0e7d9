"""Matrices in microscaled 4 bits on the GPU against plain 64-bit forms: quantisation, layout, values and products."""
import math

import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import mx4_util as X
from tests.gpu_util import DEV, f64, sync, to_dev

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _rows(m, k, dtype, seed, special=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, k, generator=g) * torch.exp(2.0 * torch.randn(m, 1, generator=g))
    if special:
        flat = x.view(-1)
        flat[::7] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -2.5, 7.9, 6.0, 0.0, -0.0])[torch.arange(len(flat[::7])) % 12]
        x[0] *= 2.0 ** -126                    # subnormal numbers and scales at the lower end
        if m > 1:
            x[1] = x[1].sign() * 2.0 ** 127    # the upper end
        if m > 2:
            x[2] = 0.0
            x[2, ::3] = -0.0
        if m > 3:
            x[3, k // 2] = math.nan
        if m > 4:
            x[4, 0], x[4, -1] = math.inf, -math.inf
    return x.to(dtype)


def _same(a, b):
    """Equal as numbers, zeros by their sign as well, NaN for NaN."""
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return a.shape == b.shape and bool((((a == b) & (np.signbit(a) == np.signbit(b))) | (np.isnan(a) & np.isnan(b))).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 32), (2, 8), (5, 33), (16, 128), (17, 100), (40, 520), (33, 1000), (3, 4104)])
@pytest.mark.parametrize("gap,first", [(0, 0), (8, 0), (1, 1), (5, 3)])
def test_quantize(m, k, dtype, gap, first):
    x = _rows(m, k, dtype, m * 31 + k, special=True)
    wide = torch.full((m, k + gap + first), 9.0, dtype=dtype, device=DEV)
    wide[:, first:first + k] = x
    a = ie.Mx4Matrix(m, k)
    a.packed.fill_(0x5A)
    a.quantize(wide[:, first:first + k])
    codes, scales = X.quantize(f64(x))
    sync()
    np.testing.assert_array_equal(a.packed.cpu().numpy(), X.packed(codes, scales, m, k))
    for out_type in (BF, F32):
        out = torch.full((m + 1, k + gap + first), 3.0, dtype=out_type, device=DEV)
        a.values(out[:m, first:first + k])
        sync()
        assert _same(f64(out[:m, first:first + k]), X.values(codes, scales)[:, :k])
        assert (out[m] == 3.0).all() and (out[:, :first] == 3.0).all() and (out[:, first + k:] == 3.0).all()


def test_every_bf16_in_every_place():
    """All bit patterns of bf16, each as the largest of its block and beside larger ones."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF)
    rows = [bits.view(2048, 32), bits.view(32, 2048).t().contiguous(), bits[torch.randperm(65536, generator=torch.Generator().manual_seed(3))].view(2048, 32)]
    x = torch.cat(rows)
    a = ie.Mx4Matrix(*x.shape)
    a.quantize(to_dev(x))
    out = torch.empty(x.shape, dtype=F32, device=DEV)
    a.values(out)
    codes, scales = X.quantize(f64(x))
    sync()
    np.testing.assert_array_equal(a.packed.cpu().numpy(), X.packed(codes, scales, *x.shape))
    assert _same(f64(out), X.values(codes, scales))


def test_fewer_rows_leave_the_rest():
    a = ie.Mx4Matrix(70, 200)
    a.packed.fill_(0x77)
    x = _rows(20, 200, F32, 5)
    a.quantize(to_dev(x))
    sync()
    tile = len(a.packed) // 5
    got = a.packed.cpu().numpy()
    codes, scales = X.quantize(f64(x))
    np.testing.assert_array_equal(got[:2 * tile], X.packed(codes, scales, 20, 200))
    assert (got[2 * tile:] == 0x77).all()


@pytest.mark.parametrize("n,k", [(1, 32), (16, 128), (50, 160), (33, 1056), (130, 544)])
def test_load(n, k):
    rng = np.random.default_rng(n * k)
    codes, scales = rng.integers(0, 16, (n, k), dtype=np.uint8), rng.integers(0, 256, (n, k // 32), dtype=np.uint8)
    w = ie.Mx4Matrix(n, k)
    w.packed.fill_(0x5A)
    w.load(to_dev(torch.from_numpy(X.pairs(codes))), to_dev(torch.from_numpy(scales)))
    out = torch.empty((n, k), dtype=F32, device=DEV)
    w.values(out)
    sync()
    np.testing.assert_array_equal(w.packed.cpu().numpy(), X.packed(codes, scales, n, k))
    with np.errstate(over="ignore"):
        assert _same(f64(out), X.values(codes, scales).astype(np.float32))      # 6 times 2^127 and the like: infinite in fp32


def _weight(n, k, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, k, generator=g) * 0.05
    codes, scales = X.quantize(f64(x))
    w = ie.Mx4Matrix(n, k)
    if k % 32 == 0:
        w.load(to_dev(torch.from_numpy(X.pairs(codes))), to_dev(torch.from_numpy(scales)))
    else:
        w.quantize(to_dev(x))
    return w, X.values(codes, scales)[:, :k]


def _given(m, k, seed):
    x = _rows(m, k, BF, seed)
    codes, scales = X.quantize(f64(x))
    return x, X.values(codes, scales)[:, :k]


MS = [1, 2, 4, 5, 8, 11, 16, 17, 32, 33, 64, 65, 127, 130, 257]


@pytest.mark.parametrize("m", MS)
@pytest.mark.parametrize("n,k", [(16, 128), (1, 32), (50, 384), (257, 1000), (1040, 2176), (768, 768)])
def test_product(m, n, k):
    w, wv = _weight(n, k, n + k)
    x, av = _given(m, k, m)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(m)).to(BF)
    y = av @ wv.T + f64(bias)
    tol = X.product_tolerance(av, wv, y, k, False)
    a = ie.Mx4Matrix(m, k)
    a.quantize(to_dev(x))
    ways = [a] + ([to_dev(x)] if m <= 16 else [])
    for way in ways:
        out = torch.full((m + 1, n), 7.0, dtype=BF, device=DEV)
        w.product(way, out[:m], bias=to_dev(bias))
        sync()
        assert (np.abs(f64(out[:m]) - y) <= tol).all()
        assert (out[m:] == 7.0).all()


@pytest.mark.parametrize("m", [1, 7, 16, 40, 129, 300])
@pytest.mark.parametrize("n,k", [(80, 96), (321, 640), (512, 4160)])
def test_epilogues(m, n, k):
    w, wv = _weight(n, k, n * 3 + k)
    x, av = _given(m, k, m + 1)
    g = torch.Generator().manual_seed(k)
    bias, resid = torch.randn(n, generator=g).to(BF), torch.randn(m, n, generator=g)
    plain = av @ wv.T
    a = ie.Mx4Matrix(m + 5, k)      # more rows than the product takes
    a.quantize(to_dev(x))
    for way in [a] + ([to_dev(x)] if m <= 16 else []):
        out = torch.empty((m, n), dtype=BF, device=DEV)
        w.product(way, out)
        sync()
        assert (np.abs(f64(out) - plain) <= X.product_tolerance(av, wv, plain, k, False)).all()
        y = plain + f64(bias)
        w.product(way, out, ie.EPI_BIAS_GELU_BF16, bias=to_dev(bias))
        sync()
        act = 0.5 * y * (1.0 + np.vectorize(math.erf)(y / math.sqrt(2.0)))
        # the GELU's slope is at most 1.13; its erf is good to 1.5e-7 and its exponential to 2^-20
        tol = 1.13 * X.product_tolerance(av, wv, y, k, True) + 2.0 ** -19 * np.abs(y) + 2.0 ** -8 * np.abs(act)
        assert (np.abs(f64(out) - act) <= tol).all()
        rd = to_dev(resid)
        w.product(way, rd, ie.EPI_BIAS_RESID_F32, bias=to_dev(bias), resid=rd)      # in place
        sync()
        z = y + f64(resid)
        assert (np.abs(f64(rd) - z) <= X.product_tolerance(av, wv, np.abs(y) + np.abs(z), k, True)).all()


@pytest.mark.parametrize("m", [3, 16, 40, 200])
def test_not_a_number_stays_in_its_row_and_column(m):
    n, k = 100, 416
    g = torch.Generator().manual_seed(m)
    x, wx = torch.randn(m, k, generator=g).to(BF), torch.randn(n, k, generator=g)
    x[1, 77] = math.inf
    x[m - 1, 400] = math.nan
    wx[63, 5] = math.nan
    w, a = ie.Mx4Matrix(n, k), ie.Mx4Matrix(m, k)
    w.quantize(to_dev(wx))
    a.quantize(to_dev(x))
    want = np.zeros((m, n), bool)
    want[[1, m - 1]] = True
    want[:, 63] = True
    for way in [a] + ([to_dev(x)] if m <= 16 else []):
        out = torch.zeros((m, n), dtype=BF, device=DEV)
        w.product(way, out)
        sync()
        np.testing.assert_array_equal(np.isnan(f64(out)), want)


@pytest.mark.parametrize("m", [5, 16, 48, 300])
def test_rows_do_not_depend_on_each_other(m):
    n, k = 272, 1280
    w, _ = _weight(n, k, 8)
    x, _ = _given(m, k, 9)
    other = _rows(m, k, BF, 10)
    other[m // 2] = x[m // 2]
    outs = []
    for rows in (x, other):
        a = ie.Mx4Matrix(m, k)
        a.quantize(to_dev(rows))
        out = torch.empty((m, n), dtype=F32, device=DEV)
        w.product(a, out, ie.EPI_BIAS_RESID_F32, resid=torch.zeros_like(out))
        outs.append(out[m // 2].clone())
        if m <= 16:
            w.product(to_dev(rows), out, ie.EPI_BIAS_RESID_F32, resid=torch.zeros_like(out))
            outs.append(out[m // 2].clone())
    sync()
    assert torch.equal(outs[0], outs[-2 if m <= 16 else -1])
    if m <= 16:
        assert torch.equal(outs[1], outs[3])


def test_captured_and_on_another_stream():
    m, n, k = 24, 160, 640
    w, wv = _weight(n, k, 4)
    x, av = _given(m, k, 11)
    xd, a = to_dev(x), ie.Mx4Matrix(m, k)
    out, back = torch.empty((m, n), dtype=BF, device=DEV), torch.empty((m, k), dtype=BF, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.quantize(xd)
        a.values(back)
        w.product(a, out)
    for seed in (11, 12, 13):
        x, av = _given(m, k, seed)
        xd.copy_(x)
        out.zero_()
        graph.replay()
        sync()
        y = av @ wv.T
        assert _same(f64(back), av)
        assert (np.abs(f64(out) - y) <= X.product_tolerance(av, wv, y, k, False)).all()
    out.zero_()
    sync()
    a.quantize(xd, stream=side)
    w.product(a, out, stream=side)
    side.synchronize()
    assert (np.abs(f64(out) - y) <= X.product_tolerance(av, wv, y, k, False)).all()


def test_refusals_of_the_binding():
    a, w = ie.Mx4Matrix(20, 64), ie.Mx4Matrix(30, 64)
    x = torch.zeros((20, 64), dtype=BF, device=DEV)
    out = torch.zeros((20, 30), dtype=BF, device=DEV)
    bad = [lambda: a.quantize(torch.zeros((21, 64), dtype=BF, device=DEV)), lambda: a.quantize(x[:, :32]), lambda: a.quantize(x.half()),
           lambda: a.quantize(x.cpu()), lambda: a.quantize(torch.zeros((64, 20), dtype=BF, device=DEV).t()),
           lambda: a.values(torch.zeros((21, 64), dtype=BF, device=DEV)), lambda: a.values(torch.zeros((20, 63), dtype=BF, device=DEV)),
           lambda: w.product(ie.Mx4Matrix(20, 32), out), lambda: w.product(ie.Mx4Matrix(19, 64), out),
           lambda: w.product(a, out[:, :29]), lambda: w.product(a, out.float()), lambda: w.product(a, out, bias=out[0].float()),
           lambda: w.product(a, out.float(), ie.EPI_BIAS_RESID_F32), lambda: w.product(x.float(), out),
           lambda: a.load(torch.zeros((20, 32), dtype=torch.uint8, device=DEV), torch.zeros((20, 3), dtype=torch.uint8, device=DEV)),
           lambda: ie.Mx4Matrix(3, 40).load(torch.zeros((3, 20), dtype=torch.uint8, device=DEV), torch.zeros((3, 1), dtype=torch.uint8, device=DEV))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in [lambda: w.product(x, out), lambda: ie.Mx4Matrix(0, 5), lambda: ie.Mx4Matrix(5, 0),      # more than 16 rows of bf16
                 lambda: ie.Mx4Matrix(5, 12).product(torch.zeros((2, 12), dtype=BF, device=DEV), torch.zeros((2, 5), dtype=BF, device=DEV))]:
        with pytest.raises(ie.IefwdError) as e:
            call()
        assert e.value.status == ie.EINVAL


@pytest.mark.parametrize("m,n,k", [(1100, 1040, 416), (1025, 1025, 128), (2100, 700, 1700), (3501, 3603, 384), (4096, 3500, 640), (8200, 1601, 96),
                                   (2100, 2100, 300), (1601, 2304, 1152), (4000, 1500, 2700), (3500, 3600, 2176), (1100, 1040, 4160),
                                   (5200, 3608, 256), (6100, 3100, 160)])
@pytest.mark.parametrize("epilogue", ["bias", "residual"])
def test_many_rows(m, n, k, epilogue):
    w, wv = _weight(n, k, n + k)
    x, av = _given(m, k, m)
    g = torch.Generator().manual_seed(m)
    bias, resid = torch.randn(n, generator=g).to(BF), torch.randn(m, n, generator=g)
    y = (torch.from_numpy(av) @ torch.from_numpy(wv).T).numpy() + f64(bias)
    a = ie.Mx4Matrix(m, k)
    a.quantize(to_dev(x))
    if epilogue == "bias":
        out = torch.full((m + 1, n), 7.0, dtype=BF, device=DEV)
        w.product(a, out[:m], bias=to_dev(bias))
    else:
        out = torch.full((m + 1, n), 7.0, device=DEV)
        w.product(a, out[:m], ie.EPI_BIAS_RESID_F32, bias=to_dev(bias), resid=to_dev(resid))
        y = y + f64(resid)
    sync()
    assert (out[m:] == 7.0).all()
    size = torch.from_numpy(np.abs(av)) @ torch.from_numpy(np.abs(wv)).T
    tol = 2.0 ** -23 * (128 + -(-k // 128) + 12) * size.numpy() + 2.0 ** -21 * (np.abs(y) + np.abs(f64(resid)))
    assert (np.abs(f64(out[:m]) - y) <= tol + (2.0 ** -8 * np.abs(y) if epilogue == "bias" else 0)).all()


@pytest.mark.parametrize("m", [1, 6, 16, 29])
@pytest.mark.parametrize("n,k", [(8200, 160), (16400, 672), (96, 8192), (40, 16500), (8208, 8320)])
def test_few_rows_of_wide_and_long_matrices(m, n, k):
    w, wv = _weight(n, k, n + k)
    x, av = _given(m, k, m)
    y = (torch.from_numpy(av) @ torch.from_numpy(wv).T).numpy()
    size = (torch.from_numpy(np.abs(av)) @ torch.from_numpy(np.abs(wv)).T).numpy()
    tol = 2.0 ** -23 * (128 + -(-k // 128) + 12) * size + 2.0 ** -22 * np.abs(y) + 2.0 ** -8 * np.abs(y)
    a = ie.Mx4Matrix(m, k)
    a.quantize(to_dev(x))
    for way in [a] + ([to_dev(x)] if m <= 16 and k % 8 == 0 else []):
        out = torch.full((m + 1, n), 7.0, dtype=BF, device=DEV)
        w.product(way, out[:m])
        sync()
        assert (np.abs(f64(out[:m]) - y) <= tol).all() and (out[m:] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_matrices_are_their_parts(dtype):
    """More than the last cache keeps (non-temporal reads and writes) against the same rows a few at a time; short and
    unaligned rows as well."""
    rows, k = (6303, 8200) if dtype is BF else (3101, 8200)
    g = torch.Generator(device=DEV).manual_seed(5)
    wide = torch.randn((rows, k + 9), generator=g, device=DEV).to(dtype)
    for first, cols in ((0, k), (1, k)):
        x = wide[:, first:first + cols]
        if first == 0:
            x = x.contiguous()
        a, part = ie.Mx4Matrix(rows, cols), ie.Mx4Matrix(800, cols)
        a.quantize(x)
        outs = [torch.empty(rows, cols, dtype=t, device=DEV) for t in (BF, F32)]
        for out in outs:
            a.values(out)
        small = torch.empty(800, cols, dtype=BF, device=DEV)
        for at in range(0, rows, 800):
            n = min(800, rows - at)
            part.quantize(x[at:at + n])
            part.values(small[:n])
            assert torch.equal(outs[0][at:at + n], small[:n]) and torch.equal(outs[1][at:at + n], small[:n].float())
            if n == 800:
                size = part.packed.numel()
                assert torch.equal(a.packed[at // 800 * size:][:size], part.packed)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_more_than_32_bits_apart(dtype):
    k, stride = 1000, (1 << 31) + 8
    x = torch.empty(2 * stride if dtype is BF else stride + k, dtype=dtype, device=DEV)
    x = x.as_strided((3, k) if dtype is BF else (2, k), (stride - 500 if dtype is BF else stride, 1))
    rows = torch.randn(x.shape, generator=torch.Generator().manual_seed(1)).to(dtype)
    x.copy_(rows)
    a = ie.Mx4Matrix(len(x), k)
    a.quantize(x)
    x.zero_()
    a.values(x)
    sync()
    codes, scales = X.quantize(f64(rows))
    assert _same(f64(x.cpu()), X.values(codes, scales)[:, :k])


@pytest.mark.parametrize("m", [3, 16, 24, 70, 300])
def test_a_weight_of_more_than_32_bits(m):
    """4.5 GB of a repeated tile with another one at the end."""
    n, k = (1 << 20) - 5, 8192
    w, tile, last = ie.Mx4Matrix(n, k), ie.Mx4Matrix(16, k), ie.Mx4Matrix(11, k)
    g = torch.Generator(device=DEV).manual_seed(2)
    tile.quantize(torch.randn(16, k, generator=g, device=DEV))
    last.quantize(torch.randn(11, k, generator=g, device=DEV))
    size = tile.packed.numel()
    w.packed.view(-1, size)[:] = tile.packed
    w.packed[-size:] = last.packed
    x = torch.randn(m, k, generator=g, device=DEV).to(BF)
    a = ie.Mx4Matrix(m, k)
    a.quantize(x)
    out = torch.empty(m, n, dtype=BF, device=DEV)
    few = [torch.empty(m, 16, dtype=BF, device=DEV), torch.empty(m, 11, dtype=BF, device=DEV)]
    for way in [a] + [x] * (m <= 16):
        out.zero_()
        w.product(way, out)
        tile.product(way, few[0])
        last.product(way, few[1])
        sync()
        # another split of K may round otherwise: half a step of the result and the sums' order
        for got, want, terms in ((out[:, :16], few[0], tile), (out[:, -27:-11], few[0], tile), (out[:, -11:], few[1], last)):
            wv, av = (torch.empty(t.rows, k, device=DEV) for t in (terms, a))
            terms.values(wv)
            a.values(av)
            sync()
            y = f64(av) @ f64(wv).T
            assert (np.abs(f64(got) - y) <= X.product_tolerance(f64(av), f64(wv), y, k, False)).all()
            assert (np.abs(f64(want) - y) <= X.product_tolerance(f64(av), f64(wv), y, k, False)).all()
