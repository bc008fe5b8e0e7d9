"""A paged cache in microscaled 4 bits on the GPU (append, read, attention), reading back the other kinds, and capped and
distance-lowered scores over all of them, against plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import mx4_util as X
from tests import paged_util as P
from tests.gpu_util import DEV, f64, sync, to_dev

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _pool(kind, x, written, scales=None):
    """A pool's tensor (on the GPU) with x [pages, place, head, column] fp32 where `written` [pages, place], any bits (NaN in bf16
    and e4m3 and as a scale in 4 bits) elsewhere, and the fp64 values that it stands for; which: "k" or "v"."""
    which, kind = kind
    w = torch.from_numpy(written)[..., None, None]
    if kind == "mx4":
        codes, s = X.quantize(x.double().numpy())
        vals = X.values(codes, s)
        codes[~written], s[~written] = 15, 255
        return torch.from_numpy((X.k_pages if which == "k" else X.v_pages)(codes, s)).to(DEV), vals
    if kind == "bf16":
        b = x.to(BF)
        return P.to_pages(torch.where(w, b, math.nan), which, 8).to(DEV), f64(b)
    b = (x / scales.view(1, 1, -1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn)
    vals = b.double().numpy() * scales.double().numpy()[None, None, :, None]
    raw = torch.where(w, b.view(torch.uint8), torch.tensor(0x7F, dtype=torch.uint8))
    return P.to_pages(raw, which, 16).view(torch.float8_e4m3fn).to(DEV), vals


def _case(kind, batch, heads, kv, dim, page, lens, seed, cols=None, q_std=2.0, gap=0):
    g = torch.Generator().manual_seed(seed)
    held = [-(-max(n, 0) // page) for n in lens]
    cols = cols or max(max(held), 1)
    held = [min(h, cols) for h in held]
    pages = sum(held) + 3
    order = torch.randperm(pages, generator=g).int().numpy()
    table, at = np.full((batch, cols), -1, np.int32), 0
    written = np.zeros((pages, page), bool)
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
        pos = np.arange(min(max(lens[b], 0), cols * page))
        written[table[b][pos // page], pos % page] = True
    scales = [0.01 + 0.02 * torch.rand(kv, generator=g) for _ in range(2)]
    xs = [torch.randn(pages, page, kv, dim, generator=g) * torch.exp(0.5 * torch.randn(pages, page, kv, 1, generator=g)) for _ in range(2)]
    (k, kk), (v, vv) = (_pool((w, kind), x, written, s) for w, x, s in zip("kv", xs, scales))
    cache = ie.PagedCache(k, v, *([s.to(DEV) for s in scales] if kind == "e4m3" else []))
    q = (q_std * torch.randn(batch, heads * dim + gap, generator=g)).to(BF)
    qd = q.to(DEV)[:, :heads * dim].unflatten(1, (heads, dim))
    ops = dict(cache=cache, q=qd, table=torch.from_numpy(table).to(DEV), lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
               out=torch.full((batch + 1, heads, dim), 5.0, dtype=BF, device=DEV))
    return ops, (f64(q[:, :heads * dim].unflatten(1, (heads, dim))), kk, vv, table, lens)


def _attend(ops, **kw):
    c, batch, heads = ops["cache"], len(ops["lens"]), ops["q"].shape[1]
    ws = c.workspace(batch, heads, ops["table"].shape[1])
    ws.fill_(0xFF)
    c.attention(ops["q"], ops["table"], ops["lens"], ops["out"][:batch], ws, **kw)
    sync()
    assert (ops["out"][batch:] == 5.0).all()
    return ops["out"][:batch]


def _check(kind, ops, plain, cap=0.0, slopes=None, scale=None):
    q, k, v, table, lens = plain
    sd = None if slopes is None else slopes.to(DEV)
    got = f64(_attend(ops, cap=cap, slopes=sd, scale=scale))
    ref, mag, err = X.scored_attention(q, k, v, table, lens, q.shape[2] ** -0.5 if scale is None else scale, cap,
                                       None if slopes is None else f64(slopes), kind != "mx4")
    tol = X.scored_tolerance(ref, mag, err, max(max(lens), 1))
    bad = np.abs(got - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:5], (np.abs(got - ref) / tol).max())


SHAPES = [(12, 12, 64, 16), (16, 4, 64, 32), (8, 1, 128, 16), (40, 2, 128, 64), (6, 2, 128, 256), (4, 4, 64, 128)]


@pytest.mark.parametrize("heads,kv,dim,page", SHAPES)
@pytest.mark.parametrize("lens", [[1, 0, 15, 16, 17, 31, 33], [300, 512, 513, 1], [5000, 7, 2049]])
def test_attention_in_4_bits(heads, kv, dim, page, lens):
    ops, plain = _case("mx4", len(lens), heads, kv, dim, page, lens, heads * 100 + len(lens), gap=8)
    _check("mx4", ops, plain)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv,dim,page", [(12, 12, 64, 16), (28, 4, 128, 16), (34, 2, 64, 64)])
@pytest.mark.parametrize("cap,slope", [(20.0, 0.0), (0.0, 0.3), (5.0, 0.02), (1000.0, 1.0), (0.5, 0.0)])
def test_scores_capped_and_lowered(kind, heads, kv, dim, page, cap, slope):
    lens = [1, 0, 40, 517, 3000]
    ops, plain = _case(kind, len(lens), heads, kv, dim, page, lens, heads + int(cap), q_std=3.0)
    _check(kind, ops, plain, cap, slope * 2.0 ** -torch.linspace(0, 8, heads) if slope else None)


@pytest.mark.parametrize("kind", ["mx4", "bf16"])
def test_many_short_requests(kind):
    lens = [(i * 37) % 61 for i in range(1030)]      # more than 4096 rows: the small workgroups
    ops, plain = _case(kind, len(lens), 4, 4, 64, 16, lens, 3)
    _check(kind, ops, plain, 10.0 if kind == "bf16" else 0.0, torch.full((4,), 0.1) if kind == "bf16" else None)


def test_no_cap_and_no_slopes_are_the_plain_call():
    for kind in ("mx4", "bf16", "e4m3"):
        ops, _ = _case(kind, 3, 8, 2, 128, 16, [700, 3, 60], 5)
        want = _attend(ops).clone()
        assert torch.equal(_attend(ops, cap=0.0, slopes=torch.zeros(8, device=DEV)), want)


def test_pages_outside_the_pool_and_lengths_outside_the_table():
    ops, plain = _case("mx4", 4, 8, 2, 64, 16, [200, 90, 70, 40], 9)
    q, k, v, table, _ = plain
    table[0, 3], table[0, 7], table[1, 0] = -1, k.shape[0], 2 ** 31 - 1
    table[2, :] = -5
    lens = [100000, 90, 70, -3]
    # the first request's table is 13 pages long, the length beyond it is cut; the places behind its 200th token hold NaN
    lens[0] = 200
    ops["table"], ops["lens"] = to_dev(torch.from_numpy(table)), torch.tensor(lens, dtype=torch.int32, device=DEV)
    plain = (q, k, v, table, lens)
    _check("mx4", ops, plain)
    assert (ops["out"][2:4] == 0).all()
    ops, plain = _case("mx4", 1, 8, 2, 64, 16, [208], 9)
    ops["lens"][0] = 2 ** 31 - 1
    _check("mx4", ops, plain)


def test_blocks_that_are_not_numbers():
    """A NaN block of a key makes its head's rows NaN, one of a value its columns; neither where the token is past the end."""
    lens = [50, 50]
    ops, plain = _case("mx4", 2, 4, 2, 128, 16, lens, 4)
    c, table = ops["cache"], plain[3]
    kb, vb = ops["cache"].k, ops["cache"].v
    p, place = int(table[0, 2]), 3                   # token 35 of the first request
    kb[p, 1, 16].view(-1)[2 * 16 + place] = 255      # key head 1, columns 64 to 95
    out = _attend(ops).clone()
    assert torch.isnan(out[0, 2:]).all() and not torch.isnan(out[0, :2]).any() and not torch.isnan(out[1]).any()
    kb[p, 1, 16].view(-1)[2 * 16 + place] = 127
    vb[p, 0, 16].view(-1)[(place // 4 * 4 + 1) * 4 + place % 4] = 255      # value head 0, columns 32 to 63
    out = _attend(ops).clone()
    nan = torch.isnan(out[0])
    assert nan[:2, 32:64].all() and int(nan.sum()) == 64 and not torch.isnan(out[1]).any()
    ops["lens"][0] = 35
    assert not torch.isnan(_attend(ops)).any()
    ops["lens"][0] = 50
    vb[p, 0, 16].view(-1)[(place // 4 * 4 + 1) * 4 + place % 4] = 127
    ops["q"][1, 3, 77] = math.inf
    out = _attend(ops)
    assert torch.isnan(out[1, 3]).all() and not torch.isnan(out[1, :3]).any() and not torch.isnan(out[0]).any()


@pytest.mark.parametrize("dim", [64, 128])
def test_queries_of_any_size(dim):
    """Elements far below their block's largest, zero rows, the smallest and the largest exponents."""
    ops, plain = _case("mx4", 6, 4, 2, dim, 16, [60] * 6, 8)
    q = ops["q"].clone()
    q[0] *= torch.exp2(-torch.arange(dim, device=DEV) % 24.0).to(BF)
    q[1] = 0.0
    q[2] *= 2.0 ** -120
    q[3] *= 2.0 ** -133
    q[4] *= 2.0 ** 60
    q[5, :, ::3] = -0.0
    ops["q"] = q
    scales = [dim ** -0.5, dim ** -0.5, 2.0 ** 120, 2.0 ** 126, 2.0 ** -62, dim ** -0.5]
    for b, scale in enumerate(scales):
        one = dict(ops, q=q[b:b + 1], table=ops["table"][b:b + 1], lens=ops["lens"][b:b + 1], out=ops["out"][b:b + 2].clone().fill_(5.0))
        _check("mx4", one, (f64(q[b:b + 1]), plain[1], plain[2], plain[3][b:b + 1], plain[4][b:b + 1]), scale=scale)


# ------------------------------------------------------------------------------------ append and read
def _empty(kind, pages, page, kv, dim, g):
    scales = [(0.01 + 0.02 * torch.rand(kv, generator=g)).to(DEV) for _ in range(2)] if kind == "e4m3" else [None, None]
    return ie.PagedCache.empty(pages, page, kv, dim, *scales, mx4=kind == "mx4")


@pytest.mark.parametrize("kv,dim,page", [(1, 64, 16), (4, 128, 16), (3, 64, 32), (8, 128, 256)])
@pytest.mark.parametrize("tokens", [1, 7, 50, 333])
def test_append_in_4_bits(kv, dim, page, tokens):
    g = torch.Generator().manual_seed(tokens + dim)
    pages = tokens // page + 6
    c = _empty("mx4", pages, page, kv, dim, g)
    c.k.copy_(torch.randint(0, 256, c.k.shape, generator=g, dtype=torch.uint8))
    c.v.copy_(torch.randint(0, 256, c.v.shape, generator=g, dtype=torch.uint8))
    before = [x.cpu().numpy() for x in (c.k, c.v)]
    rows = torch.randn(tokens, 3 * kv * dim, generator=g).to(BF)
    rows[tokens // 2, 5] = math.inf
    rows[0, kv * dim + 33] = math.nan
    rows[tokens - 1, :32] = 0.0
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    slots[::9] = torch.tensor([-1, pages * page, 2 ** 40, -2 ** 50])[torch.arange(len(slots[::9])) % 4]
    slots[tokens // 2] = 5 if tokens > 1 else slots[0]
    slots[slots == 5] = -1
    slots[tokens // 2] = 5
    d = rows.to(DEV)
    c.append(d[:, :kv * dim], d[:, kv * dim:2 * kv * dim], slots.to(DEV))
    sync()
    for which, x, old, got in (("k", rows[:, :kv * dim], before[0], c.k), ("v", rows[:, kv * dim:2 * kv * dim], before[1], c.v)):
        codes, scales = X.quantize(f64(x).reshape(tokens, kv, dim))
        want = _insert(which, old, codes, scales, slots.numpy(), page)
        np.testing.assert_array_equal(got.cpu().numpy(), want)


def _insert(which, pool, codes, scales, slots, page):
    p, h = pool.shape[:2]
    flat = pool.copy().reshape(p, h, 17, -1)
    d = codes.shape[2]
    b = X.pairs(codes)
    c, s = flat[:, :, :16].reshape(p, h, -1).copy(), flat[:, :, 16].copy()
    c = c.reshape(p, h, d // 32, page, 16) if which == "k" else c.reshape(p, h, page // 4, d // 8, 4, 4)
    s = s.reshape(p, h, d // 32, page) if which == "k" else s.reshape(p, h, page // 4, d // 32, 4)
    for t, slot in enumerate(slots):
        if not 0 <= slot < p * page:
            continue
        i, j = divmod(int(slot), page)
        if which == "k":
            c[i, :, :, j], s[i, :, :, j] = b[t].reshape(h, d // 32, 16), scales[t]
        else:
            c[i, :, j // 4, :, j % 4], s[i, :, j // 4, :, j % 4] = b[t].reshape(h, d // 8, 4), scales[t]
    return np.concatenate([c.reshape(p, h, 16, -1), s.reshape(p, h, 1, -1)], 2).reshape(pool.shape)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "e4m3"])
@pytest.mark.parametrize("kv,dim,page", [(1, 64, 16), (4, 128, 32), (2, 128, 256)])
def test_read(kind, kv, dim, page):
    g = torch.Generator().manual_seed(dim + page)
    tokens = 70
    c = _empty(kind, 12, page, kv, dim, g)
    k, v = (3.0 * torch.randn(tokens, kv, dim, generator=g).to(BF) for _ in range(2))
    slots = torch.randperm(12 * page, generator=g)[:tokens].to(DEV)
    c.append(to_dev(k), to_dev(v), slots)
    pick = torch.randint(0, tokens, (99,), generator=g)
    reads = slots.cpu()[pick].to(DEV)
    reads[5], reads[6], reads[7] = -1, 12 * page, 2 ** 45
    wide = torch.full((100, 2 * kv * dim + 16), 7.0, dtype=BF, device=DEV)
    ko, vo = wide[:99, :kv * dim].unflatten(1, (kv, dim)), wide[:99, kv * dim + 8:2 * kv * dim + 8].unflatten(1, (kv, dim))
    c.read(reads, ko, vo)
    sync()
    for x, got, scale in ((k, ko, c.k_scale), (v, vo, c.v_scale)):
        if kind == "mx4":
            want = X.values(*X.quantize(f64(x)))
        elif kind == "bf16":
            want = f64(x)
        else:
            s = scale.cpu().view(1, -1, 1)
            want = f64(((x.float() / s).clamp(-448, 448).to(torch.float8_e4m3fn).float() * s).to(BF))
        want = want[pick.numpy()]
        want[5:8] = 0.0
        np.testing.assert_array_equal(f64(got), want)
    assert (wide[99] == 7.0).all() and (wide[:, 2 * kv * dim + 8:] == 7.0).all() and (wide[:, kv * dim:kv * dim + 8] == 7.0).all()


def test_no_tokens():
    c = _empty("mx4", 3, 16, 2, 64, torch.Generator())
    none = torch.empty(0, 2, 64, dtype=BF, device=DEV)
    c.append(none, none, torch.empty(0, dtype=torch.int64, device=DEV))
    c.read(torch.empty(0, dtype=torch.int64, device=DEV), none, none)
    sync()


def test_offsets_beyond_32_bits():
    # 2 x 5.85 GB; the tokens go to the first and the last pages
    page, heads, dim, pages = 64, 8, 128, 168000
    c = ie.PagedCache.empty(pages, page, heads, dim, mx4=True)
    table = torch.tensor([[pages - 1, 0, pages - 2, 133333]], dtype=torch.int32)
    n = 4 * page - 5
    pos = torch.arange(n)
    slots = (table[0, pos // page].long() * page + pos % page).to(DEV)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(n, heads, dim, generator=g).to(BF) for _ in range(2))
    q = torch.randn(1, heads, dim, generator=g).to(BF)
    c.append(k.to(DEV), v.to(DEV), slots)
    out, back = torch.empty(1, heads, dim, dtype=BF, device=DEV), [torch.empty(n, heads, dim, dtype=BF, device=DEV) for _ in range(2)]
    c.attention(q.to(DEV), table.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV), out, c.workspace(1, heads, 4))
    c.read(slots, *back)
    sync()
    dense = [X.values(*X.quantize(f64(x))) for x in (k, v)]
    for x, y in zip(back, dense):
        np.testing.assert_array_equal(f64(x), y)
    padded = [np.concatenate([x, np.zeros((5, heads, dim))]).reshape(4, page, heads, dim) for x in dense]
    ref, mag, err = X.scored_attention(f64(q), *padded, np.arange(4)[None], [n], dim ** -0.5, q_exact=False)
    assert (np.abs(f64(out) - ref) <= X.scored_tolerance(ref, mag, err, n)).all()


def test_a_result_depends_on_no_other_request():
    lens = [700, 3, 0, 5000, 256, 900] * 4
    ops, _ = _case("mx4", len(lens), 8, 2, 128, 16, lens, 9)
    slopes = torch.linspace(0.01, 0.2, 8, device=DEV)
    kw = dict(cap=30.0, slopes=slopes)
    full = _attend(ops, **kw).clone()
    keep = torch.arange(len(lens), device=DEV) % 3 == 0
    assert torch.equal(_attend(dict(ops, lens=torch.where(keep, ops["lens"], 0)), **kw)[keep], full[keep])
    order = torch.randperm(len(lens), generator=torch.Generator().manual_seed(1)).to(DEV)
    assert torch.equal(_attend(dict(ops, q=ops["q"][order], table=ops["table"][order], lens=ops["lens"][order]), **kw), full[order])


def test_refusals_of_the_binding():
    ops, _ = _case("mx4", 2, 4, 2, 64, 16, [300, 30], 13)
    c = ops["cache"]
    ws = c.workspace(2, 4, ops["table"].shape[1])
    out = ops["out"][:2]
    for kw in (dict(slopes=torch.ones(4)), dict(slopes=torch.ones(3, device=DEV)), dict(slopes=torch.ones(4, device=DEV).half())):
        with pytest.raises(ValueError):
            c.attention(ops["q"], ops["table"], ops["lens"], out, ws, **kw)
    for cap in (-1.0, math.nan, math.inf, 1e-20, 1e20):
        with pytest.raises(ie.IefwdError) as e:
            c.attention(ops["q"], ops["table"], ops["lens"], out, ws, cap=cap)
        assert e.value.status == ie.EINVAL
    for k, v in ((c.k[:, :, :16], c.v), (c.k, c.v[:, :, :16]), (c.k, c.v.view(torch.int8)), (c.k, c.v[:1])):
        with pytest.raises(ValueError):
            ie.PagedCache(k, v)
    with pytest.raises(ValueError):
        ie.PagedCache(c.k, c.v, torch.ones(2, device=DEV), torch.ones(2, device=DEV))
    with pytest.raises(ValueError):
        ie.PagedCache.empty(3, 18, 2, 64, mx4=True)
    k = torch.zeros(3, 2, 64, dtype=BF, device=DEV)
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    for b in (dict(k=k.half()), dict(k=k[:2]), dict(v=k.transpose(1, 2)), dict(slots=slots.int()), dict(slots=slots[::2])):
        with pytest.raises(ValueError):
            c.read(**dict(dict(k=k, v=k, slots=slots), **b))
    sync()
    assert (out == 5.0).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_many_tokens_are_their_parts(dim):
    """More than the last cache keeps of (non-temporal reads and writes) against the same tokens in parts."""
    kv, page, tokens = 2048 // dim, 32, 16501
    pages = tokens // page + 2
    g = torch.Generator(device=DEV).manual_seed(dim)
    k, v = (torch.randn(tokens, kv, dim, generator=g, device=DEV).to(BF) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens]
    caches = [ie.PagedCache.empty(pages, page, kv, dim, mx4=True) for _ in range(2)]
    for c in caches:
        c.k.fill_(7)
        c.v.fill_(7)
    caches[0].append(k, v, slots)
    out = [torch.empty_like(k) for _ in range(4)]
    caches[0].read(slots, *out[:2])
    for at in range(0, tokens, 3001):
        some = slice(at, at + 3001)
        caches[1].append(k[some], v[some], slots[some])
        caches[1].read(slots[some], out[2][some], out[3][some])
    sync()
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
