"""The paged cache's operators on the GPU against plain 64-bit implementations: planning, append, attention, and a
run of them together as a server generates tokens."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import paged_util as P
from tests.gpu_util import DEV, f64, sync

pytestmark = pytest.mark.gpu

NAN8, NAN16 = 0x7F, 0x7FC0


# ------------------------------------------------------------------------------------ plan
def _plan_inputs(rng, page, lens, new, columns, ring_size, free, head, stride=None):
    """A consistent state: the pages held by the requests and `free` others in the ring from `head` on."""
    lens, new = np.array(lens, np.int32), np.array(new, np.int32)
    order = rng.permutation(ring_size).astype(np.int32)
    table = np.full((len(lens), columns), -7, np.int32)
    used = 0
    for b, o in enumerate(lens):
        if 0 <= o <= columns * page:
            held = -(-int(o) // page)
            table[b, :held] = order[used:used + held]
            used += held
    assert used + free <= ring_size
    ring = np.full(ring_size, -9, np.int32)
    ring[(head + np.arange(free)) % ring_size] = order[used:used + free]
    return lens, new, table, ring, np.array([head, head + free], np.int64)


def _run_plan(page, lens, new, table, ring, counters, room, stride=None, stream=None):
    stride = stride or table.shape[1]
    wide = torch.full((len(lens), stride), 55, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = torch.from_numpy(table)
    d = {k: torch.from_numpy(v.copy()).to(DEV) for k, v in dict(lens=lens, new=new, ring=ring, counters=counters).items()}
    lens_out, counters_out = torch.full_like(d["lens"], -5), torch.full_like(d["counters"], -5)
    slots = torch.full((room + 3,), -5, dtype=torch.int64, device=DEV)
    starts = torch.full((len(lens) + 2,), -5, dtype=torch.int32, device=DEV)
    refused = torch.full((2,), -5, dtype=torch.int32, device=DEV)
    ie.paged_plan(page, d["lens"], d["new"], wide[:, :table.shape[1]], d["ring"], d["counters"], lens_out, counters_out,
                  slots[:room], starts[:-1], refused[:1], stream=stream)
    sync()
    assert (wide[:, table.shape[1]:] == 55).all() and (slots[room:] == -5).all()
    assert starts[-1] == -5 and refused[1] == -5
    got = dict(table=wide[:, :table.shape[1]], ring=d["ring"], counters_out=counters_out, lens_out=lens_out,
               slots=slots[:room], starts=starts[:-1], refused=refused[:1])
    return {k: v.cpu().numpy() for k, v in got.items()}


def _check_plan(page, state, room, **kw):
    want = P.plan(page, *state, room)
    got = _run_plan(page, *state, room, **kw)
    for k, v in want.items():
        np.testing.assert_array_equal(got[k], v, err_msg=k)
    return want


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("case", ["one_token", "grow_all", "ends", "few_pages", "few_slots", "nothing", "bad_lengths"])
def test_plan(page, case):
    rng = np.random.default_rng(page * 7 + len(case))
    columns, batch = 9, 37
    cap = columns * page
    lens = rng.integers(0, cap - 5, batch)
    lens[:4] = [0, page, page - 1, cap]
    new = np.minimum(lens + 1, cap)
    room, free = 60, 200
    if case == "grow_all":
        new, room, free = rng.integers(lens, cap + 1), 40 * cap, 400
    elif case == "ends":
        new[rng.random(batch) < 0.4] = 0
        new[5] = lens[5] // 2          # cut back, not ended
    elif case == "few_pages":
        new, room, free = rng.integers(lens, cap + 1), 40 * cap, 60
    elif case == "few_slots":
        new, room, free = rng.integers(lens, cap + 1), 10 * page + 3, 400
    elif case == "nothing":
        new, free = lens.copy(), 0
    elif case == "bad_lengths":
        new[3], lens[7], new[9], lens[11] = cap + 1, -1, -2, cap + 9
    for head in (0, 795, 10 ** 12 + 7):
        state = _plan_inputs(rng, page, lens, new, columns, 800, free, head)
        want = _check_plan(page, state, room, stride=columns + 3)
    assert (want["refused"][0] > 0) == (case in ("few_pages", "few_slots", "bad_lengths"))


@pytest.mark.parametrize("batch", [1, 2, 63, 255, 256, 257, 1000, 4096])
def test_plan_batches(batch):
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 100, batch)
    new = np.where(rng.random(batch) < 0.1, 0, lens + rng.integers(0, 28, batch))
    state = _plan_inputs(rng, 16, lens, new, 8, 9 * batch + 5, batch, 3)
    _check_plan(16, state, int(np.maximum(new - lens, 0).sum()) + 2)


def test_plan_one_long_prompt_and_no_slots():
    rng = np.random.default_rng(1)
    state = _plan_inputs(rng, 16, [3, 0, 5000], [3, 70001, 5001], 4400, 6000, 4500, 5990)
    _check_plan(16, state, 70002)
    state = _plan_inputs(rng, 16, [30, 500], [0, 499], 40, 200, 3, 5)       # only gives pages back
    want = P.plan(16, *state, 0)
    d = [torch.from_numpy(x).to(DEV) for x in state]
    out = [torch.empty_like(d[0]), torch.empty_like(d[4]), torch.empty(0, dtype=torch.int64, device=DEV),
           torch.empty(3, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)]
    ie.paged_plan(16, *d, *out)
    sync()
    np.testing.assert_array_equal(d[3].cpu().numpy(), want["ring"])
    np.testing.assert_array_equal(out[1].cpu().numpy(), want["counters_out"])


@pytest.mark.parametrize("counters", [[5, 3], [-4, 2], [0, 801]])
def test_plan_of_broken_counters_hands_out_nothing(counters):
    rng = np.random.default_rng(5)
    state = list(_plan_inputs(rng, 16, [3, 40, 0], [4, 0, 90], 8, 800, 100, 0))
    state[4] = np.array(counters, np.int64)
    want = _check_plan(16, state, 200)
    assert want["refused"][0] == 2       # the one that stays within its page is served


# ------------------------------------------------------------------------------------ append
def _cache(kind, pages, page, heads, dim, g, fill="random"):
    scales = [None, None]
    if kind == "e4m3":
        scales = [(0.5 + torch.rand(heads, generator=g)).mul(0.03).to(DEV) for _ in range(2)]
    c = ie.PagedCache.empty(pages, page, heads, dim, *scales)
    for t in (c.k, c.v):
        raw = t.view(torch.uint8)
        raw.copy_(torch.randint(0, 256, raw.shape, generator=g, dtype=torch.uint8))
        if fill == "nan":
            t.view(torch.int16 if kind == "bf16" else torch.uint8).fill_(NAN16 if kind == "bf16" else NAN8)
    return c


def _places(c):
    """The cache's contents as [page, place, head, column] bit patterns on the host."""
    raw = torch.int16 if c.k.dtype == torch.bfloat16 else torch.uint8
    return [P.from_pages(t.view(raw).cpu(), n) for t, n in ((c.k, "k"), (c.v, "v"))]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,dim,page,tokens,stride", [(1, 64, 16, 1, 0), (8, 128, 16, 33, 24), (3, 64, 64, 500, 8),
                                                          (2, 128, 256, 1203, 0), (16, 64, 32, 70, 512),
                                                          (16, 128, 16, 9001, 8)])
def test_append(kind, heads, dim, page, tokens, stride):
    g = torch.Generator().manual_seed(tokens)
    pages = tokens // page + 12
    c = _cache(kind, pages, page, heads, dim, g)
    before = _places(c)
    # runs of following places, single tokens, a gap, tokens of a padded batch, slots outside the pool
    slots, free, at = [], torch.randperm(pages, generator=g).tolist(), 0
    while len(slots) < tokens:
        p = free.pop()
        n = int(torch.randint(1, page + 1, (1,), generator=g))
        first = int(torch.randint(0, page - n + 1, (1,), generator=g))
        slots += [p * page + first + i for i in range(n)]
        if not free:
            break
    slots = (slots + [-1] * tokens)[:tokens]
    for i in range(0, tokens, 11):
        slots[i] = [-1, pages * page, -2 ** 40, 2 ** 40][i // 11 % 4]
    width = heads * dim
    rows = torch.randn(tokens, 2 * width + stride, generator=g).bfloat16()
    flat = rows.view(-1)
    flat[::97] = torch.tensor([1e30, -1e30, float("inf"), float("-inf"), float("nan"), 0.0, -0.0, 1e-4]).bfloat16().repeat(
        len(flat[::97]) // 8 + 1)[:len(flat[::97])]
    dev = rows.to(DEV)
    k, v = dev[:, :width], dev[:, width + stride:]
    c.append(k.unflatten(1, (heads, dim)), v, torch.tensor(slots).to(DEV))
    sync()
    for want, got, new, scale in zip(before, _places(c), (rows[:, :width], rows[:, width + stride:]), (c.k_scale, c.v_scale)):
        x = new.unflatten(1, (heads, dim))
        if kind == "e4m3":
            x = (x.float() / scale.cpu().view(1, -1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn)
        x = x.contiguous().view(want.dtype)
        for i, s in enumerate(slots):
            if 0 <= s < pages * page:
                want[s // page, s % page] = x[i]
        if kind == "e4m3":      # any NaN is as good as another
            want, got = (torch.where((t & 127) == 127, torch.tensor(127, dtype=torch.uint8), t) for t in (want, got))
        assert torch.equal(want, got)


def test_append_e4m3_rounds_every_bf16_value_to_the_nearest():
    x = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(-1, 1, 64)
    one = torch.ones(1, device=DEV)
    c = ie.PagedCache.empty(64, 16, 1, 64, one, one)
    slots = torch.arange(1024)
    c.append(x.to(DEV), x.to(DEV), slots.to(DEV))
    sync()
    k, v = _places(c)
    want = x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).view(64, 16, 1, 64)
    for got in (k, v):
        same = (got == want) | (((got & 127) == 127) & ((want & 127) == 127))
        assert same.all()


# ------------------------------------------------------------------------------------ attention
def _attention_case(kind, batch, heads, kv, dim, page, lens, seed, q_pad=0, extra_columns=0, bad_pages=False):
    """Returns the device call's operands and the fp64 reference; unused places hold NaN bits."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.as_tensor(lens, dtype=torch.int32)
    held = (lens.clamp(min=0) + page - 1) // page
    columns = max(1, int(held.max())) + extra_columns
    pages = int(held.sum()) + 2
    c = _cache(kind, pages, page, kv, dim, g, fill="nan")
    order = torch.randperm(pages, generator=g).int()
    table = torch.full((batch, columns), 2 ** 31 - 1, dtype=torch.int32)
    table[torch.arange(columns)[None] < held[:, None]] = order[:int(held.sum())]
    piece = 8 if kind == "bf16" else 16
    dense = []
    for t, n, scale in ((c.k, "k", c.k_scale), (c.v, "v", c.v_scale)):
        x = torch.randn(pages, page, kv, dim, generator=g)
        if kind == "e4m3":
            x = (x / scale.cpu().view(1, 1, -1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn)
        else:
            x = x.bfloat16()
        raw = torch.int16 if kind == "bf16" else torch.uint8
        bits, place = x.view(raw), torch.arange(page)
        for b in range(batch):          # only the cached tokens' places are written
            for j in range(int(held[b])):
                pid = int(table[b, j])
                bits[pid, place + j * page >= int(lens[b])] = NAN16 if kind == "bf16" else NAN8
        unused = [int(o) for o in order[int(held.sum()):]]
        bits[unused] = NAN16 if kind == "bf16" else NAN8
        t.view(raw).copy_(P.to_pages(bits, n, piece).to(DEV))
        y = x.double()
        dense.append((y * scale.cpu().double().view(1, 1, -1, 1) if kind == "e4m3" else y).numpy())
    if bad_pages:
        table[0, 0], table[-1, int(held[-1]) // 2] = -1, pages
    q = (2.5 * torch.randn(batch, heads * dim + q_pad, generator=g)).bfloat16()
    out = torch.full((batch + 1, heads, dim), 9.0, dtype=torch.bfloat16, device=DEV)
    ops = dict(cache=c, q=q.to(DEV)[:, :heads * dim], table=table.to(DEV), lens=lens.to(DEV), out=out)
    return ops, (f64(q[:, :heads * dim]).reshape(batch, heads, dim), *dense, table.numpy(), lens.numpy())


def _attend(ops, scale=None, stream=None):
    c, batch, heads = ops["cache"], ops["lens"].shape[0], ops["out"].shape[1]
    ws = c.workspace(batch, heads, ops["table"].shape[1])
    ws.fill_(0xFF)                                         # NaN in every word
    c.attention(ops["q"], ops["table"], ops["lens"], ops["out"][:batch], ws, scale, stream)
    sync()
    assert (ops["out"][batch:] == 9.0).all()
    return ops["out"][:batch]


def _check_attention(ops, ref_in, scale=None):
    got = f64(_attend(ops, scale))
    scale = ops["cache"].head_dim ** -0.5 if scale is None else scale
    ref, mag, dots = P.attention(*ref_in, scale)
    tol = P.attention_tolerance(ref, mag, dots, int(ref_in[4].max()), ops["cache"].head_dim, scale)
    assert np.isfinite(got).all()
    worst = np.max((np.abs(got - ref) - tol))
    print(f"  max error {np.abs(got - ref).max():.3e}, largest excess over the tolerance {worst:.3e}", flush=True)
    assert worst <= 0


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 127, 128, 129, 255, 256, 257, 300, 511, 513, 1000]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 64, 16), (4, 4, 128, 32), (8, 2, 128, 16), (7, 1, 64, 64), (16, 1, 128, 128),
                                               (17, 1, 64, 16), (40, 2, 128, 256), (12, 4, 64, 32), (64, 1, 128, 16)])
def test_attention_lengths(kind, heads, kv, dim, page):
    _check_attention(*_attention_case(kind, len(LENGTHS), heads, kv, dim, page, LENGTHS, heads * 31 + dim, q_pad=16,
                                      extra_columns=3))


@pytest.mark.parametrize("kind,heads,kv,dim,page,lens", [
    ("bf16", 16, 16, 64, 16, [9000, 1, 8193]),            # parts longer than 256 keys
    ("bf16", 8, 8, 128, 64, [40000]),
    ("e4m3", 4, 1, 128, 16, [131073, 3]),                 # parts longer than 1024 keys
    ("e4m3", 32, 32, 64, 128, [20001, 0, 300]),
    ("e4m3", 8, 8, 128, 64, [52000]),                     # more than the last cache is taken to hold
    ("bf16", 8, 8, 64, 32, [52000]),
    ("bf16", 24, 1, 64, 16, [70000]),                     # two tiles of query heads
    ("e4m3", 2, 1, 64, 256, [1100000]),                   # each wave's steps looked up in two rounds
    ("bf16", 64, 64, 64, 16, [2100, 513, 512, 511, 4097]),    # many rows: parts of 1024 keys
    ("bf16", 36, 36, 128, 32, [1025, 8200, 0, 31, 33, 600, 1024, 5]),
])
def test_attention_long(kind, heads, kv, dim, page, lens):
    _check_attention(*_attention_case(kind, len(lens), heads, kv, dim, page, lens, 77))


@pytest.mark.parametrize("batch", [1, 63, 64, 65, 130, 700])
def test_attention_batches(batch):
    rng = np.random.default_rng(batch)
    lens = np.where(rng.random(batch) < 0.2, 0, rng.integers(1, 900, batch))
    _check_attention(*_attention_case("bf16", batch, 4, 2, 64, 32, lens, batch))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_attention_of_thousands_of_rows(kind):
    """4096 rows and more: workgroups of 2 waves, and requests of several parts among them."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 60, 520)
    lens[[0, 77, 300, 519]] = 1100, 513, 2048, 300
    _check_attention(*_attention_case(kind, 520, 8, 8, 64, 16, lens, 21))
    _check_attention(*_attention_case(kind, 260, 16, 16, 128, 32, lens[-260:] + 60, 22))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_attention_drops_tokens_of_pages_outside_the_pool(kind):
    _check_attention(*_attention_case(kind, 4, 8, 2, 128, 16, [16, 300, 40, 700], 5, bad_pages=True))


def test_attention_cuts_lengths_and_takes_any_scale():
    ops, ref = _attention_case("bf16", 3, 4, 4, 64, 16, [48, 30, 48], 6)
    ops["lens"] = torch.tensor([10 ** 9, -3, 48], dtype=torch.int32, device=DEV)
    ref = ref[:4] + (np.array([48, 0, 48]),)
    _check_attention(ops, ref)
    _check_attention(ops, ref, scale=0.0)
    _check_attention(ops, ref, scale=-0.31)


def test_attention_of_scores_with_infinities():
    ops, ref = _attention_case("bf16", 1, 2, 2, 64, 16, [600], 8)
    c = ops["cache"]
    c.k.fill_(0)                                    # scores 0 ...
    ops["q"][:] = 1.0
    first = int(ops["table"][0, 0])
    c.k[first] = float("-inf")                      # ... and -inf on the first page, and in all of a part
    for j in range(16, 32):
        c.k[int(ops["table"][0, j])] = float("-inf")
    got = f64(_attend(ops))
    v = ref[2][ref[3][0]].reshape(-1, 2, 64)
    keep = [i for i in range(600) if not (i < 16 or 256 <= i < 512)]
    want = v[keep].mean(0)
    assert np.abs(got[0] - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-4 * np.abs(v[keep]).mean()
    c.k.fill_(float("-inf"))                        # nothing to attend to
    assert (_attend(ops) == 0).all()
    c.k.fill_(0)
    c.k[first, :, :, 3] = float("nan")
    assert torch.isnan(_attend(ops)).all()


@pytest.mark.parametrize("batch", [3, 60, 400])
def test_attention_result_depends_on_no_other_request(batch):
    lens = ([700, 3, 0, 5000, 256, 900] * batch)[:batch]
    ops, _ = _attention_case("bf16", batch, 8, 2, 128, 16, lens, 9)
    full = _attend(ops).clone()
    assert torch.equal(full, _attend(ops))
    # the others shorter, gone or in another order
    keep = torch.arange(batch, device=DEV) % 3 == 0
    assert torch.equal(_attend(dict(ops, lens=torch.where(keep, ops["lens"], ops["lens"] // 2)))[keep], full[keep])
    assert torch.equal(_attend(dict(ops, lens=torch.where(keep, ops["lens"], 0)))[keep], full[keep])
    order = torch.randperm(batch, generator=torch.Generator().manual_seed(1)).to(DEV)
    assert torch.equal(_attend(dict(ops, q=ops["q"][order], table=ops["table"][order], lens=ops["lens"][order])), full[order])
    # columns of the table that no request uses
    wide = torch.full((batch, 900), -1, dtype=torch.int32, device=DEV)
    wide[:, :ops["table"].shape[1]] = ops["table"]
    assert torch.equal(_attend(dict(ops, table=wide)), full)


def test_offsets_beyond_32_bits():
    # 2 x 5.6 GB; the tokens go to the first and the last pages, in different ones of a request
    page, heads, dim, pages = 64, 8, 128, 43000
    c = ie.PagedCache.empty(pages, page, heads, dim)
    table = torch.tensor([[pages - 1, 0, pages - 2, 33333]], dtype=torch.int32)
    n = 4 * page - 5
    pos = torch.arange(n)
    slots = table[0, pos // page].long() * page + pos % page
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(n, heads, dim, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(1, heads, dim, generator=g).bfloat16()
    c.append(k.to(DEV), v.to(DEV), slots.to(DEV))
    out = torch.empty(1, heads, dim, dtype=torch.bfloat16, device=DEV)
    c.attention(q.to(DEV), table.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV), out, c.workspace(1, heads, 4))
    sync()
    dense = [f64(x) for x in (k, v)]
    ref, mag, dots = P.attention(f64(q), *(np.concatenate([x, np.zeros((5, heads, dim))]).reshape(4, page, heads, dim) for x in dense),
                                 np.arange(4)[None], [n], dim ** -0.5)
    assert (np.abs(f64(out) - ref) <= P.attention_tolerance(ref, mag, dots, n, dim, dim ** -0.5)).all()


# ------------------------------------------------------------------------------------ together
class _Server:
    """Requests with a paged cache as a program drives it: plan, append, attend, on the device alone."""

    def __init__(self, kind, batch, heads, kv, dim, page, pages, columns, seed):
        g = torch.Generator().manual_seed(seed)
        self.c, self.heads, self.page = _cache(kind, pages, page, kv, dim, g, fill="nan"), heads, page
        z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device=DEV)  # noqa: E731
        self.lens, self.lens_out, self.new = z(batch), z(batch), z(batch)
        self.counters, self.counters_out = torch.tensor([0, pages], device=DEV), z(2, t=torch.int64)
        self.ring = torch.randperm(pages, generator=g).int().to(DEV)
        self.table = torch.full((batch, columns), -1, dtype=torch.int32, device=DEV)
        self.starts, self.refused = z(batch + 1), z(1)
        self.ws = self.c.workspace(batch, heads, columns)

    def step(self, q, k, v, slots, out, stream=None):
        ie.paged_plan(self.page, self.lens, self.new, self.table, self.ring, self.counters, self.lens_out, self.counters_out,
                      slots, self.starts, self.refused, stream=stream)
        self.c.append(k, v, slots, stream=stream)
        self.c.attention(q, self.table, self.lens_out, out, self.ws, stream=stream)

    def swap(self):
        self.lens.copy_(self.lens_out)
        self.counters.copy_(self.counters_out)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_requests_come_grow_and_end(kind):
    batch, heads, kv, dim, page = 6, 6, 2, 64, 16
    s = _Server(kind, batch, heads, kv, dim, page, 60, 20, 4)
    g = torch.Generator().manual_seed(8)
    want = [[] for _ in range(batch)]                # each request's (k, v) by token
    script = [[5, 0, 33, 0, 1, 0], [6, 17, 34, 0, 2, 0], [7, 18, 0, 300, 3, 0], [8, 19, 0, 301, 4, 90], [9, 0, 50, 302, 0, 91],
              [10, 3, 51, 303, 64, 92], [0, 4, 52, 900, 65, 93], [1, 5, 53, 304, 66, 0], [2, 6, 54, 320, 67, 1]]
    seen_refusal = False
    for new in script:
        old = [len(w) for w in want]
        grow = [max(0, n - o) for n, o in zip(new, old)]
        total, room = sum(grow), sum(grow) + 3
        k, v = (torch.randn(room, kv, dim, generator=g).bfloat16() for _ in range(2))
        q = torch.randn(batch, heads, dim, generator=g).bfloat16()
        s.new.copy_(torch.tensor(new, dtype=torch.int32))
        slots = torch.empty(room, dtype=torch.int64, device=DEV)
        out = torch.empty(batch, heads, dim, dtype=torch.bfloat16, device=DEV)
        s.step(q.to(DEV), k.to(DEV), v.to(DEV), slots, out)
        s.swap()
        sync()
        assert (slots[total:] == -1).all()
        lens = s.lens_out.tolist()
        at = 0
        for b, n in enumerate(new):
            if lens[b] != n:
                assert n == 900 and int(s.refused) == 1      # beyond the table
                seen_refusal = True
                continue
            want[b] = want[b][:n] + [(k[at + i], v[at + i]) for i in range(grow[b])]
            at += grow[b]
        used = sum(-(-n // page) for n in lens)
        assert int(s.counters[1] - s.counters[0]) == 60 - used
        for b in range(batch):
            if not want[b]:
                assert (out[b] == 0).all()
                continue
            kk, vv = (torch.stack([t[i] for t in want[b]]) for i in range(2))
            if kind == "e4m3":
                kk, vv = ((x.float() / sc.cpu().view(1, -1, 1)).to(torch.float8_e4m3fn).double() * sc.cpu().double().view(1, -1, 1)
                          for x, sc in ((kk, s.c.k_scale), (vv, s.c.v_scale)))
            n = len(want[b])
            ref, mag, dots = P.attention(f64(q[b:b + 1]), f64(kk)[None], f64(vv)[None], np.zeros((1, 1), int), [n], dim ** -0.5)
            assert (np.abs(f64(out[b:b + 1]) - ref) <= P.attention_tolerance(ref, mag, dots, n, dim, dim ** -0.5)).all()
    assert seen_refusal


def test_captured_step_follows_the_lengths():
    """A step captured once and replayed while the requests grow, against the same steps run one by one, with other work and
    waits between the replays."""
    batch, heads, kv, dim, page = 5, 8, 2, 128, 16
    a, b = (_Server("bf16", batch, heads, kv, dim, page, 400, 70, 4) for _ in range(2))
    g = torch.Generator().manual_seed(2)
    prompts = torch.tensor([250, 31, 16, 0, 1000], dtype=torch.int32)
    n = int(prompts.sum())
    pk, pv = (torch.randn(n, kv, dim, generator=g).bfloat16().to(DEV) for _ in range(2))
    pq = torch.zeros(batch, heads, dim, dtype=torch.bfloat16, device=DEV)
    for s in (a, b):
        s.new.copy_(prompts)
        s.step(pq, pk, pv, torch.empty(n, dtype=torch.int64, device=DEV), torch.empty_like(pq))
        s.swap()
    q, k, v = (torch.randn(batch, h, dim, generator=g).bfloat16().to(DEV) for h in (heads, kv, kv))
    slots = [torch.empty(batch, dtype=torch.int64, device=DEV) for _ in range(2)]
    out = [torch.zeros_like(pq) for _ in range(2)]
    add = torch.tensor([1, 1, 1, 0, 1], dtype=torch.int32, device=DEV)
    sync()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.new.copy_(a.lens + add)
        a.step(q, k, v, slots[0], out[0])
        a.swap()
    for i in range(9):
        for t, h in ((q, heads), (k, kv), (v, kv)):
            t.copy_(torch.randn(batch, h, dim, generator=g).bfloat16())
        graph.replay()
        b.new.copy_(b.lens + add)
        b.step(q, k, v, slots[1], out[1])
        b.swap()
        sync()
        for x, y in ((out[0], out[1]), (slots[0], slots[1]), (a.lens, b.lens), (a.counters, b.counters), (a.table, b.table)):
            assert torch.equal(x, y), i
    assert a.lens.tolist() == [259, 40, 25, 0, 1009]


def test_runs_on_the_current_or_given_stream():
    ops, ref = _attention_case("bf16", 2, 4, 2, 64, 16, [500, 30], 12)
    want = _attend(ops).clone()
    s = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=DEV)
    for given in (True, False):
        ops["out"][:2] = 0
        q = ops["q"].clone()
        sync()
        with torch.cuda.stream(s):
            for _ in range(20):
                busy = (busy @ busy).clamp(-1, 1)        # holds this stream back
            late = q * 1.0
            ws = ops["cache"].workspace(2, 4, ops["table"].shape[1])
            if not given:
                ops["cache"].attention(late, ops["table"], ops["lens"], ops["out"][:2], ws)
        if given:
            ops["cache"].attention(late, ops["table"], ops["lens"], ops["out"][:2], ws, stream=s)
        sync()
        assert torch.equal(ops["out"][:2], want)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_decoder_block_of_4_bit_products_over_the_cache(kind):
    """The QKV product, plan, append, attention and the out-projection with its residual, a token after the other for
    requests of different lengths; each product and context against 64 bits on the inputs that it had."""
    batch, d, heads, kv, dim, page = 5, 256, 4, 2, 64, 16
    s = _Server(kind, batch, heads, kv, dim, page, 80, 25, 6)
    g = torch.Generator().manual_seed(17)

    def weight(n, k, group):
        codes = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8)
        scales = (0.02 * (0.5 + torch.rand(n, k // group, generator=g))).bfloat16()
        w = P.q4_weight(codes.numpy(), f64(scales), None)
        return ie.Q4Weight(codes.to(DEV), scales.to(DEV)), w, f64(scales), group

    def bound(a, scales, group, y):       # as in the product's own tests
        mag = np.abs(a).reshape(len(a), -1, group).sum(-1) @ np.abs(scales).T
        return 2.0 ** -24 * (62 * (group + 4) + 16 * scales.shape[1]) * mag + 2.0 ** -22 * np.abs(y)

    qkv_w, out_w = weight((heads + 2 * kv) * dim, d, 64), weight(d, heads * dim, 128)
    bias = torch.randn((heads + 2 * kv) * dim, generator=g).bfloat16().to(DEV)
    lens = [0, 250, 16, 31, 256]                                     # prompts first, with keys and values as they come
    n = sum(lens)
    pk, pv = (torch.randn(n, kv, dim, generator=g).bfloat16().to(DEV) for _ in range(2))
    s.new.copy_(torch.tensor(lens, dtype=torch.int32))
    out = torch.empty(batch, heads * dim, dtype=torch.bfloat16, device=DEV)
    s.step(torch.zeros_like(out), pk, pv, torch.empty(n, dtype=torch.int64, device=DEV), out)
    s.swap()
    qkv = torch.empty(batch, (heads + 2 * kv) * dim, dtype=torch.bfloat16, device=DEV)
    slots = torch.empty(batch, dtype=torch.int64, device=DEV)
    x, h = torch.empty(batch, d, dtype=torch.bfloat16, device=DEV), torch.empty(batch, d, device=DEV)
    sync()

    def block():
        s.new.copy_(s.lens + 1)
        qkv_w[0].product(x, qkv, bias=bias)
        q, k, v = qkv.split([heads * dim, kv * dim, kv * dim], 1)
        s.step(q, k, v, slots, out)
        out_w[0].product(out, h, ie.EPI_BIAS_RESID_F32, resid=h)
        s.swap()

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    rounds = []
    for step in range(4):
        x.copy_(torch.randn(batch, d, generator=g).bfloat16())
        h.copy_(torch.randn(batch, d, generator=g))
        before = f64(h)
        graph.replay() if step % 2 else block()
        sync()
        y = f64(x) @ qkv_w[1].T + f64(bias)
        assert (np.abs(f64(qkv) - y) <= bound(f64(x), *qkv_w[2:], y) + 2.0 ** -8 * np.abs(y)).all()
        rounds.append(f64(qkv))
        assert s.lens.tolist() == [m + step + 1 for m in lens] and int(s.refused) == 0
        at = 0
        for b, m in enumerate(lens):
            dense = []
            for old, lo, scale in ((pk, heads * dim, s.c.k_scale), (pv, (heads + kv) * dim, s.c.v_scale)):
                t = np.concatenate([f64(old)[at:at + m]] + [r[b, lo:lo + kv * dim].reshape(1, kv, dim) for r in rounds])
                if kind == "e4m3":
                    sc = scale.cpu().view(1, -1, 1)
                    t = ((torch.from_numpy(t).float() / sc).clamp(-448, 448).to(torch.float8_e4m3fn).double() * sc.double()).numpy()
                dense.append(t[None])
            at += m
            keys = m + step + 1
            ref, mag, dots = P.attention(rounds[-1][b, :heads * dim].reshape(1, heads, dim), *dense, np.zeros((1, 1), int), [keys],
                                         dim ** -0.5)
            tol = P.attention_tolerance(ref, mag, dots, keys, dim, dim ** -0.5)
            assert (np.abs(f64(out[b]).reshape(1, heads, dim) - ref) <= tol).all()
        y = f64(out) @ out_w[1].T
        assert (np.abs(f64(h) - before - y) <= bound(f64(out), *out_w[2:], y) + 2.0 ** -23 * (np.abs(before) + np.abs(y))).all()


def test_two_calls_at_once_on_streams_of_their_own():
    ops, _ = _attention_case("bf16", 6, 8, 2, 128, 16, [5000, 40, 700, 0, 2049, 513], 31)
    want = _attend(ops).clone()
    c, streams = ops["cache"], [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros(6, 8, 128, dtype=torch.bfloat16, device=DEV) for _ in streams]
    spaces = [c.workspace(6, 8, ops["table"].shape[1]) for _ in streams]
    sync()
    for _ in range(5):
        for s, o, w in zip(streams, outs, spaces):
            c.attention(ops["q"], ops["table"], ops["lens"], o, w, stream=s)
    sync()
    assert all(torch.equal(o, want) for o in outs)


def test_the_binding_refuses_other_types_shapes_and_sizes():
    ops, _ = _attention_case("bf16", 2, 4, 2, 64, 16, [2000, 30], 13)
    c, q, table, lens = (ops[k] for k in ("cache", "q", "table", "lens"))
    out, ws = torch.full((2, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV), c.workspace(2, 4, table.shape[1])
    bad = [dict(q=q.float()), dict(q=q[:1]), dict(q=q.cpu()), dict(q=q[:, ::2]), dict(table=table.long()), dict(table=table[:1]),
           dict(table=table.t().contiguous().t()), dict(lens=lens.long()), dict(lens=lens[::2]), dict(lens=lens[:, None]),
           dict(out=out.float()), dict(out=out[:, :, ::2]), dict(out=out[:1]), dict(workspace=ws.float())]
    for b in bad:
        args = dict(dict(q=q, table=table, lens=lens, out=out, workspace=ws), **b)
        with pytest.raises(ValueError):
            c.attention(**args)
    with pytest.raises(ie.IefwdError) as e:
        c.attention(q, table, lens, out, ws[:-16])
    assert e.value.status == ie.EINVAL and "workspace" in str(e.value)
    with pytest.raises(ie.IefwdError):
        c.attention(q, table, lens, out, ws, scale=float("nan"))
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    for b in (dict(k=k.half()), dict(k=k[:2]), dict(v=k.transpose(1, 2)), dict(slots=slots.int()), dict(slots=slots[::2])):
        with pytest.raises(ValueError):
            c.append(**dict(dict(k=k, v=k, slots=slots), **b))
    with pytest.raises(ValueError):
        ie.PagedCache(c.k, c.v[:1])
    with pytest.raises(ValueError):
        ie.PagedCache(c.k, c.v, torch.ones(2, device=DEV), torch.ones(2, device=DEV))
    with pytest.raises(ValueError):
        ie.PagedCache(c.k.view(torch.float8_e4m3fn), c.v.view(torch.float8_e4m3fn))
    sync()
    assert (out == 9.0).all()
