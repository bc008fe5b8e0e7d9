"""Performance cases of libiefwd's operators for batched token generation over a paged key-value cache.

A server that generates tokens for many requests of different lengths keeps their keys and values in
pages of a common pool, and its weights in 4 bits.  Per generated token it
  - plans: takes pages from the pool for the requests that grow, gives back those of the requests that
    end, and makes the slot of every new token (``plan``);
  - appends the new tokens' keys and values to their slots (``append``);
  - attends from each request's newest token to all of its cached ones (``attend``);
  - multiplies the tokens' activations with the 4-bit matrices of the layer (``product``).
Prompts go through ``plan`` and ``append`` with many tokens per request.

Where ``own`` is false, ``run`` is the operator written out in elementary torch operations on 32-bit
numbers; where it is true, it is the library's call.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------------------------ cases
def _plan(name, batch, page, shortest, longest, grow, ending, short_pool=False):
    """`batch` requests of shortest .. longest cached tokens; one in `ending` ends (0: none), the others get 1 .. grow
    new tokens; short_pool: the pool has pages for about half of them."""
    return dict(name=name, kind="plan", batch=batch, page=page, shortest=shortest, longest=longest, grow=grow, ending=ending,
                short_pool=short_pool)


def _append(name, tokens, requests, page, kv_heads, head_dim, dtype, pages):
    return dict(name=name, kind="append", tokens=tokens, requests=requests, page=page, kv_heads=kv_heads, head_dim=head_dim,
                dtype=dtype, pages=pages)


def _attend(name, batch, heads, kv_heads, head_dim, shortest, longest, page, dtype, idle=0):
    """One query per request and head over shortest .. longest cached tokens; one in `idle` rows of the batch has none."""
    return dict(name=name, kind="attend", batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, shortest=shortest,
                longest=longest, page=page, dtype=dtype, idle=idle)


def _product(name, rows, n, k, group, zeros, epilogue):
    return dict(name=name, kind="product", rows=rows, n=n, k=k, group=group, zeros=zeros, epilogue=epilogue)


def listed():
    return [
        # one token for each of a few requests: the time of a launch
        _plan("plan_decode_small", 4, 16, 20, 900, 1, 0),
        # one token for each request of a full server, every 32nd of which has ended
        _plan("plan_decode_full", 512, 16, 30, 8000, 1, 32),
        # a burst of prompts of very different lengths, for which the pool holds too few pages
        _plan("plan_prompts", 192, 32, 1, 60, 4000, 0, True),
        # the new tokens of a decode step, a layer with 8 key-value heads
        _append("append_decode", 48, 48, 16, 8, 128, "bf16", 2048),
        # prompts of several requests, stored in 8 bits
        _append("append_prompt", 24001, 13, 32, 8, 128, "e4m3", 1024),
        # one short request of the large causal model (16 heads of 128, a key-value head each): latency
        _attend("attend_short", 1, 16, 16, 128, 300, 300, 16, "bf16"),
        # one long request with shared key-value heads: split over its length
        _attend("attend_long", 1, 32, 8, 128, 32001, 32001, 64, "bf16"),
        # a server's batch: lengths from a few tokens to thousands, 8-bit cache, unused rows of the batch
        _attend("attend_ragged", 96, 16, 4, 64, 5, 12000, 16, "e4m3", 12),
        # many long requests: the cache is as good as all of the bytes
        _attend("attend_full", 64, 32, 8, 128, 4000, 8192, 16, "bf16"),
        # one request of a small model: the output projection of width 1024
        _product("product_small", 1, 1024, 1024, 64, False, "residual"),
        # two requests of the large causal model: its up projection with bias and GELU
        _product("product_up", 2, 8192, 2048, 128, True, "gelu"),
        # sixteen requests, a wide matrix with a scale for every 32 weights
        _product("product_wide", 16, 16384, 4096, 32, True, "bias"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "product", "product"])
    page = rng.choice([16, 16, 32, 64, 128])
    if kind == "plan":
        if rng.random() < 0.5:
            c = _plan("", _log_int(rng, 1, 1024), page, 1, _log_int(rng, 50, 8000), rng.choice([1, 1, 4]), rng.choice([0, 7, 32]))
        else:
            batch = _log_int(rng, 1, 256)
            c = _plan("", batch, page, 1, 100, _log_int(rng, 20, min(8000, 400000 // batch)), 0, rng.random() < 0.3)
    elif kind == "append":
        requests = _log_int(rng, 1, 64)
        c = _append("", max(requests, _log_int(rng, 1, 24000)), requests, page, rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 128]),
                    rng.choice(["bf16", "e4m3"]), 0)
        while c["tokens"] * c["kv_heads"] * c["head_dim"] > 24000 * 1024:
            c["tokens"] = max(requests, c["tokens"] // 2)
        c["pages"] = c["tokens"] // page + 2 * requests + rng.randint(10, 500)
    elif kind == "attend":
        heads, kv_heads = rng.choice([(12, 12), (16, 16), (16, 4), (32, 8), (32, 8), (24, 8), (28, 4), (16, 1), (40, 2)])
        longest = _log_int(rng, 1, 40000)
        c = _attend("", _log_int(rng, 1, 128), heads, kv_heads, rng.choice([64, 128, 128]), rng.choice([longest, max(1, longest // 3), 1]),
                    longest, page, rng.choice(["bf16", "bf16", "e4m3"]), rng.choice([0, 0, 5]))
        while c["batch"] * longest * kv_heads * c["head_dim"] > 64 * 6000 * 1024:
            c["batch"] = max(1, c["batch"] // 2)
    else:
        group = rng.choice([32, 64, 128, 128])
        c = _product("", _log_int(rng, 1, 16), 16 * _log_int(rng, 16, 1024), group * max(1, _log_int(rng, 256, 12000) // group), group,
                     rng.random() < 0.5, rng.choice(["bias", "gelu", "residual"]))
        while c["n"] * c["k"] > 16384 * 4096:
            c["n"] = 16 * max(16, c["n"] // 32)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 131 + 29)


def _lengths(count, lo, hi):
    """`count` lengths spread over the logarithm of lo .. hi."""
    step = (math.log(hi) - math.log(lo)) / count
    return [max(lo, min(hi, int(round(math.exp(math.log(lo) + (i + 0.5) * step))))) for i in range(count)]


def _shuffled(values, g, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)[torch.randperm(len(values), generator=g, device=DEV)]


def _requests(case):
    """(cached tokens, wanted tokens) of each request of a plan, in an order that prepare shuffles."""
    old = _lengths(case["batch"], case["shortest"], case["longest"])
    more = _lengths(case["batch"], 1, case["grow"])
    more = [more[(i * 7919 + 3) % len(more)] for i in range(len(more))]   # lengths and growths in unrelated orders
    ends = [case["ending"] > 0 and i % case["ending"] == case["ending"] // 2 for i in range(len(old))]
    return [(o, 0 if e else o + m) for o, m, e in zip(old, more, ends)]


def _attended(case):
    lens = _lengths(case["batch"], case["shortest"], case["longest"])
    return [0 if case["idle"] and i % case["idle"] == 1 else n for i, n in enumerate(lens)]


def _cache_shapes(pages, page, kv_heads, head_dim, dtype):
    """Pages of keys in pieces of 16 bytes of one token, and of values in pieces of 4 tokens of one column."""
    piece = 8 if dtype == "bf16" else 16
    return (pages, kv_heads, head_dim // piece, page, piece), (pages, kv_heads, page // 4, head_dim, 4)


def _random_cache(case, pages, g):
    shapes = _cache_shapes(pages, case["page"], case["kv_heads"], case["head_dim"], case["dtype"])
    if case["dtype"] == "bf16":
        return [torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for s in shapes] + [None, None]
    scales = [0.01 + 0.02 * torch.rand(case["kv_heads"], generator=g, device=DEV) for _ in range(2)]
    parts = [torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for s in shapes]
    return [(p / s.view(1, -1, 1, 1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn) for p, s in zip(parts, scales)] + scales


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["kind"] == "plan":
        pairs = torch.tensor(_requests(case), dtype=torch.int32, device=DEV)
        pairs = pairs[torch.randperm(len(pairs), generator=g, device=DEV)]
        s["lens"], s["new_lens"] = pairs[:, 0].contiguous(), pairs[:, 1].contiguous()
        page, batch = case["page"], case["batch"]
        held = (s["lens"] + page - 1) // page
        need = ((s["new_lens"] + page - 1) // page - held).clamp(min=0)
        n_held, n_need = int(held.sum()), int(need.sum())
        free = n_need // 2 + 1 if case["short_pool"] else n_need + 100
        n_pages = n_held + free
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        width = (case["longest"] + case["grow"] + page - 1) // page + 1
        s["table"] = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        s["table"][torch.arange(width, device=DEV)[None] < held[:, None]] = order[:n_held]
        head = int(torch.randint(0, 5 * n_pages, (1,), generator=g, device=DEV))   # the ring has gone round before
        s["ring"] = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        s["ring"][(head + torch.arange(free, device=DEV)) % n_pages] = order[n_held:]
        s["counters"] = torch.tensor([head, head + free], dtype=torch.int64, device=DEV)
        new = int((s["new_lens"] - s["lens"]).clamp(min=0).sum())
        s["slots"] = torch.empty(new + new // 8, dtype=torch.int64, device=DEV)   # room for a larger batch than this one
        s["starts"] = torch.empty(batch + 1, dtype=torch.int32, device=DEV)
        s["lens_out"], s["counters_out"] = torch.empty_like(s["lens"]), torch.empty_like(s["counters"])
        s["refused"] = torch.empty(1, dtype=torch.int32, device=DEV)
    elif case["kind"] == "append":
        page, heads, width = case["page"], case["kv_heads"], case["kv_heads"] * case["head_dim"]
        s["k"], s["v"], s["k_scale"], s["v_scale"] = _random_cache(case, case["pages"], g)
        # the new tokens' rows as a projection leaves them: queries of twice the width, then keys, then values
        rows = torch.empty((case["tokens"], 4 * width), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        s["new_k"] = rows[:, 2 * width:3 * width].unflatten(1, (heads, -1))
        s["new_v"] = rows[:, 3 * width:].unflatten(1, (heads, -1))
        # requests of about equal numbers of new tokens, each beginning anywhere in a page
        cut = [case["tokens"] * i // case["requests"] for i in range(case["requests"] + 1)]
        first = torch.randint(0, page, (case["requests"],), generator=g, device=DEV).tolist()
        order = torch.randperm(case["pages"], generator=g, device=DEV)
        slots, taken = [], 0
        for r in range(case["requests"]):
            pos = first[r] + torch.arange(cut[r + 1] - cut[r], device=DEV)
            slots.append(order[taken + pos // page] * page + pos % page)
            taken += (first[r] + cut[r + 1] - cut[r] + page - 1) // page
        s["slots"] = torch.cat(slots)
    elif case["kind"] == "attend":
        page, lens = case["page"], _attended(case)
        held = [(n + page - 1) // page for n in lens]
        pages, width = sum(held) + 3, max(held)
        s["k"], s["v"], s["k_scale"], s["v_scale"] = _random_cache(case, pages, g)
        s["lens"] = _shuffled(lens, g)
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        s["table"] = torch.full((case["batch"], width), -1, dtype=torch.int32, device=DEV)
        s["table"][torch.arange(width, device=DEV)[None] < ((s["lens"] + page - 1) // page)[:, None]] = order[:sum(held)]
        # the queries as a projection leaves them, beside the keys and values; scores have a standard deviation of 2.8
        rows = torch.empty((case["batch"], (case["heads"] + 2 * case["kv_heads"]) * case["head_dim"]), device=DEV)
        rows = (2.8 * rows.normal_(generator=g)).bfloat16()
        s["q"] = rows[:, :case["heads"] * case["head_dim"]].unflatten(1, (case["heads"], -1))
        s["out"] = torch.empty((case["batch"], case["heads"], case["head_dim"]), dtype=torch.bfloat16, device=DEV)
    else:
        n, k, group = case["n"], case["k"], case["group"]
        w = torch.empty((n, k // group, group), device=DEV).normal_(std=0.02, generator=g)
        if case["zeros"]:
            lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
            s["scales"] = ((hi - lo) / 15).bfloat16()
            zeros = torch.round(-lo / s["scales"].float()).clamp(0, 15)
            s["zeros"] = zeros.to(torch.uint8)
        else:
            s["scales"], s["zeros"] = (w.abs().amax(-1) / 7.5).bfloat16(), None
            zeros = torch.full_like(w[..., 0], 8.0)
        codes = (torch.round(w / s["scales"].float()[..., None]) + zeros[..., None]).clamp(0, 15).to(torch.uint8).view(n, k)
        s["codes"] = codes[:, 0::2] | (codes[:, 1::2] << 4)
        s["a"] = torch.empty((case["rows"], k), device=DEV).normal_(generator=g).bfloat16()
        s["bias"] = torch.empty(n, device=DEV).normal_(std=0.02, generator=g).bfloat16()
        s["resid"] = torch.empty((case["rows"], n), device=DEV).normal_(generator=g) if case["epilogue"] == "residual" else None
        s["out"] = torch.empty((case["rows"], n), dtype=torch.float32 if case["epilogue"] == "residual" else torch.bfloat16, device=DEV)
    if own:   # what a program keeps from its start: the cache's handle and workspace, the weights in the library's layout
        import paper_2503_05130_amd as ie
        s["ie"] = ie
        if case["kind"] in ("append", "attend"):
            s["cache"] = ie.PagedCache(s["k"], s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        if case["kind"] == "attend":
            s["workspace"] = s["cache"].workspace(case["batch"], case["heads"], s["table"].shape[1])
        if case["kind"] == "product":
            s["weight"] = ie.Q4Weight(s["codes"], s["scales"], s["zeros"])
    return s


# ------------------------------------------------------------------------------------ the operators
def _plan_plain(s):
    page, ring, counters = s["case"]["page"], s["ring"], s["counters"]
    old, new = s["lens"].long(), s["new_lens"].long()
    cap, room = s["table"].shape[1] * page, s["slots"].numel()
    valid = (old >= 0) & (old <= cap) & (new >= 0) & (new <= cap)
    held, want = (old + page - 1) // page, (new + page - 1) // page
    tokens = torch.where(valid, new - old, 0).clamp(min=0)
    need = torch.where(valid, want - held, 0).clamp(min=0)
    back = torch.where(valid, held - want, 0).clamp(min=0)
    ends, need_to, back_to = tokens.cumsum(0), need.cumsum(0), back.cumsum(0)
    head, tail = counters[0], counters[1]
    granted = valid & ((need == 0) | (need_to <= tail - head)) & ((tokens == 0) | (ends <= room))
    lens_out = torch.where(granted, new, old)
    # pages of the requests that grow, taken from the ring's head
    column = torch.arange(s["table"].shape[1], device=DEV)[None]
    taken = (column >= held[:, None]) & (column < want[:, None]) & granted[:, None]
    place = (head + (need_to - need)[:, None] + column - held[:, None]) % ring.numel()
    table = torch.where(taken, ring[place], s["table"])
    # and of those that shrink, given back at its tail
    given = (column >= want[:, None]) & (column < held[:, None]) & granted[:, None]
    place = (tail + (back_to - back)[:, None] + column - want[:, None]) % ring.numel()
    ring_out = ring.clone()
    ring_out[place[given]] = s["table"][given]
    # the slot of each new token
    i = torch.arange(room, device=DEV)
    b = torch.searchsorted(ends, i, right=True)
    inside = b < len(ends)
    b = b.clamp(max=len(ends) - 1)
    pos = old[b] + i - (ends - tokens)[b]
    entry = table[b, (pos // page).clamp(0, table.shape[1] - 1)].long()
    slots = torch.where(inside & granted[b], entry * page + pos % page, -1)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), ends]).clamp(max=room).int()
    used = torch.stack([head + torch.where(granted, need, 0).sum(), tail + back.sum()])
    return {"table": table, "ring": ring_out, "counters": used, "lens": lens_out.int(), "slots": slots, "starts": starts,
            "refused": (~granted).sum().int().reshape(1)}


def _append_plain(s):
    page, n, heads, dim = s["case"]["page"], s["case"]["tokens"], s["case"]["kv_heads"], s["case"]["head_dim"]
    k, v = s["new_k"].float(), s["new_v"].float()
    if s["k_scale"] is not None:
        k = (k / s["k_scale"][None, :, None]).clamp(-448, 448)
        v = (v / s["v_scale"][None, :, None]).clamp(-448, 448)
    p, o = s["slots"] // page, s["slots"] % page
    raw = torch.int16 if s["k_scale"] is None else torch.int8   # indexed as integers of the same width
    s["k"].view(raw)[p, :, :, o] = k.to(s["k"].dtype).view(raw).reshape(n, heads, -1, s["k"].shape[-1])
    s["v"].view(raw)[p, :, o // 4, :, o % 4] = v.to(s["v"].dtype).view(raw).reshape(n, heads, dim)
    return s["k"], s["v"]


def _attend_plain(s):
    c = s["case"]
    rows, heads, dim = s["table"].clamp(min=0).long(), c["kv_heads"], c["head_dim"]
    batch, keys = c["batch"], rows.shape[1] * c["page"]
    k = s["k"][rows].float().permute(0, 2, 1, 4, 3, 5).reshape(batch, heads, keys, dim)
    v = s["v"][rows].float().permute(0, 2, 1, 3, 5, 4).reshape(batch, heads, keys, dim)
    if s["k_scale"] is not None:
        k, v = k * s["k_scale"].view(1, -1, 1, 1), v * s["v_scale"].view(1, -1, 1, 1)
    there = torch.arange(keys, device=DEV)[None] < s["lens"][:, None]
    q = s["q"].float().reshape(batch, heads, -1, dim).transpose(-1, -2).contiguous()
    score = (k @ q) / math.sqrt(dim)                                    # [batch, kv head, key, query of the head]
    score = score.masked_fill(~there[:, None, :, None], -math.inf)
    top = score.amax(2, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(2).unsqueeze(-1)
    out = p.transpose(-1, -2).contiguous() @ v.masked_fill(~there[:, None, :, None], 0.0)
    out = torch.where(s["lens"].view(-1, 1, 1, 1) > 0, out / total, 0.0)  # a request of no tokens: zeros
    return out.reshape(batch, c["heads"], dim).bfloat16()


def _product_plain(s):
    c = s["case"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).reshape(c["n"], -1, c["group"]).float()
    zeros = 8.0 if s["zeros"] is None else s["zeros"].float()[..., None]
    w = ((codes - zeros) * s["scales"].float()[..., None]).reshape(c["n"], c["k"])
    y = s["a"].float() @ w.t() + s["bias"].float()
    if c["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
    return y + s["resid"] if c["epilogue"] == "residual" else y.bfloat16()


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"plan": _plan_plain, "append": _append_plain, "attend": _attend_plain, "product": _product_plain}[kind](s)
    ie = s["ie"]
    if kind == "plan":
        ie.paged_plan(s["case"]["page"], s["lens"], s["new_lens"], s["table"], s["ring"], s["counters"], s["lens_out"],
                      s["counters_out"], s["slots"], s["starts"], s["refused"])
        return {"table": s["table"], "ring": s["ring"], "counters": s["counters_out"], "lens": s["lens_out"], "slots": s["slots"],
                "starts": s["starts"], "refused": s["refused"]}
    if kind == "append":
        s["cache"].append(s["new_k"], s["new_v"], s["slots"])
        return s["k"], s["v"]
    if kind == "attend":
        s["cache"].attention(s["q"], s["table"], s["lens"], s["out"], s["workspace"])
        return s["out"]
    epilogue = {"bias": ie.EPI_BIAS_BF16, "gelu": ie.EPI_BIAS_GELU_BF16, "residual": ie.EPI_BIAS_RESID_F32}[s["case"]["epilogue"]]
    s["weight"].product(s["a"], s["out"], epilogue, bias=s["bias"], resid=s["resid"])
    return s["out"]


def work(case):
    if case["kind"] == "plan":
        pairs = _requests(case)
        new = sum(max(0, n - o) for o, n in pairs)
        pages = sum(abs((n + case["page"] - 1) // case["page"] - (o + case["page"] - 1) // case["page"]) for o, n in pairs)
        return {"bytes": 16 * len(pairs) + 8 * pages + 8 * new, "flops": 0}
    if case["kind"] == "append":
        n = 2 * case["tokens"] * case["kv_heads"] * case["head_dim"]
        return {"bytes": n * (4 if case["dtype"] == "bf16" else 3) + 8 * case["tokens"], "flops": 0}
    if case["kind"] == "attend":
        lens = _attended(case)
        keys, dim = sum(lens), case["head_dim"]
        pages = sum((n + case["page"] - 1) // case["page"] for n in lens)
        return {"bytes": 2 * keys * case["kv_heads"] * dim * (2 if case["dtype"] == "bf16" else 1) + 4 * case["batch"] * case["heads"] * dim
                + 4 * (pages + case["batch"]), "flops": 4 * keys * case["heads"] * dim}
    n, k, rows = case["n"], case["k"], case["rows"]
    out = 8 if case["epilogue"] == "residual" else 2
    return {"bytes": n * k // 2 + n * (k // case["group"]) * (3 if case["zeros"] else 2) + 2 * rows * k + out * rows * n + 2 * n,
            "flops": 2 * rows * n * k}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _plan_exact(s):
    page, room, ring_n = s["case"]["page"], s["slots"].numel(), s["ring"].numel()
    lens, new, table, ring = (s[k].cpu().numpy().astype(np.int64) for k in ("lens", "new_lens", "table", "ring"))
    free_head, free_tail = s["counters"].tolist()
    head, tail, first, lacking, refused = free_head, free_tail, 0, False, 0
    table, ring_out = table.copy(), ring.copy()
    slots, starts, lens_out = np.full(room, -1, np.int64), np.zeros(len(lens) + 1, np.int32), lens.copy()
    for b, (o, n) in enumerate(zip(lens.tolist(), new.tolist())):
        have, want = -(-o // page), -(-n // page)
        starts[b] = min(first, room)
        fits = first + max(0, n - o) <= room
        if want > have and (lacking or head + want - have > free_tail or not fits):
            lacking = True
        if (want > have and lacking) or (n > o and not fits):
            refused += 1
        else:
            for j in range(have, want):
                table[b, j] = ring[head % ring_n]
                head += 1
            for j in range(want, have):
                ring_out[tail % ring_n] = table[b, j]
                tail += 1
            pos = np.arange(o, max(o, n))
            slots[first:first + len(pos)] = table[b][pos // page] * page + pos % page
            lens_out[b] = n
        first += max(0, n - o)
    starts[-1] = min(first, room)
    return {"table": table.astype(np.int32), "ring": ring_out.astype(np.int32), "counters": np.array([head, tail], np.int64),
            "lens": lens_out.astype(np.int32), "slots": slots, "starts": starts, "refused": np.array([refused], np.int32)}


def _append_exact(s):
    page, k, v = s["case"]["page"], s["k"].double(), s["v"].double()
    new_k, new_v = s["new_k"].double(), s["new_v"].double()
    if s["k_scale"] is not None:
        new_k = torch.clamp(new_k / s["k_scale"].double().view(1, -1, 1), -448.0, 448.0)
        new_v = torch.clamp(new_v / s["v_scale"].double().view(1, -1, 1), -448.0, 448.0)
    # the caches as [page, place, head, column], written and turned back
    kk = k.permute(0, 3, 1, 2, 4).contiguous()
    kk.view(-1, *new_k.shape[1:])[s["slots"]] = new_k
    vv = v.permute(0, 2, 4, 1, 3).contiguous()
    vv.view(-1, *new_v.shape[1:])[s["slots"]] = new_v
    shape = kk.shape
    return (kk.view(shape).permute(0, 2, 3, 1, 4).contiguous(), vv.permute(0, 3, 1, 4, 2).contiguous())


def _attend_exact(s):
    c, lens = s["case"], s["lens"].tolist()
    group, dim = c["heads"] // c["kv_heads"], c["head_dim"]
    out = torch.zeros((c["batch"], c["heads"], dim), dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        if not n:
            continue
        pages = s["table"][b, :(n + c["page"] - 1) // c["page"]].long()
        for h in range(c["kv_heads"]):
            k = s["k"][pages, h].double().permute(0, 2, 1, 3).reshape(-1, dim)[:n]
            v = s["v"][pages, h].double().transpose(-1, -2).reshape(-1, dim)[:n]
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            q = s["q"][b, h * group:(h + 1) * group].double()
            out[b, h * group:(h + 1) * group] = torch.softmax(q @ k.t() / dim ** 0.5, -1) @ v
    return out


def _product_exact(s):
    c = s["case"]
    w = torch.empty((c["n"], c["k"]), dtype=torch.float64, device=DEV)
    w[:, 0::2], w[:, 1::2] = (s["codes"] % 16).double(), (s["codes"] // 16).double()
    w = w.view(c["n"], c["k"] // c["group"], c["group"])
    w -= 8.0 if s["zeros"] is None else s["zeros"].double().unsqueeze(-1)
    w *= s["scales"].double().unsqueeze(-1)
    y = torch.mm(s["a"].double(), w.view(c["n"], c["k"]).t()) + s["bias"].double()
    if c["epilogue"] == "gelu":
        return y * torch.special.ndtr(y)
    return y + s["resid"].double() if c["epilogue"] == "residual" else y


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _plan_exact, "append": _append_exact, "attend": _attend_exact, "product": _product_exact}[case["kind"]](s)
