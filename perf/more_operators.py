"""Performance cases of libiefwd's operators for generation in 4 bits: microscaled matrices and their products, a
paged cache in 4 bits with the attention that reads it, and the log probabilities of the tokens that come out.

A number of the microscaled form (OCP MX, "MXFP4") is one of 0, 0.5, 1, 1.5, 2, 3, 4 and 6 with a sign, in 4 bits; 32
neighbours of a row share a scale, a power of two in 8 bits.  A block's scale is 2^(floor(log2(its largest)) - 2),
its values are rounded to the nearest (ties to even codes) and cut off at +-6.
  - ``quantize``: activations to this form and back to the values that it stands for;
  - ``product``: activations, quantised in the same pass, times a weight matrix in this form;
  - ``store``: new tokens' keys and values to a cache in this form, and tokens of it read back, as when a
    request's cache is handed on;
  - ``attend``: one query per request and head over such a cache or one in 16 bits, with scores that may be capped
    by a tanh and lowered by the distance;
  - ``logprobs``: log probabilities of given tokens, entropy and the most probable alternatives; or, in
    training, the gradient of the first two as well.

Where ``own`` is false, ``run`` is the operator written out in elementary torch operations on 32-bit
numbers; where it is true, it is the library's call.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------------------------ cases
def _quantize(name, rows, k, dtype, gap):
    """gap: elements between the end of a row and the beginning of the next (a slice of a wider matrix)."""
    return dict(name=name, kind="quantize", rows=rows, k=k, dtype=dtype, gap=gap)


def _product(name, rows, n, k, epilogue):
    return dict(name=name, kind="product", rows=rows, n=n, k=k, epilogue=epilogue)


def _store(name, tokens, requests, page, kv_heads, head_dim, pages, reads):
    """`reads` tokens are read back: as many new ones as there are, and others of the pool."""
    return dict(name=name, kind="store", tokens=tokens, requests=requests, page=page, kv_heads=kv_heads, head_dim=head_dim,
                pages=pages, reads=reads)


def _attend(name, batch, heads, kv_heads, head_dim, shortest, longest, page, dtype, cap, slopes, idle=0):
    """One query per request and head over shortest .. longest cached tokens; one in `idle` rows of the batch has none."""
    return dict(name=name, kind="attend", batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, shortest=shortest,
                longest=longest, page=page, dtype=dtype, cap=cap, slopes=slopes, idle=idle)


def _logprobs(name, rows, vocab, gap, dtype, top, scale, masked, train):
    """masked: one in so many rows may only choose among a few tokens, the others' logits are -inf (0: no such row)."""
    return dict(name=name, kind="logprobs", rows=rows, vocab=vocab, gap=gap, dtype=dtype, top=top, scale=scale, masked=masked,
                train=train)


def listed():
    return [
        # one token's hidden state of the large causal model: the time of two launches
        _quantize("quantize_token", 1, 2048, "bf16", 0),
        # a long prompt's activations, a slice of a wider matrix
        _quantize("quantize_prompt", 8191, 8192, "bf16", 64),
        # one token through the up projection of the large causal model, with bias and GELU
        _product("product_token", 1, 8192, 2048, "gelu"),
        # the prompts of a few short requests through a square projection, added to the residual stream
        _product("product_batch", 201, 4096, 4096, "residual"),
        # a long prompt through a wide layer: the largest product
        _product("product_prompt", 8192, 8192, 8192, "bias"),
        # the new tokens of a decode step, a layer with 8 key-value heads
        _store("store_decode", 48, 48, 16, 8, 128, 2048, 48),
        # prompts of several requests, as many tokens read back and some older ones
        _store("store_prompt", 24001, 13, 32, 8, 128, 1024, 26000),
        # one short request of the large causal model (16 heads of 128, a key-value head each): latency
        _attend("attend_short", 1, 16, 16, 128, 300, 300, 16, "mx4", 0.0, False),
        # many long requests with shared key-value heads and capped scores: the cache is as good as all of the bytes
        _attend("attend_full", 64, 32, 8, 128, 4000, 8192, 16, "mx4", 30.0, False),
        # a server's batch on a cache in 16 bits, capped scores lowered by the distance, unused rows of the batch
        _attend("attend_ragged", 96, 16, 4, 64, 5, 12000, 16, "bf16", 50.0, True, 12),
        # the answers of a decode step: chosen tokens, and five alternatives each
        _logprobs("logprobs_decode", 48, 131072, 0, "bf16", 5, 1.0, 6, False),
        # a training batch's tokens under a temperature, with gradients; rows of a padded vocabulary
        _logprobs("logprobs_train", 4095, 65003, 21, "bf16", 0, 1.25, 0, True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["quantize", "product", "product", "product", "store", "attend", "attend", "attend", "logprobs", "logprobs"])
    page = rng.choice([16, 16, 32, 64, 128])
    if kind == "quantize":
        c = _quantize("", _log_int(rng, 1, 8191), _log_int(rng, 1, 16384), rng.choice(["bf16", "bf16", "f32"]), rng.choice([0, 8, 1, 200]))
        while c["rows"] * c["k"] > 8191 * 8192:
            c["rows"] //= 2
    elif kind == "product":
        c = _product("", _log_int(rng, 1, 8192), _log_int(rng, 16, 16384), 32 * _log_int(rng, 1, 512),
                     rng.choice(["bias", "gelu", "residual"]))
        while c["rows"] * c["n"] * c["k"] > 8192 ** 3:
            c["rows"] //= 2
    elif kind == "store":
        requests = _log_int(rng, 1, 64)
        c = _store("", max(requests, _log_int(rng, 1, 24000)), requests, page, rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 128]), 0, 0)
        while c["tokens"] * c["kv_heads"] * c["head_dim"] > 24000 * 1024:
            c["tokens"] = max(requests, c["tokens"] // 2)
        c["pages"] = c["tokens"] // page + 2 * requests + rng.randint(10, 500)
        c["reads"] = c["tokens"] + rng.randint(0, min(2000, c["tokens"]))
    elif kind == "attend":
        heads, kv_heads = rng.choice([(12, 12), (16, 16), (16, 4), (32, 8), (32, 8), (24, 8), (28, 4), (16, 1), (40, 2)])
        longest = _log_int(rng, 1, 40000)
        c = _attend("", _log_int(rng, 1, 128), heads, kv_heads, rng.choice([64, 128, 128]), rng.choice([longest, max(1, longest // 3), 1]),
                    longest, page, rng.choice(["mx4", "mx4", "mx4", "bf16"]), rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.4,
                    rng.choice([0, 0, 5]))
        if c["dtype"] == "bf16" and not c["cap"]:
            c["slopes"] = True          # without either it is an attention of another file's
        while c["batch"] * longest * kv_heads * c["head_dim"] > 64 * 6000 * 1024:
            c["batch"] = max(1, c["batch"] // 2)
    else:
        train = rng.random() < 0.5
        c = _logprobs("", _log_int(rng, 1, 4096), _log_int(rng, 100, 200000), rng.choice([0, 0, 8, 13]), rng.choice(["bf16", "bf16", "f32"]),
                      0 if train else rng.choice([0, 1, 5, 20, 32]), rng.choice([1.0, 1.0, 0.7, 1.4]), rng.choice([0, 0, 3]), train)
        while c["rows"] * c["vocab"] > 4095 * 65003 // (1 if c["dtype"] == "bf16" else 2):
            c["rows"] = max(1, c["rows"] // 2)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ the 4-bit form
def _to_mx4(x):
    """Codes (uint8, one a value) and scale bytes of fp32 rows whose length is a multiple of 32."""
    x = x.unflatten(-1, (-1, 32))
    exponent = (x.abs().amax(-1).contiguous().view(torch.int32) >> 23) - 2      # floor(log2), biased by 127, less 2
    exponent = exponent.clamp(min=0)
    y = x * ((254 - exponent) << 23).view(torch.float32).unsqueeze(-1)      # exact: by a power of two
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5.0).byte()
    return (code + 8 * torch.signbit(y).byte()).flatten(-2), exponent.byte()


def _from_mx4(codes, scales):
    """The values of codes (one a byte, blocks of 32 in the last dimension) under scale bytes, in 32 bits."""
    m = (codes & 7).float()
    size = torch.where(m < 5, torch.where(m < 4, m * 0.5, 2.0), torch.where(m < 6, 3.0, 2.0 * m - 8.0))
    value = torch.where(codes >= 8, -size, size).unflatten(-1, (-1, 32))
    e = scales.int()
    power = torch.where(e > 0, e << 23, 1 << 22).view(torch.float32)      # 2^(e - 127)
    return (value * power.unsqueeze(-1)).flatten(-2)


def _pairs(codes):
    """Two codes a byte, the first in the low half."""
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpair(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 137 + 41)


def _normal(shape, g, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(std=std, generator=g)


def _lengths(case):
    """The requests' lengths, spread over the logarithm of shortest .. longest."""
    count, lo, hi = case["batch"], case["shortest"], case["longest"]
    step = (math.log(hi) - math.log(lo)) / count
    lens = [max(lo, min(hi, int(round(math.exp(math.log(lo) + (i + 0.5) * step))))) for i in range(count)]
    return [0 if case["idle"] and i % case["idle"] == 1 else n for i, n in enumerate(lens)]


def _pages_mx4(x, kind):
    """Pages [pages, place, head, column] in fp32 as the cache holds them in 4 bits, uint8 [pages, heads, 17, ...]: per
    head of a page the codes, and behind them a scale byte for each 16 bytes of codes.  Keys: 16 bytes are 32 columns of
    one token, [columns / 32, place].  Values: 16 bytes are 4 tokens times 8 columns, [place / 4, columns / 8], and a
    scale is one token's for 32 columns, [place / 4, columns / 32, 4]."""
    p, page, h, d = x.shape
    codes, scales = _to_mx4(x)
    codes = _pairs(codes)
    if kind == "k":
        codes = codes.reshape(p, page, h, d // 32, 16).permute(0, 2, 3, 1, 4)
        scales = scales.permute(0, 2, 3, 1)
        shape = (d // 32, page)
    else:
        codes = codes.reshape(p, page // 4, 4, h, d // 8, 4).permute(0, 3, 1, 4, 2, 5)
        scales = scales.reshape(p, page // 4, 4, h, d // 32).permute(0, 3, 1, 4, 2)
        shape = (page // 4, d // 8)
    return torch.cat([codes.reshape(p, h, -1), scales.reshape(p, h, -1)], -1).reshape(p, h, 17, *shape)


def _rows_mx4(pool, kind):
    """The inverse: codes, one a byte, [pages, place, head, column] and scales [pages, place, head, column / 32]."""
    p, h = pool.shape[:2]
    if kind == "k":
        blocks, page = pool.shape[3:]
        codes = pool[:, :, :16].reshape(p, h, blocks, page, 16).permute(0, 3, 1, 2, 4).reshape(p, page, h, blocks * 16)
        return _unpair(codes), pool[:, :, 16].permute(0, 3, 1, 2)
    quads, eights = pool.shape[3:]
    codes = pool[:, :, :16].reshape(p, h, quads, eights, 4, 4).permute(0, 2, 4, 1, 3, 5).reshape(p, quads * 4, h, eights * 4)
    scales = pool[:, :, 16].reshape(p, h, quads, eights // 4, 4).permute(0, 2, 4, 1, 3).reshape(p, quads * 4, h, eights // 4)
    return _unpair(codes), scales


def _pool(case, pages, g):
    page, h, d = case["page"], case["kv_heads"], case["head_dim"]
    if case.get("dtype") == "bf16":
        return _normal((pages, h, d // 8, page, 8), g), _normal((pages, h, page // 4, d, 4), g)
    return tuple(_pages_mx4(_normal((pages, page, h, d), g).float(), kind) for kind in "kv")


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["kind"] == "quantize":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        wide = _normal((case["rows"], case["k"] + case["gap"]), g, dtype=dtype)
        wide *= torch.exp(1.5 * _normal((case["rows"], 1), g, dtype=torch.float32)).to(dtype)      # tokens of different norms
        s["x"] = wide[:, :case["k"]]
        s["values"] = torch.empty((case["rows"], case["k"]), dtype=dtype, device=DEV)
    elif case["kind"] == "product":
        rows, n, k = case["rows"], case["n"], case["k"]
        codes, s["scales"] = _to_mx4(_normal((n, k), g, 0.02, torch.float32))
        s["codes"] = _pairs(codes)
        s["a"] = _normal((rows, k), g)
        s["bias"] = _normal((n,), g, 0.02)
        residual = case["epilogue"] == "residual"
        s["resid"] = _normal((rows, n), g, dtype=torch.float32) if residual else None
        s["out"] = torch.empty((rows, n), dtype=torch.float32 if residual else torch.bfloat16, device=DEV)
    elif case["kind"] == "store":
        page, heads, dim = case["page"], case["kv_heads"], case["head_dim"]
        s["k"], s["v"] = _pool(case, case["pages"], g)
        # the new tokens' rows as a projection leaves them: queries of twice the width, then keys, then values
        rows = _normal((case["tokens"], 4 * heads * dim), g).unflatten(1, (4 * heads, dim))
        s["new_k"], s["new_v"] = rows[:, 2 * heads:3 * heads], rows[:, 3 * heads:]
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
        others = torch.randint(0, case["pages"] * page, (case["reads"] - case["tokens"],), generator=g, device=DEV)
        s["read_slots"] = torch.cat([s["slots"], others])
        s["out_k"], s["out_v"] = (torch.empty((case["reads"], heads, dim), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    elif case["kind"] == "attend":
        page, lens = case["page"], _lengths(case)
        held = [(n + page - 1) // page for n in lens]
        pages, width = sum(held) + 3, max(max(held), 1)
        s["k"], s["v"] = _pool(case, pages, g)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)[torch.randperm(len(lens), generator=g, device=DEV)]
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        s["table"] = torch.full((case["batch"], width), -1, dtype=torch.int32, device=DEV)
        s["table"][torch.arange(width, device=DEV)[None] < ((s["lens"] + page - 1) // page)[:, None]] = order[:sum(held)]
        # the queries as a projection leaves them, beside the keys and values; scores have a standard deviation of 2.8
        rows = _normal((case["batch"], (case["heads"] + 2 * case["kv_heads"]) * case["head_dim"]), g, 2.8)
        s["q"] = rows[:, :case["heads"] * case["head_dim"]].unflatten(1, (case["heads"], -1))
        # a geometric series of slopes over the heads, from 1/2 to 1/256
        s["slopes"] = 2.0 ** -torch.linspace(1.0, 8.0, case["heads"], device=DEV) if case["slopes"] else None
        s["out"] = torch.empty((case["batch"], case["heads"], case["head_dim"]), dtype=torch.bfloat16, device=DEV)
    else:
        rows, vocab = case["rows"], case["vocab"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["logits"] = _normal((rows, vocab + case["gap"]), g, 2.5, dtype)[:, :vocab]
        s["tokens"] = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
        # half of the rows are nearly sure of their token
        sure = torch.arange(0, rows, 2, device=DEV)
        s["logits"][sure, s["tokens"][sure]] += 12.0
        if case["masked"]:
            held = torch.arange(0, rows, case["masked"], device=DEV)
            allowed = torch.rand((len(held), vocab), generator=g, device=DEV) < 0.01
            allowed[torch.arange(len(held), device=DEV), s["tokens"][held]] = True
            s["logits"][held] = s["logits"][held].masked_fill(~allowed, -math.inf)
        if case["train"]:
            s["tokens"][torch.rand(rows, generator=g, device=DEV) < 0.1] = -100      # padding: no token
            s["grad_logprobs"], s["grad_entropy"] = _normal((rows,), g, dtype=torch.float32), _normal((rows,), g, 0.01, torch.float32)
            s["dlogits"] = torch.empty((rows, vocab), dtype=dtype, device=DEV)
        s["logprobs"], s["entropy"] = (torch.empty(rows, dtype=torch.float32, device=DEV) for _ in "le")
        s["stats"] = torch.empty((rows, 2), dtype=torch.float32, device=DEV)
        s["top_ids"] = torch.empty((rows, case["top"]), dtype=torch.int32, device=DEV)
        s["top_logprobs"] = torch.empty((rows, case["top"]), dtype=torch.float32, device=DEV)
    if own:   # what a program keeps from its start: weights in the library's layout, handles, workspaces
        import paper_2503_05130_amd as ie
        s["ie"] = ie
        if case["kind"] == "quantize":
            s["matrix"] = ie.Mx4Matrix(case["rows"], case["k"])
        elif case["kind"] == "product":
            s["weight"] = ie.Mx4Matrix(case["n"], case["k"])
            s["weight"].load(s["codes"], s["scales"])
            s["matrix"] = ie.Mx4Matrix(case["rows"], case["k"])
        elif case["kind"] in ("store", "attend"):
            s["cache"] = ie.PagedCache(s["k"], s["v"])
            if case["kind"] == "attend":
                s["workspace"] = s["cache"].workspace(case["batch"], case["heads"], s["table"].shape[1])
        else:
            s["workspace"] = ie.token_logprobs_workspace(case["rows"], case["vocab"], case["top"])
    return s


# ------------------------------------------------------------------------------------ the operators
def _padded(x, to=32):
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % to))


def _quantize_plain(s):
    return _from_mx4(*_to_mx4(_padded(s["x"].float())))[:, :s["case"]["k"]].to(s["x"].dtype)


def _product_plain(s):
    a = _from_mx4(*_to_mx4(s["a"].float()))
    w = _from_mx4(_unpair(s["codes"]), s["scales"])
    y = a @ w.t() + s["bias"].float()
    if s["case"]["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
    return y + s["resid"] if s["case"]["epilogue"] == "residual" else y.bfloat16()


def _store_plain(s):
    page, heads, dim = s["case"]["page"], s["case"]["kv_heads"], s["case"]["head_dim"]
    p, o = s["slots"] // page, s["slots"] % page
    n, rp, ro = len(p), s["read_slots"] // page, s["read_slots"] % page
    # keys: the pool as codes [pages, head, column block, place, 16 bytes] and scales [pages, head, column block, place]
    codes, scales = _to_mx4(s["new_k"].float())
    flat = s["k"].flatten(2)
    pool = flat[:, :, :page * dim // 2].unflatten(2, (dim // 32, page, 16))
    bytes_ = flat[:, :, page * dim // 2:].unflatten(2, (dim // 32, page))
    pool[p, :, :, o] = _pairs(codes).reshape(n, heads, dim // 32, 16)
    bytes_[p, :, :, o] = scales
    k = _from_mx4(_unpair(pool[rp, :, :, ro].reshape(-1, heads, dim // 2)), bytes_[rp, :, :, ro]).bfloat16()
    # values: [pages, head, place / 4, eight columns, place % 4, 4 bytes] and [pages, head, place / 4, column block, place % 4]
    codes, scales = _to_mx4(s["new_v"].float())
    flat = s["v"].flatten(2)
    pool = flat[:, :, :page * dim // 2].unflatten(2, (page // 4, dim // 8, 4, 4))
    bytes_ = flat[:, :, page * dim // 2:].unflatten(2, (page // 4, dim // 32, 4))
    pool[p, :, o // 4, :, o % 4] = _pairs(codes).reshape(n, heads, dim // 8, 4)
    bytes_[p, :, o // 4, :, o % 4] = scales
    v = _from_mx4(_unpair(pool[rp, :, ro // 4, :, ro % 4].reshape(-1, heads, dim // 2)), bytes_[rp, :, ro // 4, :, ro % 4]).bfloat16()
    return k, v


def _attend_plain(s):
    c = s["case"]
    rows, heads, dim = s["table"].clamp(min=0).long(), c["kv_heads"], c["head_dim"]
    batch, keys = c["batch"], rows.shape[1] * c["page"]
    if c["dtype"] == "bf16":
        k = s["k"][rows].float().permute(0, 2, 1, 4, 3, 5).reshape(batch, heads, keys, dim)
        v = s["v"][rows].float().permute(0, 2, 1, 3, 5, 4).reshape(batch, heads, keys, dim)
    else:
        k, v = (_from_mx4(*_rows_mx4(s[kind], kind))[rows].reshape(batch, keys, heads, dim).transpose(1, 2).contiguous() for kind in "kv")
    there = torch.arange(keys, device=DEV)[None] < s["lens"][:, None]
    q = s["q"].float().reshape(batch, heads, -1, dim).transpose(-1, -2).contiguous()
    score = (k @ q) / math.sqrt(dim)                                    # [batch, kv head, key, query of the head]
    if c["cap"]:
        score = c["cap"] * torch.tanh(score / c["cap"])
    if c["slopes"]:
        distance = (s["lens"][:, None] - 1 - torch.arange(keys, device=DEV)[None]).float()
        score = score - s["slopes"].view(1, heads, 1, -1) * distance.view(batch, 1, keys, 1)
    score = score.masked_fill(~there[:, None, :, None], -math.inf)
    top = score.amax(2, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(2).unsqueeze(-1)
    out = p.transpose(-1, -2).contiguous() @ v.masked_fill(~there[:, None, :, None], 0.0)
    out = torch.where(s["lens"].view(-1, 1, 1, 1) > 0, out / total, 0.0)  # a request of no tokens: zeros
    return out.reshape(batch, c["heads"], dim).bfloat16()


def _logprobs_plain(s):
    c, x = s["case"], s["logits"].float()
    rows = torch.arange(len(x), device=DEV)
    most = x.amax(1, keepdim=True)
    z = (x - most) * c["scale"]
    p = torch.exp(z)
    total = p.sum(1, keepdim=True)
    log_total = torch.log(total)
    given = s["tokens"].clamp(min=0)
    none = s["tokens"] < 0
    out = {"logprobs": torch.where(none, 0.0, z[rows, given] - log_total[:, 0])}
    entropy = log_total[:, 0] - torch.where(p > 0, p * z, 0.0).sum(1) / total[:, 0]
    out["entropy"] = entropy
    if c["top"]:
        ids = torch.sort(s["logits"], dim=1, descending=True, stable=True).indices[:, :c["top"]]      # of equal ones the lowest index first
        out["top_ids"], out["top_logprobs"] = ids.int(), z.gather(1, ids) - log_total
    if c["train"]:
        p /= total
        d = -s["grad_logprobs"].masked_fill(none, 0.0)[:, None] * p - s["grad_entropy"][:, None] * torch.where(p > 0, p * (z - log_total + entropy[:, None]), 0.0)
        d[rows, given] += s["grad_logprobs"].masked_fill(none, 0.0)
        out["dlogits"] = (c["scale"] * d).to(s["logits"].dtype)
    return out


def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"quantize": _quantize_plain, "product": _product_plain, "store": _store_plain, "attend": _attend_plain,
                "logprobs": _logprobs_plain}[kind](s)
    ie = s["ie"]
    if kind == "quantize":
        s["matrix"].quantize(s["x"])
        s["matrix"].values(s["values"])
        return s["values"]
    if kind == "product":
        epilogue = {"bias": ie.EPI_BIAS_BF16, "gelu": ie.EPI_BIAS_GELU_BF16, "residual": ie.EPI_BIAS_RESID_F32}[c["epilogue"]]
        a = s["a"]
        if c["rows"] > 16:      # up to 16 rows the product quantises them by itself
            s["matrix"].quantize(a)
            a = s["matrix"]
        s["weight"].product(a, s["out"], epilogue, bias=s["bias"], resid=s["resid"])
        return s["out"]
    if kind == "store":
        s["cache"].append(s["new_k"], s["new_v"], s["slots"])
        s["cache"].read(s["read_slots"], s["out_k"], s["out_v"])
        return s["out_k"], s["out_v"]
    if kind == "attend":
        s["cache"].attention(s["q"], s["table"], s["lens"], s["out"], s["workspace"], cap=c["cap"], slopes=s["slopes"])
        return s["out"]
    out = {"logprobs": s["logprobs"], "entropy": s["entropy"]}
    if c["top"]:
        out |= {"top_ids": s["top_ids"], "top_logprobs": s["top_logprobs"]}
    ie.token_logprobs(s["logits"], s["tokens"], s["logprobs"], s["workspace"], entropy=s["entropy"], stats=s["stats"],
                      top_ids=s["top_ids"], top_logprobs=s["top_logprobs"], scale=c["scale"])
    if c["train"]:
        ie.token_logprobs_grad(s["logits"], s["tokens"], s["stats"], s["dlogits"], grad_logprobs=s["grad_logprobs"],
                               entropy=s["entropy"], grad_entropy=s["grad_entropy"], scale=c["scale"])
        out["dlogits"] = s["dlogits"]
    return out


def work(case):
    kind = case["kind"]
    if kind == "quantize":      # to the form and back
        n, es = case["rows"] * case["k"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * es, "flops": 0}
    if kind == "product":
        n, k, rows = case["n"], case["k"], case["rows"]
        out = 8 if case["epilogue"] == "residual" else 2
        return {"bytes": n * k * 17 // 32 + 2 * rows * k + out * rows * n + 2 * n, "flops": 2 * rows * n * k}
    if kind == "store":
        width = 2 * case["kv_heads"] * case["head_dim"]
        # new tokens read and written; others than these read from the pool, all written in 16 bits
        return {"bytes": case["tokens"] * (width * 2 + width * 17 // 32 + 8) + (case["reads"] - case["tokens"]) * width * 17 // 32
                + case["reads"] * (2 * width + 8), "flops": 0}
    if kind == "attend":
        lens = _lengths(case)
        keys, dim = sum(lens), case["head_dim"]
        pages = sum((n + case["page"] - 1) // case["page"] for n in lens)
        token = 2 * case["kv_heads"] * (dim * 2 if case["dtype"] == "bf16" else dim * 17 // 32)
        return {"bytes": keys * token + 4 * case["batch"] * case["heads"] * dim + 4 * (pages + case["batch"]),
                "flops": 4 * keys * case["heads"] * dim}
    n = case["rows"] * case["vocab"] * (2 if case["dtype"] == "bf16" else 4)
    return {"bytes": (2 if case["train"] else 1) * n + case["rows"] * (16 + 8 * case["top"] + (8 if case["train"] else 0)), "flops": 0}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _nearest(x):
    """Values of the 4-bit form nearest to fp64 rows of whole blocks, with the scales of the definition."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.clamp(torch.frexp(most).exponent.double() - 3, min=-127.0))      # frexp: most = m 2^e, 1/2 <= m < 1
    unit = torch.where(most == 0, 1.0, unit)
    y = x / unit
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (torch.clamp(torch.round(y / step) * step, -6.0, 6.0) * unit).flatten(-2)


def _listed_values(codes, scales):
    """What bytes of two codes and scale bytes stand for, by the list of the values."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64, device=DEV)
    values = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device=DEV)
    values[..., 0::2], values[..., 1::2] = table[(codes % 16).int()], table[(codes // 16).int()]
    return values * torch.exp2(scales.double() - 127.0).repeat_interleave(32, -1)


def _quantize_exact(s):
    x, k = s["x"].double(), s["case"]["k"]
    whole = torch.zeros((len(x), (k + 31) // 32 * 32), dtype=torch.float64, device=DEV)
    whole[:, :k] = x
    return _nearest(whole)[:, :k]


def _product_exact(s):
    y = torch.mm(_nearest(s["a"].double()), _listed_values(s["codes"], s["scales"]).t().contiguous()) + s["bias"].double()
    if s["case"]["epilogue"] == "gelu":
        return y * torch.special.ndtr(y)
    return y + s["resid"].double() if s["case"]["epilogue"] == "residual" else y


def _token_bytes(pool, kind, pages, places):
    """Bytes of codes and of scales of some tokens, [tokens, heads, column / 2] and [tokens, heads, column / 32]."""
    p, h = pool.shape[:2]
    planes = pool.reshape(p, h, 17, -1)
    codes, scales = planes[:, :, :16].reshape(p, h, -1), planes[:, :, 16]
    if kind == "k":
        blocks, page = pool.shape[3:]
        return (codes.view(p, h, blocks, page, 16)[pages, :, :, places].flatten(2), scales.view(p, h, blocks, page)[pages, :, :, places])
    quads, eights = pool.shape[3:]
    return (codes.view(p, h, quads, eights, 4, 4)[pages, :, places // 4, :, places % 4].flatten(2),
            scales.view(p, h, quads, eights // 4, 4)[pages, :, places // 4, :, places % 4])


def _store_exact(s):
    page, out = s["case"]["page"], []
    for kind in "kv":
        new = _nearest(s["new_" + kind].double())
        read = _listed_values(*_token_bytes(s[kind], kind, s["read_slots"] // page, s["read_slots"] % page))
        # what was read is new where its slot was written
        where = torch.full((s["case"]["pages"] * page,), -1, dtype=torch.int64, device=DEV)
        where[s["slots"]] = torch.arange(len(new), device=DEV)
        at = where[s["read_slots"]]
        out.append(torch.where((at >= 0).view(-1, 1, 1), new[at.clamp(min=0)], read))
    return tuple(out)


def _attend_exact(s):
    c, lens, page = s["case"], s["lens"].tolist(), s["case"]["page"]
    group, dim = c["heads"] // c["kv_heads"], c["head_dim"]
    out = torch.zeros((c["batch"], c["heads"], dim), dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        if not n:
            continue
        pos = torch.arange(n, device=DEV)
        pages, places = s["table"][b].long()[pos // page], pos % page
        if c["dtype"] == "bf16":
            k, v = s["k"][pages, :, :, places].flatten(2).double(), s["v"][pages, :, places // 4, :, places % 4].double()
        else:
            k, v = (_listed_values(*_token_bytes(s[kind], kind, pages, places)) for kind in "kv")
        for h in range(c["kv_heads"]):
            mine = slice(h * group, (h + 1) * group)
            score = s["q"][b, mine].double() @ k[:, h].t().contiguous() / dim ** 0.5
            if c["cap"]:
                score = torch.tanh(score / c["cap"]) * c["cap"]
            if c["slopes"]:
                score = score + s["slopes"][mine].double()[:, None] * (pos - (n - 1)).double()
            out[b, mine] = torch.softmax(score, -1) @ v[:, h].contiguous()
    return out


def _logprobs_exact(s):
    c = s["case"]
    out = {"logprobs": [], "entropy": [], "top_ids": [], "top_logprobs": [], "dlogits": []}
    for first in range(0, c["rows"], 256):      # some rows at a time
        part = slice(first, first + 256)
        logp = torch.log_softmax(s["logits"][part].double() * c["scale"], 1)
        tokens = s["tokens"][part]
        p = torch.exp(logp)
        finite = torch.clamp(logp, min=-1e300)
        entropy = -(p * finite).sum(1)
        picked = torch.gather(logp, 1, tokens.clamp(min=0)[:, None])[:, 0]
        out["logprobs"].append(torch.where(tokens < 0, 0.0, picked))
        out["entropy"].append(entropy)
        if c["top"]:
            # the largest logit first, of equal ones the lowest index
            place = torch.arange(c["vocab"], device=DEV)
            left, ids = s["logits"][part].double(), []
            taken = torch.zeros_like(left, dtype=torch.bool)
            for _ in range(c["top"]):
                best = left.masked_fill(taken, -math.inf).amax(1, keepdim=True)
                at = torch.where(~taken & (left == best), place, c["vocab"]).amin(1, keepdim=True)
                ids.append(at)
                taken.scatter_(1, at, True)
            out["top_ids"].append(torch.cat(ids, 1).int())
            out["top_logprobs"].append(torch.gather(logp, 1, torch.cat(ids, 1)))
        if c["train"]:
            weight = torch.where(tokens < 0, 0.0, s["grad_logprobs"][part].double())
            hot = torch.zeros_like(p).scatter_(1, tokens.clamp(min=0)[:, None], 1.0)
            out["dlogits"].append(c["scale"] * (weight[:, None] * (hot - p) - s["grad_entropy"][part].double()[:, None] * p * (finite + entropy[:, None])))
    return {name: torch.cat(parts) for name, parts in out.items() if parts}


def exact(case, seed):
    s = prepare(case, seed)
    return {"quantize": _quantize_exact, "product": _product_exact, "store": _store_exact, "attend": _attend_exact,
            "logprobs": _logprobs_exact}[case["kind"]](s)
