"""A model's step in 4 bits as a program runs it: products over microscaled weights, pages and slots, keys and values to a cache
in 4 bits, capped attention over it, the answers' log probabilities; each stage against a plain 64-bit form of its own inputs,
and the whole step captured and replayed."""
import numpy as np
import pytest
import torch

import paper_2503_05130_amd as ie
from tests import mx4_util as X
from tests.gpu_util import DEV, f64, sync

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HEADS, KV, DIM, PAGE, VOCAB, CAP, TOP = 8, 2, 64, 16, 1003, 30.0, 4
WIDTH = HEADS * DIM
SIZES = dict(qkv=((HEADS + 2 * KV) * DIM, WIDTH), o=(WIDTH, WIDTH), up=(1056, WIDTH), down=(WIDTH, 1056), head=(VOCAB, WIDTH))


class _Model:
    def __init__(self, batch, tokens, pages, columns, seed):
        g = torch.Generator().manual_seed(seed)
        self.w, self.values, self.bias = {}, {}, {}
        for name, (n, k) in SIZES.items():
            x = (torch.randn(n, k, generator=g) * k ** -0.5).to(BF)
            self.w[name] = ie.Mx4Matrix(n, k)
            self.w[name].quantize(x.to(DEV))
            self.values[name] = X.values(*X.quantize(f64(x)))[:, :k]
            self.bias[name] = torch.randn(n, generator=g).mul(0.1).to(BF).to(DEV)
        self.cache = ie.PagedCache.empty(pages, PAGE, KV, DIM, mx4=True)
        self.cache.k.fill_(255)
        self.cache.v.fill_(255)
        z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device=DEV)  # noqa: E731
        self.lens, self.lens_out, self.new, self.starts, self.refused = z(batch), z(batch), z(batch), z(batch + 1), z(1)
        self.counters, self.counters_out = torch.tensor([0, pages], device=DEV), z(2, t=torch.int64)
        self.ring = torch.randperm(pages, generator=g).int().to(DEV)
        self.table = torch.full((batch, columns), -1, dtype=torch.int32, device=DEV)
        self.slopes = torch.tensor([2.0 ** -(i + 1) for i in range(HEADS)], device=DEV)
        self.x, self.slots, self.last = z(tokens, WIDTH, t=F32), z(tokens, t=torch.int64), z(batch, t=torch.int64)
        self.tokens = z(batch, t=torch.int64)
        self.a = {k: ie.Mx4Matrix(max(tokens, 17), k) for k in (WIDTH, 1056)}
        self.ws = self.cache.workspace(batch, HEADS, columns)
        self.lws = ie.token_logprobs_workspace(batch, VOCAB, TOP)
        self.out = dict(hidden=z(tokens, WIDTH, t=BF), qkv=z(tokens, SIZES["qkv"][0], t=BF), ctx=z(batch, HEADS, DIM, t=BF),
                        o=z(batch, WIDTH, t=F32), mid=z(batch, WIDTH, t=BF), up=z(batch, 1056, t=BF), down=z(batch, WIDTH, t=F32),
                        final=z(batch, WIDTH, t=BF), logits=z(batch, VOCAB, t=BF), lp=z(batch, t=F32), entropy=z(batch, t=F32),
                        ids=z(batch, TOP), top=z(batch, TOP, t=F32))

    def _product(self, name, x, out, epilogue, resid=None):
        """Few rows in one launch, more with their quantisation before it."""
        a = x
        if len(x) > 16:
            a = self.a[x.shape[1]]
            a.quantize(x)
        self.w[name].product(a, out, epilogue, bias=self.bias[name], resid=resid)

    def step(self):
        o = self.out
        ie.paged_plan(PAGE, self.lens, self.new, self.table, self.ring, self.counters, self.lens_out, self.counters_out, self.slots,
                      self.starts, self.refused)
        o["hidden"].copy_(self.x)
        self._product("qkv", o["hidden"], o["qkv"], ie.EPI_BIAS_BF16)
        q, k, v = o["qkv"].split([WIDTH, KV * DIM, KV * DIM], 1)
        self.cache.append(k.unflatten(1, (KV, DIM)), v.unflatten(1, (KV, DIM)), self.slots)
        last = q.unflatten(1, (HEADS, DIM)).index_select(0, self.last)
        self.cache.attention(last, self.table, self.lens_out, o["ctx"], self.ws, cap=CAP, slopes=self.slopes)
        o["q"] = last
        o["resid"] = self.x.index_select(0, self.last)
        self._product("o", o["ctx"].flatten(1), o["o"], ie.EPI_BIAS_RESID_F32, o["resid"])
        o["mid"].copy_(o["o"])
        self._product("up", o["mid"], o["up"], ie.EPI_BIAS_GELU_BF16)
        self._product("down", o["up"], o["down"], ie.EPI_BIAS_RESID_F32, o["o"])
        o["final"].copy_(o["down"])
        self._product("head", o["final"], o["logits"], ie.EPI_BIAS_BF16)
        ie.token_logprobs(o["logits"], self.tokens, o["lp"], self.lws, entropy=o["entropy"], top_ids=o["ids"], top_logprobs=o["top"])
        self.tokens.copy_(o["ids"][:, 0])
        self.lens.copy_(self.lens_out)
        self.counters.copy_(self.counters_out)


def _check_product(m, name, x, got, resid=None, gelu=False):
    xq, w, k = X.values(*X.quantize(f64(x)))[:, :x.shape[1]], m.values[name], x.shape[1]
    y = xq @ w.T + f64(m.bias[name])
    tol = X.product_tolerance(xq, w, y, k, resid is not None)
    if resid is not None:
        y = y + f64(resid)
        tol = tol + 2.0 ** -23 * np.abs(y)
    if gelu:            # its slope is at most 1.13, its own error 2^-19 of its argument
        z = torch.from_numpy(y)
        y = (0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))).numpy()
        tol = 1.13 * tol + 2.0 ** -19 * np.abs(z.numpy()) + 2.0 ** -8 * np.abs(y)
    assert (np.abs(f64(got) - y) <= tol).all(), name


def _check_step(m, held, given):
    """Every stage from what the stage before it left; held: each request's keys and values by token, given: the tokens asked for."""
    o = m.out
    _check_product(m, "qkv", o["hidden"], o["qkv"])
    starts = m.starts.tolist()
    kv = f64(o["qkv"])[:, WIDTH:].reshape(-1, 2, KV, DIM)
    kv = X.values(*X.quantize(kv))
    batch = len(m.lens)
    for b in range(batch):
        held[b] += list(kv[starts[b]:starts[b + 1]])
        n = len(held[b])
        assert int(m.lens_out[b]) == n
        if not n:
            assert (o["ctx"][b] == 0).all()
            continue
        pool = np.zeros((2, -(-n // PAGE) * PAGE, KV, DIM))
        pool[:, :n] = np.stack(held[b], 1)
        k, v = pool.reshape(2, -1, PAGE, KV, DIM)
        ref, mag, err = X.scored_attention(f64(o["q"])[b:b + 1], k, v, np.arange(len(k))[None], [n], DIM ** -0.5, CAP, f64(m.slopes), False)
        assert (np.abs(f64(o["ctx"])[b:b + 1] - ref) <= X.scored_tolerance(ref, mag, err, n)).all(), b
    _check_product(m, "o", o["ctx"].flatten(1), o["o"], o["resid"])
    _check_product(m, "up", o["mid"], o["up"], gelu=True)
    _check_product(m, "down", o["up"], o["down"], o["o"])
    _check_product(m, "head", o["final"], o["logits"])
    x = o["logits"].cpu().double()
    logp = torch.log_softmax(x, 1)
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :TOP]
    assert torch.equal(o["ids"].cpu().long(), ids)
    # an exponential of a logit d below the best: 2^-22 d and 2^-21; the sums' 2^-24 an addition; log and differences 2^-22 of their sizes
    far = (x.amax(1) - x.amin(1))[:, None]
    tol = 2.0 ** -20 + 2.0 ** -22 * (far + logp.abs()) + 200 * 2.0 ** -24
    assert ((o["top"].cpu().double() - logp.gather(1, ids)).abs() <= tol.gather(1, ids)).all()
    assert ((o["lp"].cpu().double()[:, None] - logp.gather(1, given[:, None])).abs() <= tol.gather(1, given[:, None])).all()
    h = -(logp.exp() * logp).sum(1)
    assert ((o["entropy"].cpu().double() - h).abs() <= 2 * tol.amax(1) * (1 + far[:, 0])).all()


@pytest.mark.parametrize("batch", [1, 5, 21])
def test_steps_of_a_model(batch):
    """Prompts in one step, then tokens one by one, the last ones from a captured graph, with other work between the replays."""
    g = torch.Generator().manual_seed(batch)
    prompts = [[37], [300, 1, 16, 0, 33], [300] + [0, 1, 15, 16, 17] * 4][[1, 5, 21].index(batch)]
    a = _Model(batch, sum(prompts), 120, 30, 3)
    held = [[] for _ in range(batch)]
    a.new.copy_(torch.tensor(prompts, dtype=torch.int32))
    a.last.copy_((torch.tensor(prompts).cumsum(0) - 1).clamp(min=0))
    a.x.copy_(torch.randn(a.x.shape, generator=g))
    a.step()
    sync()
    _check_step(a, held, torch.zeros(batch, dtype=torch.int64))

    b = _Model(batch, batch, 120, 30, 3)            # the same weights; a step of a token each from here on
    for name in ("lens", "counters", "ring", "table", "tokens"):
        getattr(b, name).copy_(getattr(a, name))
    b.cache.k.copy_(a.cache.k)
    b.cache.v.copy_(a.cache.v)
    add = torch.tensor([1 if n else 0 for n in prompts], dtype=torch.int32, device=DEV)
    b.last.copy_((add.long().cumsum(0) - 1).clamp(min=0))

    def step():
        b.new.copy_(b.lens + add)
        b.step()

    for _ in range(3):
        b.x.copy_(torch.randn(b.x.shape, generator=g))
        given = b.tokens.cpu()
        step()
        sync()
        _check_step(b, held, given)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        b.x.copy_(torch.randn(b.x.shape, generator=g))
        given = b.tokens.cpu()
        graph.replay()
        sync()
        _check_step(b, held, given)
        torch.randn(1000, device=DEV).sum().item()
    assert b.lens.tolist() == [n + 7 if n else 0 for n in prompts]


def test_a_training_step_over_its_answers():
    """Logits of a product, the tokens' log probabilities and entropy, and the gradient of the hidden state and the weight's values
    by autograd through fp64 against ours through the logits."""
    g = torch.Generator().manual_seed(4)
    rows = 40
    m = _Model(1, 1, 4, 4, 5)
    x = torch.randn(rows, WIDTH, generator=g).to(BF)
    a = ie.Mx4Matrix(rows, WIDTH)
    logits = torch.empty(rows, VOCAB, dtype=BF, device=DEV)
    tokens = torch.randint(VOCAB, (rows,), generator=g)
    lp, h, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    gl, gh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    grad = torch.empty_like(logits)
    ws = ie.token_logprobs_workspace(rows, VOCAB)
    xd, td, gld, ghd = x.to(DEV), tokens.to(DEV), gl.to(DEV), gh.to(DEV)

    def step():
        a.quantize(xd)
        m.w["head"].product(a, logits)
        ie.token_logprobs(logits, td, lp, ws, entropy=h, stats=stats, scale=0.8)
        ie.token_logprobs_grad(logits, td, stats, grad, grad_logprobs=gld, entropy=h, grad_entropy=ghd, scale=0.8)

    def check():
        z = logits.cpu().double().requires_grad_()
        logp = torch.log_softmax(0.8 * z, 1)
        p = logp.exp()
        ent = -(p * logp).sum(1)
        picked = logp.gather(1, tokens[:, None])[:, 0]
        ((picked * gl.double()).sum() + (ent * gh.double()).sum()).backward()
        # p off by e in its size, log p + h by e as well (twice for the sum's part); the result's half step
        e = 2.0 ** -19 + 2.0 ** -21 * logp.detach().abs().amax(1, keepdim=True)
        pd, ld, hd = p.detach(), logp.detach().abs(), ent.detach()[:, None]
        tol = 0.8 * (pd * e * (gl.abs()[:, None] + gh.abs()[:, None] * (ld + hd + 2)) + 2.0 ** -22 * gl.abs()[:, None]) + 2.0 ** -8 * z.grad.abs()
        assert ((grad.cpu().double() - z.grad).abs() <= tol).all()

    step()
    sync()
    _check_product_no_bias(m, x, logits)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x = torch.randn(rows, WIDTH, generator=g).to(BF)
        xd.copy_(x)
        grad.zero_()
        graph.replay()
        sync()
        _check_product_no_bias(m, x, logits)
        check()
        (xd.float() @ xd.float().T).sum().item()


def _check_product_no_bias(m, x, logits):
    xq = X.values(*X.quantize(f64(x)))[:, :WIDTH]
    y = xq @ m.values["head"].T
    assert (np.abs(f64(logits) - y) <= X.product_tolerance(xq, m.values["head"], y, WIDTH, False)).all()
