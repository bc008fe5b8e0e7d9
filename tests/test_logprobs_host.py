"""What the entry points of token log probabilities refuse before any device work, and their workspace (no GPU needed)."""
import ctypes

import pytest

import paper_2503_05130_amd as ie

P = 1 << 20          # stands for an aligned device address; nothing here reads it


def _space(rows, vocab, top):
    n = ctypes.c_size_t(7)
    return ie.lib().iefwd_token_logprobs_workspace(rows, vocab, top, ctypes.byref(n)), n.value


def _forward(**kw):
    d = dict(kind=0, x=P, stride=100, rows=5, vocab=100, tokens=P, scale=1.0, lp=P, h=None, stats=None, top=0, ids=None, tops=None, ws=P,
             size=1 << 30) | kw
    return ie.lib().iefwd_token_logprobs(*d.values(), None)


def _grad(**kw):
    d = dict(kind=0, x=P, stride=100, rows=5, vocab=100, tokens=P, scale=1.0, stats=P, h=None, gl=P, gh=None, out=2 * P, os=100) | kw
    return ie.lib().iefwd_token_logprobs_grad(*d.values(), None)


SIZES = [dict(rows=0), dict(rows=(1 << 22) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1, stride=1 << 25),
         dict(rows=1 << 20, vocab=1 << 16, stride=1 << 16)]


@pytest.mark.parametrize("bad", SIZES)
def test_bad_sizes(bad):
    d = dict(rows=5, vocab=100) | {k: v for k, v in bad.items() if k != "stride"}
    assert _space(d["rows"], d["vocab"], 0) == (ie.EINVAL, 7)
    assert _forward(**bad) == ie.EINVAL and ie.last_error()
    assert _grad(**bad, **({"os": bad["stride"]} if "stride" in bad else {})) == ie.EINVAL


@pytest.mark.parametrize("bad", [dict(kind=2), dict(x=None), dict(x=P + 1), dict(kind=1, x=P + 2), dict(stride=99), dict(stride=(1 << 40) + 1),
                                 dict(tokens=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(scale=2.0 ** -31), dict(scale=2.0 ** 31)])
def test_what_both_refuse(bad):
    assert _forward(**bad) == ie.EINVAL
    assert _grad(**bad) == ie.EINVAL


@pytest.mark.parametrize("bad", [dict(lp=None), dict(top=1), dict(top=1, ids=P), dict(top=1, tops=P), dict(top=33, ids=P, tops=P),
                                 dict(top=11, vocab=10, ids=P, tops=P), dict(vocab=50000, stride=50000, size=16),
                                 dict(vocab=50000, stride=50000, ws=None), dict(vocab=50000, stride=50000, ws=P + 8)])
def test_what_the_forward_call_refuses(bad):
    assert _forward(**bad) == ie.EINVAL


@pytest.mark.parametrize("bad", [dict(stats=None), dict(gl=None), dict(gh=P), dict(out=None), dict(out=2 * P + 1), dict(os=99),
                                 dict(out=P, os=104)])
def test_what_the_gradient_refuses(bad):
    assert _grad(**bad) == ie.EINVAL


def test_workspace():
    assert _space(1, 100, 32) == (ie.OK, 0) and _space(5000, 200000, 32) == (ie.OK, 0)
    one, more = _space(1, 131072, 0), _space(1, 131072, 32)
    assert one[0] == more[0] == ie.OK and 0 < one[1] < more[1]
    assert ie.lib().iefwd_token_logprobs_workspace(1, 1, 0, None) == ie.EINVAL
    assert _space(5, 10, 11)[0] == ie.EINVAL and _space(5, 100, 33)[0] == ie.EINVAL


@pytest.mark.parametrize("rows,vocab,n", [((1 << 32) + 1, 100, 0), (1, (1 << 32) + 100, 0), (1, 100, (1 << 32) + 1), (-1, 100, 0)])
def test_sizes_beyond_32_bits_are_refused_by_the_binding(rows, vocab, n):
    with pytest.raises(ValueError, match="2.32"):
        ie.token_logprobs_workspace(rows, vocab, n)
