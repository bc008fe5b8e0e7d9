"""Q4Weight packed on another stream than torch's current one: its memory and its inputs' memory in use on both."""
import pytest
import torch

import paper_2503_05130_amd as ie
from tests.gpu_util import DEV, sync

pytestmark = pytest.mark.gpu

N, K, GROUP = 2048, 4096, 64


def _weights(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8),
            torch.rand(N, K // GROUP, generator=g, device=DEV).bfloat16(),
            torch.randint(0, 16, (N, K // GROUP), generator=g, device=DEV, dtype=torch.uint8))


def _product(weight, a, stream=None):
    out = torch.empty(len(a), N, dtype=torch.bfloat16, device=DEV)
    sync()
    weight.product(a, out, stream=stream)
    sync()
    return out


def _hold_back(busy):
    for _ in range(30):
        busy = (busy @ busy).clamp(-1, 1)
    return busy


@pytest.mark.parametrize("handle", [False, True])
def test_packed_memory_is_in_use_on_the_current_stream(handle):
    w, a = _weights(1), torch.randn(3, K, device=DEV).bfloat16()
    want = _product(ie.Q4Weight(*w), a)
    busy = torch.randn(4096, 4096, device=DEV)
    side = torch.cuda.Stream()
    old = ie.Q4Weight(*w).packed
    sync()
    busy = _hold_back(busy)
    old.fill_(0xFF)
    del old                             # its memory is free for the next allocation; its fill has not run yet
    weight = ie.Q4Weight(*w, stream=side.cuda_stream if handle else side)
    got = _product(weight, a, side)
    assert torch.equal(got, want)


@pytest.mark.parametrize("third", [False, True])
def test_inputs_are_freed_while_the_pack_waits(third):
    w, a = _weights(2), torch.randn(3, K, device=DEV).bfloat16()
    want = _product(ie.Q4Weight(*w), a)
    busy = torch.randn(4096, 4096, device=DEV)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    sync()
    with torch.cuda.stream(other if third else torch.cuda.current_stream()):
        copies = [t.clone() for t in w]                 # belong to this stream
    sync()
    with torch.cuda.stream(side):
        busy = _hold_back(busy)
    weight = ie.Q4Weight(*copies, stream=side)
    del copies
    with torch.cuda.stream(other if third else torch.cuda.current_stream()):
        for t in w:
            torch.full_like(t, 1)                       # where the inputs were, if their memory is handed out again
    assert torch.equal(_product(weight, a), want)


def test_a_weight_made_on_a_side_stream_is_ready_on_the_current_one():
    w, a = _weights(3), torch.randn(16, K, device=DEV).bfloat16()
    want = _product(ie.Q4Weight(*w), a)
    busy = torch.randn(4096, 4096, device=DEV)
    side = torch.cuda.Stream()
    sync()
    with torch.cuda.stream(side):
        busy = _hold_back(busy)
    out = torch.empty(16, N, dtype=torch.bfloat16, device=DEV)
    ie.Q4Weight(*w, stream=side).product(a, out)
    sync()
    assert torch.equal(out, want)


def test_products_beside_the_default_stream():
    w, a = _weights(4), torch.randn(9, K, device=DEV).bfloat16()
    weight = ie.Q4Weight(*w, stream=0)                  # the default stream by its handle
    want = _product(weight, a)
    side = torch.cuda.Stream()
    assert torch.equal(_product(weight, a, side), want)
    with torch.cuda.stream(side):
        inner = ie.Q4Weight(*w)
        assert torch.equal(_product(inner, a), want)


@pytest.mark.parametrize("apart", [False, True])
def test_a_weight_packed_in_a_captured_graph(apart):
    """Codes that change between the replays are packed again by each, on the capturing stream or on one beside it."""
    w, a = _weights(5), torch.randn(4, K, device=DEV).bfloat16()
    out = torch.zeros(4, N, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream() if apart else None
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        weight = ie.Q4Weight(*w, stream=side)
        weight.product(a, out)
    for i in range(4):
        for t, new in zip(w, _weights(6 + i)):
            t.copy_(new)
        graph.replay()
        sync()
        assert torch.equal(out, _product(ie.Q4Weight(*w), a)), i
