"""Stores of rows in 8 bits that are made on one stream and written on another: the memory that a store keeps for writes by id is not the
caller's to see, so it is ready on every stream, and stays the store's while a queued write needs it."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
ROWS, CYCLES = 40000, 200_000_000                             # about 0.1 s


def _tensors(block):
    return torch.zeros(ROWS, 2, 16, dtype=torch.uint8, device="cuda"), torch.zeros((ROWS + block - 1) // block, 2, dtype=torch.uint8, device="cuda")


def _rows(n=3000):
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randn(n, 2, 16, generator=g, device="cuda"), torch.randperm(ROWS, generator=g, device="cuda")[:n].int()


@pytest.mark.parametrize("block", [1, 16])
def test_made_while_its_stream_is_busy(block):
    codes, scales = _tensors(block)
    x, ids = _rows()
    want = gs.gs_coded_write(gs.CodedRows(codes.clone(), scales.clone(), 16, block), x, ids=ids)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    words = ROWS + (2 * scales.shape[0] + 2 if block > 1 else 0)
    old = torch.full((words,), 123456, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    del old                                                   # what the store gets holds this
    torch.cuda._sleep(CYCLES)
    store = gs.CodedRows(codes, scales, 16, block)
    gs.gs_coded_write(store, x, ids=ids, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(store.codes, want.codes) and torch.equal(store.scales, want.scales) and (store.claims == -1).all()


@pytest.mark.parametrize("part", [False, True])
@pytest.mark.parametrize("current", [False, True])
def test_dropped_while_a_write_is_queued(part, current):
    """The stream of the write as the argument, and as the current one; the store itself, and a part of its heads."""
    block = 16
    codes, scales = _tensors(block)
    x, ids = _rows()
    want = gs.gs_coded_write(gs.CodedRows(codes.clone(), scales.clone(), 16, block), x, ids=ids)
    side = torch.cuda.Stream()
    store = gs.CodedRows(codes, scales, 16, block)
    words = store.claims.numel()
    torch.cuda.synchronize()
    to = store.heads(0, 2) if part else store
    del store
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
    if current:
        with torch.cuda.stream(side):
            gs.gs_coded_write(to, x, ids=ids)
    else:
        gs.gs_coded_write(to, x, ids=ids, stream=side)
    del to
    later = [torch.full((words,), 5, dtype=torch.int32, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert all((t == 5).all() for t in later)
    assert torch.equal(codes, want.codes) and torch.equal(scales, want.scales)


def test_captured_on_another_stream():
    """A write that a graph holds, on a stream that the store was not made on; the store goes when the graph has gone."""
    codes, scales = _tensors(16)
    x, ids = _rows()
    want = gs.gs_coded_write(gs.CodedRows(codes.clone(), scales.clone(), 16, 16), x, ids=ids)
    store = gs.CodedRows(codes, scales, 16, 16)
    words = store.claims.numel()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        gs.gs_coded_write(store, x, ids=ids)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(codes, want.codes) and torch.equal(scales, want.scales) and (store.claims == -1).all()
    del graph, store
    later = torch.full((words,), 5, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert (later == 5).all()
