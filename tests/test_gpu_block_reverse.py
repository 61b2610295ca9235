"""The block grouped by source against a stable sort on the host: exact, over the shapes in which the offsets of sources
without edges are written in different ways (short gaps, long gaps, more than two sources to an edge)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def build(edges, sources, kind, seed):
    rng = np.random.default_rng(seed)
    if kind == "first":
        ids = np.zeros(edges, np.int32)
    elif kind == "last":
        ids = np.full(edges, sources - 1, np.int32)
    elif kind == "ends":
        ids = np.where(rng.random(edges) < 0.5, 0, sources - 1).astype(np.int32)
    elif kind == "sparse":                                   # few distinct sources: long gaps between them
        ids = rng.choice(rng.integers(0, sources, 5), edges).astype(np.int32)
    else:
        ids = rng.integers(0, sources, edges).astype(np.int32)
    rows = max(1, edges // 7)
    cuts = np.sort(rng.integers(0, edges + 1, rows - 1)) if rows > 1 else np.zeros(0, np.int64)
    if kind == "masked":                                     # ids outside the sources belong to no row
        ids[rng.random(edges) < 0.3] = rng.choice([-1, sources, sources + 7])
    return ids, np.concatenate([[0], cuts, [edges]]).astype(np.int32)


@pytest.mark.parametrize("kind", ["uniform", "first", "last", "ends", "sparse", "masked"])
@pytest.mark.parametrize("edges,sources", [(0, 1), (0, 5000), (1, 1), (1, 2), (1, 3000), (1023, 900), (1024, 1024), (1025, 2050), (1025, 2051),
                                           (2047, 4094), (4096, 100), (4097, 8194), (70_000, 1_000), (70_000, 139_999), (70_000, 300_000)])
@pytest.mark.parametrize("cap", [0, 3])
def test_offsets_order_and_rows(edges, sources, kind, cap):
    import paper_2406_17918_b200 as gs
    ids, indptr = build(edges, sources, kind, edges + sources)
    ids64 = np.where((ids < 0) | (ids >= sources), sources, ids)
    valid = int((ids64 < sources).sum())
    order = np.argsort(ids64, kind="stable").astype(np.int32)
    want_ptr = np.searchsorted(ids64[order], np.arange(sources + 1)).astype(np.int32)
    want_dst = (np.searchsorted(indptr, order, side="right") - 1).astype(np.int32)
    dev = lambda a: torch.from_numpy(a).cuda()
    work = torch.empty(gs.gs_block_attention_workspace_bytes(len(indptr) - 1, sources, max(edges, 1), 1, 1, 8), dtype=torch.uint8, device="cuda")
    gs.gs_debug_set_grid_cap(cap)
    try:
        ptr, dst, edge = gs.gs_block_reverse(dev(indptr), dev(ids), sources, work)
        torch.cuda.synchronize()
    finally:
        gs.gs_debug_set_grid_cap(0)
    assert np.array_equal(ptr.cpu().numpy(), want_ptr)
    assert np.array_equal(edge.cpu().numpy()[:valid], order[:valid])
    assert np.array_equal(dst.cpu().numpy()[:valid], want_dst[:valid])
