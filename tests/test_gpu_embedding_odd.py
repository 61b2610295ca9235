"""Tables whose bytes are no multiple of a wide store, and rows longer than a block of threads: exact where only one value is
copied or nothing is added."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 3), (1, 9), (3, 5), (7, 261), (1001, 13), (333, 33), (5001, 261)])
@pytest.mark.parametrize("n", [1, 3, 4097, 70_001])
def test_dense_gradient_of_odd_tables(t, rows, dim, n):
    g = torch.Generator(device="cuda").manual_seed(rows + dim + n)
    ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")       # ids outside the table: no gradient
    ids[0] = rows - 1
    dout = torch.randn(n, dim, generator=g, device="cuda").to(t)
    room = torch.full((rows * dim + 16,), 7.0, dtype=t, device="cuda")  # what lies behind the table stays
    out = room[: rows * dim].view(rows, dim)
    ws = torch.randint(0, 256, (gs.gs_embedding_workspace_bytes(n, rows, dim),), dtype=torch.uint8, device="cuda")
    gs.gs_embedding_backward(dout, ids, rows, ws, out=out)
    want = torch.zeros(rows, dim, dtype=t, device="cuda")
    want[rows - 1] = dout[0]
    assert torch.equal(out, want)
    assert torch.equal(room[rows * dim:], torch.full((16,), 7.0, dtype=t, device="cuda"))


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [256, 257, 1433, 2056, 4104])
@pytest.mark.parametrize("n", [1, 5, 1100, 6001])
@pytest.mark.parametrize("cap", [0, 3])
def test_lookup_of_long_rows(t, dim, n, cap):
    g = torch.Generator(device="cuda").manual_seed(dim + n)
    table = torch.randn(300, dim, generator=g, device="cuda").to(t)
    ids = torch.randint(-1, 301, (n,), generator=g, device="cuda", dtype=torch.int32)
    gs.gs_debug_set_grid_cap(cap)
    try:
        out = gs.gs_embedding_lookup(table, ids)
        torch.cuda.synchronize()
    finally:
        gs.gs_debug_set_grid_cap(0)
    inside = (ids >= 0) & (ids < 300)
    want = torch.where(inside[:, None], table[ids.clamp(0, 299).long()], torch.zeros((), dtype=t, device="cuda"))
    assert torch.equal(out, want)
