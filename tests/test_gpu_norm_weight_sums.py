"""The gradient of the norm's weight over many rows.  Rows of ones and eps = 0 make every term the incoming gradient itself, so that what is
off is the sum.  A lane adds 32 rows in 32 bits, each sum off by at most half a step of it; the sums of a warp's groups join in at
most 5 more additions, a block's sum is rounded once, all else is in 64 bits: (32 + 5 + 1) u of the magnitudes, and 4 u where the mean of
ones is not exactly one.  The terms are 1 + 2^-16 - 2^-23: sums beyond 256 lose 2^-16 of each, 135 u."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("d,lanes", [(4, 1), (8, 2), (33, 32), (64, 16), (100, 32), (128, 32), (256, 32)])
@pytest.mark.parametrize("cap", [1, 2])
def test_many_rows_of_a_lane(d, lanes, cap):
    n = cap * (256 // lanes) * 601 + 3
    x = 1 + 2.0 ** -16 - 2.0 ** -23
    h = torch.ones(n, d, device="cuda")
    dy = torch.full((n, d), x, device="cuda")
    ws = torch.empty(gs.gs_rms_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
    gs.gs_debug_set_grid_cap(cap)
    try:
        _, dw = gs.gs_rms_norm_backward(h, dy, ws, weight=torch.ones(d, device="cuda"), eps=0.0)
    finally:
        gs.gs_debug_set_grid_cap(0)
    off = (dw.double() - n * x).abs()
    assert (off <= (32 + 5 + 1 + 4 + 1) * U * n * x).all(), float((off / (U * n * x)).max())
