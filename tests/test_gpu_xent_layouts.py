"""Gradients of the softmax cross entropy into arrays of different layouts, dhidden's and dtable's chosen independently: the
sums do not depend on where they go, so the bits are those of plain contiguous arrays, and what lies between and behind the
rows stays as it was.  The shapes leave tiles that one run finishes alone, and tiles that are joined, in either gradient."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
FILL = 9.0


def _array(rows, dim, layout, t):
    """(the rows, everything around them as a mask, the buffer)."""
    pad, off = {"contiguous": (0, 0), "pitch8": (-dim % 8 + 8, 0), "odd": (1 if dim % 2 == 0 else 2, 0), "shifted": (0, 1)}[layout]
    buf = torch.full((rows * (dim + pad) + off + 64,), FILL, dtype=t, device="cuda")
    around = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    view = lambda b: b[off: off + rows * (dim + pad)].view(rows, dim + pad)[:, :dim]  # noqa: E731
    view(around)[:] = False
    return view(buf), around, buf


LAYOUTS = ["contiguous", "pitch8", "odd", "shifted"]


@pytest.mark.parametrize("n,v", [(200, 20000), (20000, 200), (100, 100)])
@pytest.mark.parametrize("d", [64, 100, 128, 33, 200])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_layouts_of_both_gradients(n, v, d, out):
    g = torch.Generator(device="cuda").manual_seed(n + v + d)
    h = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") * d ** -0.5).bfloat16()
    y = torch.randint(-1, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    dl = torch.randn(n, generator=g, device="cuda")
    ws = torch.empty(gs.gs_xent_workspace_bytes(n, v, d), dtype=torch.uint8, device="cuda")
    _, lse = gs.gs_xent_forward(h, w, y, ws)
    want = gs.gs_xent_backward(h, w, y, lse, dl, ws, out_dtype=out)
    for first in LAYOUTS:
        for second in LAYOUTS:
            dh, around_h, buf_h = _array(n, d, first, out)
            dw, around_w, buf_w = _array(v, d, second, out)
            gs.gs_xent_backward(h, w, y, lse, dl, ws, dhidden=dh, dtable=dw)
            assert torch.equal(dh, want[0]) and torch.equal(dw, want[1]), (first, second)
            assert (buf_h[around_h] == FILL).all() and (buf_w[around_w] == FILL).all(), (first, second)
    gs.gs_train_status()
