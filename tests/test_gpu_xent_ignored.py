"""Hidden rows whose label is outside the table have no part in any gradient, whatever they hold: the results are bit for bit
those with zeros in their place."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v,d", [(1, 5, 8), (140, 333, 64), (300, 700, 100), (130, 2000, 128), (200, 90, 33), (70, 400, 200), (90, 100, 256), (60, 200, 300),
                                   (2000, 40, 16), (257, 20000, 72)])
@pytest.mark.parametrize("pad", [0, 1])
def test_ignored_rows_may_hold_anything(t, n, v, d, pad):
    g = torch.Generator(device="cuda").manual_seed(n + v + d)
    h = torch.nn.functional.pad(torch.randn(n, d, generator=g, device="cuda").to(t), (0, pad))[:, :d]
    w = (torch.randn(v, d, generator=g, device="cuda") * d ** -0.5).to(t)
    y = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    off = torch.rand(n, generator=g, device="cuda") < 0.3
    off[0] = True
    y[off] = torch.where(torch.arange(n, device="cuda") % 2 == 0, -1, v).int()[off]
    dl = torch.randn(n, generator=g, device="cuda")
    ws = torch.empty(gs.gs_xent_workspace_bytes(n, v, d, t), dtype=torch.uint8, device="cuda")

    def run(fill):
        h[off] = fill
        if isinstance(fill, float) and fill == fill:
            h[off, 0] = -fill                              # infinities of both signs
        loss, lse = gs.gs_xent_forward(h, w, y, ws)
        return (loss,) + gs.gs_xent_backward(h, w, y, lse, dl, ws), lse

    want, lse = run(0)
    for fill in (float("nan"), float("inf"), 1e30):
        got, lse2 = run(fill)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert torch.equal(lse[~off], lse2[~off])
    assert (want[1][off] == 0).all() and (want[0][off] == 0).all()
    gs.gs_train_status()
