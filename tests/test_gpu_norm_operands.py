"""The norm in place: every array that a result may share with an operand, and results beside one another in wider rows."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu


def _ws(n, d):
    return torch.empty(gs.gs_rms_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d", [(1, 8), (70, 64), (300, 33), (40, 1433)])
def test_shared_arrays(t, n, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    x, r, dy, dh = (torch.randn(n, d, generator=g, device="cuda").to(t) for _ in range(4))
    w = torch.randn(d, generator=g, device="cuda")
    out, h = gs.gs_rms_norm_forward(x, w, residual=r)
    for hidden, result in ((0, None), (1, None), (None, 0), (None, 1), (0, 1), (1, 0)):
        pair = (x.clone(), r.clone())
        o, k = gs.gs_rms_norm_forward(pair[0], w, residual=pair[1], hidden=None if hidden is None else pair[hidden], out=None if result is None else pair[result])
        assert torch.equal(o, out) and torch.equal(k, h)
    dx, dw = gs.gs_rms_norm_backward(h, dy, _ws(n, d), weight=w, dhidden=dh)
    for which in range(3):
        args = (h.clone(), dy.clone(), dh.clone())
        got, gw = gs.gs_rms_norm_backward(args[0], args[1], _ws(n, d), weight=w, dhidden=args[2], dx=args[which])
        assert torch.equal(got, dx) and torch.equal(gw, dw)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_beside_one_another(t):
    """x, residual, h and the result as columns of one array."""
    g = torch.Generator(device="cuda").manual_seed(1)
    a = torch.randn(50, 160, generator=g, device="cuda").to(t)
    x, r = a[:, :32].clone(), a[:, 32:64].clone()
    out, h = gs.gs_rms_norm_forward(x, None, residual=r)
    rest = a[:, 128:].clone()
    gs.gs_rms_norm_forward(a[:, :32], None, residual=a[:, 32:64], hidden=a[:, 64:96], out=a[:, 96:128])
    assert torch.equal(a[:, :32], x) and torch.equal(a[:, 32:64], r) and torch.equal(a[:, 64:96], h) and torch.equal(a[:, 96:128], out) and torch.equal(a[:, 128:], rest)


def test_refused():
    x, r, o = torch.randn(3, 4, 64, device="cuda").unbind(0)
    with pytest.raises(Exception, match="overlap"):
        gs.gs_rms_norm_forward(x, None, residual=r, out=o, hidden=o)
    with pytest.raises(Exception, match="overlap"):
        gs.gs_rms_norm_forward(x, None, residual=r, out=x, hidden=x)
