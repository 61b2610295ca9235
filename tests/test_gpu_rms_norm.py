"""The norm against 64 bits.  u = 2^-24, h half a step of the output's type (2^-8 bf16, 2^-24 f32); D columns, N rows.
A sum of D terms in 32 bits is off by at most D u of its magnitudes, the reciprocal root by 2 u and half of its argument's:
  v: (D + 8) u relative;  y: ((D + 12) u + h) |y|
  dx: 2 (D + 12) u (|v g| + |h| v^3 mean|g h|) + 4 u |dh| + h |dx|
  dw: ((N + D + 12) u) sum|dy h v| + h |dw|
  in 8 bits: half a step of the code, 2^-4 of a normal value or 2^-10 of the scale, on top of y's."""
import pytest
import torch

import paper_2406_17918_b200 as gs
from coded_reference import byte_of, unit_of
from paper_2406_17918_b200.autograd import rms_norm

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24
F, B = torch.float32, torch.bfloat16


def _inputs(n, d, t, wt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + n * 8191 + d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return r(n, d).to(t), (r(n, d) * 2).to(t), (1 + 0.3 * r(d)).to(wt), r(n, d).to(t), r(n, d).to(t)


def _hidden(x, res):
    return x if res is None else (x.float() + res.float()).to(x.dtype)


def _reference(h, w, dy, dh, eps):
    h, dy = h.double(), dy.double()
    d = h.shape[1]
    w = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double()
    v = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    g = dy * w
    dx = v * g - h * v ** 3 * (g * h).mean(1, keepdim=True)
    mag = (v * g).abs() + h.abs() * v ** 3 * (g * h).abs().mean(1, keepdim=True)
    if dh is not None:
        dx = dx + dh.double()
    return w * h * v, dx, mag, (dy * h * v).sum(0), (dy * h * v).abs().sum(0)


def _near(got, want, slack, what):
    off = (got.double() - want).abs()
    assert (off <= slack * 1.001 + 1e-37).all(), "%s: %g" % (what, float((off / (slack + 1e-37)).max()))


def _check(x, res, w, dy, dh, eps=1e-6, **kw):
    n, d = x.shape
    t = x.dtype
    out, hidden = gs.gs_rms_norm_forward(x, w, residual=res, eps=eps, **kw)
    assert torch.equal(hidden, _hidden(x, res))
    ws = torch.randint(0, 256, (gs.gs_rms_norm_workspace_bytes(n, d),), dtype=torch.uint8, device="cuda")
    dx, dw = gs.gs_rms_norm_backward(hidden, dy, ws, weight=w, dhidden=dh, eps=eps, **kw)
    y, rdx, mag, rdw, mdw = _reference(hidden, w, dy, dh, eps)
    _near(out, y, ((d + 12) * U + HALF[t]) * y.abs(), "out")
    _near(dx, rdx, 2 * (d + 12) * U * mag + 4 * U * (0 if dh is None else dh.double().abs()) + HALF[t] * rdx.abs(), "dx")
    if w is None:
        assert dw is None
    else:
        _near(dw, rdw, (n + d + 12) * U * mdw + HALF[w.dtype] * rdw.abs(), "dweight")


@pytest.mark.parametrize("t,wt", [(F, F), (B, F), (B, B), (F, B)])
@pytest.mark.parametrize("d", [1, 3, 8, 24, 31, 32, 33, 64, 100, 128, 129, 256, 257, 512, 513, 1024, 1433, 2048, 4099, 8191, 8192])
@pytest.mark.parametrize("n", [1, 2, 37, 700])
def test_against_definition(t, wt, d, n):
    x, res, w, dy, dh = _inputs(n, d, t, wt)
    _check(x, res, w, dy, dh)
    _check(x, None, w, dy, None)


@pytest.mark.parametrize("t", [F, B])
def test_many_rows(t):
    x, res, w, dy, dh = _inputs(70001, 64, t, F)
    _check(x, res, w, dy, dh)
    _check(x, res, None, dy, None)


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("off,pitch", [(0, 136), (1, 136), (8, 137), (4, 132)])
def test_strided_rows(t, off, pitch):
    """Parts of wider rows, at bases and pitches that allow pieces of 16 bytes and that do not: the same bits."""
    x, res, w, dy, dh = _inputs(91, 120, t, F)
    wide = lambda a: torch.full((91, pitch + off), 9.0, dtype=t, device="cuda")[:, off:off + 120].copy_(a)  # noqa: E731
    ws = torch.empty(gs.gs_rms_norm_workspace_bytes(91, 120), dtype=torch.uint8, device="cuda")
    out, hid = wide(x), wide(x)
    dx = wide(x)
    got = gs.gs_rms_norm_forward(wide(x), w, residual=wide(res), out=out, hidden=hid)
    gs.gs_rms_norm_backward(hid, wide(dy), ws, weight=w, dhidden=wide(dh), dx=dx)
    assert got[0] is out and got[1] is hid and torch.equal(hid, _hidden(x, res))
    y, rdx, mag, _, _ = _reference(hid, w, dy, dh, 1e-6)
    _near(out, y, (132 * U + HALF[t]) * y.abs(), "out")
    _near(dx, rdx, 2 * 132 * U * mag + 4 * U * dh.double().abs() + HALF[t] * rdx.abs(), "dx")


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("d", [40, 100, 1433])
def test_in_place(t, d):
    x, res, w, dy, dh = _inputs(333, d, t, F)
    ws = torch.empty(gs.gs_rms_norm_workspace_bytes(333, d), dtype=torch.uint8, device="cuda")
    out, hid = gs.gs_rms_norm_forward(x, w, residual=res)
    dx, dw = gs.gs_rms_norm_backward(hid, dy, ws, weight=w, dhidden=dh)
    a, r = x.clone(), res.clone()
    gs.gs_rms_norm_forward(a, w, residual=r, out=a, hidden=r)
    assert torch.equal(a, out) and torch.equal(r, hid)
    for which in (dy, dh):
        p, q = dy.clone(), dh.clone()
        into = p if which is dy else q
        _, dw2 = gs.gs_rms_norm_backward(hid, p, ws, weight=w, dhidden=q, dx=into)
        assert torch.equal(into, dx) and torch.equal(dw2, dw)


def test_zero_rows_and_eps():
    x = torch.zeros(5, 64, device="cuda")
    x[1] = 1e-20
    x[2] = torch.randn(64, device="cuda") * 1e15
    w, dy = torch.ones(64, device="cuda"), torch.randn(5, 64, device="cuda")
    _check(x, None, w, dy, None, eps=1e-5)
    out, _ = gs.gs_rms_norm_forward(x, w, eps=0.0)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[2]).all()      # 0 / 0, as the formula has it
    x[3, 7] = float("nan")
    out, _ = gs.gs_rms_norm_forward(x, w)
    assert torch.isnan(out[3]).all() and torch.isfinite(out[:3]).all() and torch.isfinite(out[4]).all()


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("d", [64, 1433])
@pytest.mark.parametrize("live", [0, 1, 50, 90])
def test_device_counts(t, d, live):
    x, res, w, dy, dh = _inputs(50, d, t, F)
    count = torch.tensor(live, dtype=torch.int32, device="cuda")
    n = min(live, 50)
    ws = torch.randint(0, 256, (gs.gs_rms_norm_workspace_bytes(50, d),), dtype=torch.uint8, device="cuda")
    x[n:], dy[n:], dh[n:] = float("nan"), float("nan"), float("nan")
    out, hid = gs.gs_rms_norm_forward(x, w, residual=res, count=count)
    dx, dw = gs.gs_rms_norm_backward(hid, dy, ws, weight=w, dhidden=dh, count=count)
    assert (out[n:] == 0).all() and (hid[n:] == 0).all() and (dx[n:] == 0).all()
    y, rdx, mag, rdw, mdw = _reference(hid[:n], w, dy[:n], dh[:n], 1e-6)
    _near(out[:n], y, ((d + 12) * U + HALF[t]) * y.abs(), "out")
    _near(dx[:n], rdx, 2 * (d + 12) * U * mag + 4 * U * dh[:n].double().abs() + HALF[t] * rdx.abs(), "dx")
    _near(dw, rdw, (50 + d + 12) * U * mdw + U * rdw.abs(), "dweight")
    given = torch.full((50, d), 7.0, dtype=t, device="cuda")
    gs.gs_rms_norm_forward(x, w, residual=res, count=count, out=given)
    assert (given[n:] == 7).all() and torch.equal(given[:n], out[:n])


def test_no_rows():
    x, w = torch.empty(0, 24, device="cuda"), torch.ones(24, device="cuda")
    ws = torch.empty(gs.gs_rms_norm_workspace_bytes(0, 24), dtype=torch.uint8, device="cuda")
    out, hid = gs.gs_rms_norm_forward(x, w, residual=x)
    dx, dw = gs.gs_rms_norm_backward(hid, x, ws, weight=w, dweight=torch.full((24,), 5.0, device="cuda"))
    assert out.shape == hid.shape == dx.shape == (0, 24) and (dw == 0).all()


@pytest.mark.parametrize("cap", [1, 3])
def test_few_blocks(cap):
    x, res, w, dy, dh = _inputs(900, 72, B, F)
    gs.gs_debug_set_grid_cap(cap)
    try:
        _check(x, res, w, dy, dh)
        _check(*_inputs(40, 1433, F, F))
    finally:
        gs.gs_debug_set_grid_cap(0)


def test_same_bits_again():
    x, res, w, dy, dh = _inputs(30011, 96, B, F)
    ws = torch.empty(gs.gs_rms_norm_workspace_bytes(30011, 96), dtype=torch.uint8, device="cuda")
    hid = _hidden(x, res)
    a = gs.gs_rms_norm_backward(hid, dy, ws, weight=w, dhidden=dh)
    b = gs.gs_rms_norm_backward(hid, dy, ws, weight=w, dhidden=dh)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("heads,hd", [(1, 1), (1, 8), (4, 32), (8, 16), (3, 33), (1, 100), (5, 24), (2, 128), (8, 128), (128, 8), (1, 1433), (64, 64), (3, 1000), (700, 1), (12, 40)])
@pytest.mark.parametrize("n", [1, 45])
def test_in_eight_bits(t, heads, hd, n):
    d = heads * hd
    x, res, w, _, _ = _inputs(n, d, t, F)
    x[n // 2] = 0
    res[n // 2] = 0
    store = gs.gs_coded_rows(n + 3, heads, hd, 1)
    store.codes.view(torch.uint8).fill_(0x7F)
    got, hid = gs.gs_rms_norm_coded(x, store, w, residual=res)
    assert got is store and torch.equal(hid, _hidden(x, res))
    raw = store.codes.view(torch.uint8)
    assert (raw[:n, :, hd:] == 0).all() and (raw[n:] == 0x7F).all()
    y = _reference(hid, w, hid, None, 1e-6)[0].view(n, heads, hd)
    slack = (d + 12) * U
    top = y.abs().amax(2)
    scales = store.scales[:n].long()
    assert ((scales == byte_of(top * (1 - slack))) | (scales == byte_of(top * (1 + slack)))).all()
    unit = unit_of(scales)[..., None]
    values = gs.gs_coded_read(store, num_rows=n, out_dtype=F)
    # y (1 + slack) lies in the code's interval; a value in the last part of the range is not above 448 but for y's own error
    _near(values, y, torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * unit) + 2 * slack * y.abs(), "values")


def test_rows_that_are_not_finite_in_eight_bits():
    """An infinity makes its own element NaN and the others zeros, a NaN the row; squares beyond 32 bits are an infinity."""
    x = torch.ones(5, 64, device="cuda")
    x[0, 3], x[1, 4], x[2, 5] = float("inf"), float("nan"), 3e38
    x[3] = 0
    store = gs.gs_coded_rows(5, 2, 32, 1)
    gs.gs_rms_norm_coded(x, store)
    v = gs.gs_coded_read(store, num_rows=5, out_dtype=F).view(5, 64)
    assert torch.isnan(v[0, 3]) and (torch.cat([v[0, :3], v[0, 4:]]) == 0).all() and torch.isnan(v[1]).all()
    assert (v[2] == 0).all() and (v[3] == 0).all() and (v[4] == 1).all()


def test_in_eight_bits_without_residual_and_with_a_count():
    x, _, w, _, _ = _inputs(40, 128, B, F)
    a, b = gs.gs_coded_rows(40, 4, 32, 1), gs.gs_coded_rows(40, 4, 32, 1)
    _, hid = gs.gs_rms_norm_coded(x, a, w)
    assert hid is x
    gs.gs_rms_norm_coded(x, b, w, count=torch.tensor(13, dtype=torch.int32, device="cuda"))
    assert torch.equal(a.codes.view(torch.uint8)[:13], b.codes.view(torch.uint8)[:13]) and torch.equal(a.scales[:13], b.scales[:13])
    assert (b.codes.view(torch.uint8)[13:] == 0).all() and (b.scales[13:] == 0).all()


@pytest.mark.parametrize("with_residual", [True, False])
def test_autograd(with_residual):
    """Against 64-bit autograd: f32 sums of 48 terms, 1e-5 of a gradient's norm is twenty times their rounding."""
    x, res, w, _, _ = _inputs(57, 48, F, F)
    mine = [a.clone().requires_grad_() for a in (x, res, w)]
    ref = [a.double().requires_grad_() for a in (x, res, w)]
    mix = torch.linspace(-1, 1, 48, device="cuda")

    def plain(x, res, w):
        h = x + res if with_residual else x
        return w * h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6), h

    if with_residual:
        y, h = rms_norm(mine[0], mine[2], residual=mine[1])
    else:
        y, h = rms_norm(mine[0], mine[2]), mine[0]
    ((y * mix).sum() + (h ** 2 * mix).sum()).backward()
    yr, hr = plain(*ref)
    ((yr * mix).sum() + (hr ** 2 * mix).sum()).backward()
    for a, b in zip(mine, ref):
        if b.grad is None:
            assert a.grad is None
        else:
            assert (a.grad.double() - b.grad).norm() <= 1e-5 * b.grad.norm()


def test_gradient_against_differences():
    """Central differences of the 64-bit formula, step 1e-5: 1e-9 of truncation, 1e-6 of f32."""
    x, res, w, dy, _ = _inputs(3, 20, F, F)
    ws = torch.empty(gs.gs_rms_norm_workspace_bytes(3, 20), dtype=torch.uint8, device="cuda")
    dx, dw = gs.gs_rms_norm_backward(x, dy, ws, weight=w)
    f = lambda x, w: float((dy.double() * w * x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)).sum())  # noqa: E731
    for i in range(3):
        for c in (0, 7, 19):
            e = torch.zeros(3, 20, dtype=torch.float64, device="cuda")
            e[i, c] = 1e-5
            num = (f(x.double() + e, w.double()) - f(x.double() - e, w.double())) / 2e-5
            assert abs(num - float(dx[i, c])) <= 1e-5 * (1 + abs(num))
    for c in (0, 11):
        e = torch.zeros(20, dtype=torch.float64, device="cuda")
        e[c] = 1e-5
        num = (f(x.double(), w.double() + e) - f(x.double(), w.double() - e)) / 2e-5
        assert abs(num - float(dw[c])) <= 1e-5 * (1 + abs(num))


def test_only_the_sum_is_used():
    """The gradient of h alone, and of rows behind a device count: zero."""
    x, res, w, _, _ = _inputs(9, 16, F, F)
    a, b, c = (t.clone().requires_grad_() for t in (x, res, w))
    y, h = rms_norm(a, c, residual=b, count=torch.tensor(5, dtype=torch.int32, device="cuda"))
    (h * 3).sum().backward()
    assert (a.grad[:5] == 3).all() and (a.grad[5:] == 0).all() and torch.equal(a.grad, b.grad) and (c.grad == 0).all()
    a.grad += 1
    assert (b.grad[:5] == 3).all()
    with pytest.raises(RuntimeError, match="first derivatives only"):
        y, _ = rms_norm(a, c, residual=b)
        g, = torch.autograd.grad(y.sum(), a, create_graph=True)
        g.sum().backward()
