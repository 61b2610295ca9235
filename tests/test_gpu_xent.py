"""Softmax cross entropy against a table, loss and gradients, against 64-bit references.

Bounds (u = 2^-23 for one accumulation, rounded or cut; h: half an ulp of the output type, r: of the type in which the
probabilities enter the second product - bf16, 2^-8, for bf16 operands, none for f32):
a logit is off by e_n = (d + 4) u max_v scale sum|h||w|, an exponential by 2^-21; E_n = 4 (e_n + 2^-21 + (V + 4) u) bounds a
probability's relative error, lse and loss are off by E_n + u |lse|;
  dh: sum_v (E p |g scale| + r |dz|) |w| + (V + 4) u sum|dz||w| + h |dh|, dw the same over the rows with their E_n."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -23


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _reference(h, w, y, scale, dl, t_out):
    r = 2.0 ** -8 if h.dtype == torch.bfloat16 else 0.0
    half = HALF_ULP[t_out]
    d, v = h.shape[1], w.shape[0]
    hd, wd = h.double(), w.double()
    z = hd @ wd.t() * scale
    mag = (hd.abs() @ wd.abs().t() * abs(scale)).amax(1)
    valid = (y >= 0) & (y < v)
    lse = torch.logsumexp(z, 1)
    yc = y.clamp(0, v - 1).long()
    at = torch.arange(len(y), device="cuda")
    loss = torch.where(valid, lse - z[at, yc], 0.0)
    E = 4 * ((d + 4) * U * mag + 2.0 ** -21 + (v + 4) * U)
    g = torch.where(valid, dl.double(), 0.0) * scale
    p = torch.exp(z - lse[:, None])
    dz = p.clone()
    dz[at, yc] -= 1.0
    dz = dz * g[:, None]
    err = E[:, None] * p * g.abs()[:, None] + r * dz.abs()
    dh, dw = dz @ wd, dz.t() @ hd
    return {"loss": (loss, torch.where(valid, E + U * (lse.abs() + z[at, yc].abs()), 0.0)), "lse": (lse, E + U * lse.abs()),
            "dhidden": (dh, err @ wd.abs() + (v + 4) * U * (dz.abs() @ wd.abs()) + half * dh.abs()),
            "dtable": (dw, err.t() @ hd.abs() + (len(y) + 4) * U * (dz.abs().t() @ hd.abs()) + half * dw.abs())}


def _check(got, want):
    for name, (ref, slack) in want.items():
        x = got[name].double()
        assert torch.isfinite(x).all(), name
        bad = (x - ref).abs() > slack * 1.01 + 1e-30
        assert not bad.any(), "%s: %d off, worst %g of the bound" % (name, int(bad.sum()), float(((x - ref).abs() / (slack + 1e-30)).max()))


def _run(h, w, y, dl, scale=1.0, out_dtype=None, **kw):
    ws = torch.randint(0, 256, (gs.gs_xent_workspace_bytes(h.shape[0], w.shape[0], h.shape[1], h.dtype),), dtype=torch.uint8, device="cuda")
    loss, lse = gs.gs_xent_forward(h, w, y, ws, scale=scale)
    ws.random_(0, 256)
    dh, dw = gs.gs_xent_backward(h, w, y, lse, dl, ws, scale=scale, out_dtype=out_dtype, **kw)
    return dict(loss=loss, lse=lse, dhidden=dh, dtable=dw)


def _inputs(n, v, d, t, g, std=None):
    h = torch.randn(n, d, generator=g, device="cuda").to(t)
    w = (torch.randn(v, d, generator=g, device="cuda") * (2.0 / d ** 0.5 if std is None else std)).to(t)
    y = torch.randint(-1, v + 1, (n,), generator=g, device="cuda", dtype=torch.int32)     # -1 and vocab are ignored
    dl = torch.randn(n, generator=g, device="cuda")
    return h, w, y, dl


SHAPES = [(1, 1, 1), (1, 2, 3), (3, 47, 100), (64, 64, 64), (65, 129, 33), (130, 1000, 128), (257, 300, 256), (7, 5000, 130), (300, 17, 513), (128, 128, 96),
          (1000, 4097, 72), (200, 40000, 64), (4097, 40, 16), (129, 257, 200), (5, 20000, 8), (2, 3, 1100)]


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v,d", SHAPES)
def test_against_definition(t, n, v, d):
    g = _gen(n + 10 * v + 100 * d)
    h, w, y, dl = _inputs(n, v, d, t, g)
    for out in (torch.float32, torch.bfloat16):
        got = _run(h, w, y, dl, 0.9, out)
        _check(got, _reference(h, w, y, 0.9, dl, out))
        again = _run(h, w, y, dl, 0.9, out)
        assert all(torch.equal(got[k], again[k]) for k in got)        # same bits every time
        assert got["dhidden"].dtype == out
    gs.gs_train_status()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_confident_rows(t):
    """Probabilities within 1e-6 of one and of zero: p - 1 must not be taken from a rounded p."""
    g = _gen(4)
    h, w, y, dl = _inputs(150, 300, 64, t, g)
    y = y.clamp(0, 299)
    h = (w[y.long()].float() * 8.0).to(t)                              # the label's logit stands far above the others
    _check(_run(h, w, y, dl), _reference(h, w, y, 1.0, dl, t))


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_large_logits(t):
    g = _gen(5)
    h, w, y, dl = _inputs(100, 700, 80, t, g, std=20.0)                # logits of several hundred, either sign
    _check(_run(h, w, y, dl), _reference(h, w, y, 1.0, dl, t))


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 100, 128])
def test_strided_operands_and_ignored_rows(t, d):
    g = _gen(6)
    h, w, y, dl = _inputs(140, 333, d, t, g)
    y[:] = torch.where(torch.arange(140, device="cuda") % 3 == 0, y, torch.full_like(y, -7))
    pad = lambda x, k: torch.nn.functional.pad(x, (0, k))[:, :x.shape[1]]  # noqa: E731
    want = _reference(h, w, y, 1.0, dl, t)
    for k in (1, 3, 8):
        dh = torch.full((140, d + k), 9.0, device="cuda").to(t)[:, :d]
        dw = torch.full((333, d + k), 9.0, device="cuda").to(t)[:, :d]
        got = _run(pad(h, k), pad(w, k), y, dl, dhidden=dh, dtable=dw)
        _check(got, want)
        assert (got["dhidden"][y < 0] == 0).all() and (got["loss"][y < 0] == 0).all()
    got = _run(h, w, torch.full_like(y, -1), dl)
    assert (got["dhidden"] == 0).all() and (got["dtable"] == 0).all() and (got["loss"] == 0).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_capped_grids_and_streams(t):
    g = _gen(8)
    h, w, y, dl = _inputs(300, 1500, 64, t, g)
    want = _run(h, w, y, dl)
    try:
        for cap in (1, 3):
            gs.gs_debug_set_grid_cap(cap)
            got = _run(h, w, y, dl)
            _check(got, _reference(h, w, y, 1.0, dl, t))
    finally:
        gs.gs_debug_set_grid_cap(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _run(h, w, y, dl)
    side.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in got)


def test_not_finite_rows_stay_apart():
    """A row that is not finite spoils its own loss and gradient row, and the table's gradient, not the other rows."""
    g = _gen(9)
    for t in (torch.float32, torch.bfloat16):
        h, w, y, dl = _inputs(70, 130, 64, t, g)
        clean = _run(h, w, y, dl)
        h[3, 5] = float("nan")
        got = _run(h, w, y, dl)
        keep = torch.arange(70, device="cuda") != 3
        assert torch.isnan(got["lse"][3])
        assert all(torch.equal(got[k][keep], clean[k][keep]) for k in ("loss", "lse", "dhidden"))


def test_gradients_are_the_derivatives():
    """Central differences of the 64-bit loss, step 1e-6, against the f32 gradients: within 1e-4 of the sum's magnitudes."""
    g = _gen(10)
    h, w, y, dl = _inputs(9, 31, 12, torch.float32, g)
    got = _run(h, w, y, dl)

    def loss(h, w):
        return (_reference(h, w, y, 1.0, dl, torch.float32)["loss"][0] * dl.double()).sum()

    for name in ("dhidden", "dtable"):
        way = torch.randn(got[name].shape, generator=g, device="cuda", dtype=torch.float64)
        step = lambda e: loss(h.double() + (e * way if name == "dhidden" else 0), w.double() + (e * way if name == "dtable" else 0))  # noqa: E731
        slope = (step(1e-6) - step(-1e-6)) / 2e-6
        prod = got[name].double() * way
        assert abs(slope - prod.sum()) <= 1e-4 * prod.abs().sum()


def test_no_rows():
    w = torch.zeros(5, 8, device="cuda")
    h, y = torch.zeros(0, 8, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    loss, lse = gs.gs_xent_forward(h, w, y, ws)
    dh, dw = gs.gs_xent_backward(h, w, y, lse, loss, ws)
    assert loss.numel() == 0 and dh.shape == (0, 8) and (dw == 0).all()


def test_refusals():
    g = _gen(11)
    h, w, y, dl = _inputs(4, 6, 16, torch.float32, g)
    ws = torch.empty(gs.gs_xent_workspace_bytes(4, 6, 16, torch.float32), dtype=torch.uint8, device="cuda")
    lse = torch.zeros(4, device="cuda")
    with pytest.raises(TypeError):
        gs.gs_xent_forward(h, w.bfloat16(), y, ws)
    with pytest.raises(TypeError):
        gs.gs_xent_forward(h.half(), w.half(), y, ws)
    with pytest.raises(TypeError):
        gs.gs_xent_forward(h, w, y.long(), ws)
    with pytest.raises(TypeError):
        gs.gs_xent_forward(h.t(), w.t(), y, ws)
    with pytest.raises(ValueError):
        gs.gs_xent_forward(h, w, y[:3], ws)
    with pytest.raises(TypeError):
        gs.gs_xent_backward(h, w, y, lse.double(), dl, ws)
    with pytest.raises(ValueError):
        gs.gs_xent_backward(h, w, y, lse, dl, ws, dhidden=torch.zeros(4, 17, device="cuda"))
    for bad, status in ((ws[:256], 4), (torch.empty(ws.numel() + 8, dtype=torch.uint8, device="cuda")[8:], 2)):
        with pytest.raises(gs.GsError) as e:
            gs.gs_xent_forward(h, w, y, bad)
        assert e.value.status == status
    big = torch.zeros(1, 5000, device="cuda")
    with pytest.raises(gs.GsError) as e:
        gs.gs_xent_forward(big, big, y[:1], ws)
    assert e.value.status == 1


@pytest.mark.parametrize("n,v,d", [(1, 512, 32), (64, 512, 64), (300, 171, 100), (700, 1024, 128), (130, 300, 200), (90, 513, 256), (5, 3, 24)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_label_entries_keep_their_precision(n, v, d, out):
    """p - 1 of a small p lies just under one, where bf16 loses p: a bias that every row of a label would share.  The
    label's entry enters the product in two parts, 2^-16 of it is lost; the others are rounded once; an exponential of
    the gradient is off by 2^-18 beside E."""
    t = torch.bfloat16
    g = _gen(n + v + d)
    h, w, y, dl = _inputs(n, v, d, t, g, std=0.02)                     # logits near zero: p is about 1 / v
    y = y.clamp(0, v - 1)
    y[: n // 2] = 0                                                    # many rows of one label in one tile
    dl = dl.abs() + 1.0                                                # the bias would not average out
    hd, wd = h.double(), w.double()
    z = hd @ wd.t()
    lse = torch.logsumexp(z, 1)
    at, yc = torch.arange(n, device="cuda"), y.long()
    p = torch.exp(z - lse[:, None])
    dz, other = p.clone(), p.clone()
    dz[at, yc] -= 1.0
    other[at, yc] = 0.0
    E = 4 * ((d + 4) * U * (hd.abs() @ wd.abs().t()).amax(1) + 2.0 ** -21 + (v + 4) * U) + 2.0 ** -18
    label = torch.zeros_like(p)
    label[at, yc] = dz[at, yc].abs()
    dld = dl.double()[:, None]
    err = (E[:, None] * p + 2.0 ** -8 * other + 2.0 ** -16 * label) * dld
    dz = dz * dld
    dh, dw = dz @ wd, dz.t() @ hd
    half = HALF_ULP[out]
    got = _run(h, w, y, dl, 1.0, out)
    _check(got, {"dhidden": (dh, err @ wd.abs() + (v + 4) * U * (dz.abs() @ wd.abs()) + half * dh.abs()),
                 "dtable": (dw, err.t() @ hd.abs() + (n + 4) * U * (dz.abs().t() @ hd.abs()) + half * dw.abs())})
