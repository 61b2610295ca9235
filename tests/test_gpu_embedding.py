"""Embedding lookup and its gradient against 64-bit references.

Bounds: the lookup multiplies once in 32 bits (half an ulp, 2^-24 relative) and rounds once to the output type; the
gradient adds c terms in 32 bits (error at most c ulps of the sum of magnitudes), multiplies and rounds once."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _strided(t, pad, offset=0):
    """The same values with a longer row pitch (and a base that is off by `offset` elements)."""
    if not pad and not offset:
        return t
    buf = torch.zeros(t.shape[0] * (t.shape[1] + pad) + offset, dtype=t.dtype, device=t.device)
    v = buf[offset:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


@pytest.mark.parametrize("tin", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tout", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim,n,pad,offset", [(1, 1, 1, 0, 0), (7, 3, 5, 1, 1), (100, 8, 33, 0, 0), (300, 100, 1000, 0, 0), (50, 128, 4097, 8, 0),
                                                   (64, 1433, 70, 0, 0), (33, 260, 129, 4, 2), (9, 2048, 300, 0, 8)])
def test_lookup(tin, tout, rows, dim, n, pad, offset):
    g = _gen(rows * 1000 + dim)
    table = _strided(torch.randn(rows, dim, generator=g, device="cuda").to(tin), pad, offset)
    ids = torch.randint(-2, rows + 2, (n,), generator=g, device="cuda", dtype=torch.int32)
    scale = 11.25
    out = _strided(torch.full((n, dim), 7.0, device="cuda").to(tout), pad)
    gs.gs_embedding_lookup(table, ids, scale=scale, out=out)
    ok = (ids >= 0) & (ids < rows)
    ref = torch.where(ok[:, None], table.double()[ids.clamp(0, rows - 1).long()] * scale, 0.0)
    assert ((out.double() - ref).abs() <= ref.abs() * (HALF_ULP[tout] + 2.0 ** -23)).all()


def test_lookup_extremes_and_counts():
    table = torch.tensor([[float("inf"), float("nan"), -0.0, 1.0]], device="cuda").repeat(3, 1)
    ids = torch.tensor([0, -1, 2, 1], dtype=torch.int32, device="cuda")
    out = torch.full((4, 4), 5.0, device="cuda")
    gs.gs_embedding_lookup(table, ids, scale=0.0, out=out, count=torch.tensor(3, dtype=torch.int32, device="cuda"))
    assert (out[1] == 0).all()                       # masked row: zeros whatever the table and the scale hold
    assert torch.isnan(out[0, :2]).all() and (out[3] == 5.0).all()   # 0 * inf, 0 * nan; the row behind the count is left as it is
    assert gs.gs_embedding_lookup(table, ids[:0]).shape == (0, 4)


def _ids(kind, n, rows, g):
    if kind == "one":
        return torch.full((n,), rows - 1, dtype=torch.int32, device="cuda")
    if kind == "skew":
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        return (u ** 3 * rows).int().clamp_(max=rows - 1)
    if kind == "none":
        return torch.full((n,), -1, dtype=torch.int32, device="cuda")
    return torch.randint(-3, rows + 3, (n,), generator=g, device="cuda", dtype=torch.int32)


def _reference(dout, ids, rows, scale):
    ok = (ids >= 0) & (ids < rows)
    i, x = ids[ok].long(), dout.double()[ok]
    ref = torch.zeros(rows, dout.shape[1], dtype=torch.float64, device="cuda").index_add_(0, i, x) * scale
    mag = torch.zeros_like(ref).index_add_(0, i, x.abs()) * abs(scale)
    cnt = torch.zeros(rows, dtype=torch.float64, device="cuda").index_add_(0, i, torch.ones_like(i, dtype=torch.float64))
    return ref, mag * (cnt[:, None] + 2) * 2.0 ** -24, torch.unique(i)


SHAPES = [(1, 1, 1, "any", 0), (5, 3, 300, "any", 1), (1000, 128, 4096, "skew", 0), (1000, 64, 4097, "any", 0), (70000, 100, 20000, "skew", 0),
          (40, 36, 70001, "skew", 4), (3, 8, 30000, "one", 0), (200, 1433, 700, "skew", 0), (1 << 20, 16, 5000, "any", 0), (50, 128, 5000, "none", 0),
          (300000, 24, 300001, "skew", 0)]


@pytest.mark.parametrize("tin", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tout", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim,n,kind,pad", SHAPES)
def test_gradient(tin, tout, rows, dim, n, kind, pad):
    g = _gen(rows + dim + n)
    dout = _strided(torch.randn(n, dim, generator=g, device="cuda").to(tin), pad)
    ids = _ids(kind, n, rows, g)
    scale = -1.5
    ws = torch.randint(0, 256, (gs.gs_embedding_workspace_bytes(n, rows, dim),), dtype=torch.uint8, device="cuda")   # holds anything
    ref, slack, unique = _reference(dout, ids, rows, scale)
    out = _strided(torch.full((rows, dim), 3.0, device="cuda").to(tout), pad)
    gs.gs_embedding_backward(dout, ids, rows, ws, scale=scale, out=out)
    assert ((out.double() - ref).abs() <= slack + ref.abs() * HALF_ULP[tout] * 1.01).all()
    first = out.clone()
    gs.gs_embedding_backward(dout, ids, rows, ws, scale=scale, out=out)
    assert torch.equal(first, out)                       # same bits every time
    sid, count, grad = gs.gs_embedding_backward_sparse(dout, ids, rows, ws, scale=scale, out_dtype=tout)
    k = unique.numel()
    assert int(count) == k and torch.equal(sid[:k].long(), unique) and (sid[k:] == -1).all()
    assert torch.equal(grad[:k], out[unique]) and (grad[k:] == 0).all()
    gs.gs_train_status()


def test_gradient_with_device_count_and_capped_grids():
    g = _gen(5)
    n, rows, dim, live = 9000, 500, 32, 6001
    dout = torch.randn(n, dim, generator=g, device="cuda")
    ids = _ids("skew", n, rows, g)
    ws = torch.empty(gs.gs_embedding_workspace_bytes(n, rows, dim), dtype=torch.uint8, device="cuda")
    whole = gs.gs_embedding_backward(dout[:live], ids[:live], rows, ws)
    d = torch.tensor(live, dtype=torch.int32, device="cuda")
    assert torch.equal(whole, gs.gs_embedding_backward(dout, ids, rows, ws, count=d))
    try:
        for cap in (1, 3):
            gs.gs_debug_set_grid_cap(cap)
            assert torch.equal(whole, gs.gs_embedding_backward(dout, ids, rows, ws, count=d))
            sid, count, grad = gs.gs_embedding_backward_sparse(dout, ids, rows, ws, count=d)
            assert torch.equal(grad[:int(count)], whole[sid[:int(count)].long()]) and (sid[int(count):] == -1).all()
    finally:
        gs.gs_debug_set_grid_cap(0)
    zero = torch.zeros((), dtype=torch.int32, device="cuda")
    assert (gs.gs_embedding_backward(dout, ids, rows, ws, count=zero) == 0).all()
    sid, count, grad = gs.gs_embedding_backward_sparse(dout, ids, rows, ws, count=zero)
    assert int(count) == 0 and (sid == -1).all() and (grad == 0).all()
    assert (gs.gs_embedding_backward(dout[:0], ids[:0], rows, ws) == 0).all()
    assert int(gs.gs_embedding_backward_sparse(dout[:0], ids[:0], rows, ws)[1]) == 0


def test_gradient_on_another_stream():
    g = _gen(6)
    dout, ids = torch.randn(20000, 48, generator=g, device="cuda"), _ids("skew", 20000, 3000, g)
    ws = torch.empty(gs.gs_embedding_workspace_bytes(20000, 3000, 48), dtype=torch.uint8, device="cuda")
    want = gs.gs_embedding_backward(dout, ids, 3000, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    gs.gs_embedding_backward(dout, ids, 3000, ws, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_gradient_is_the_derivative():
    """<d(lookup)/dT . dT, dout> = <dT, grad> for a linear operator: compared in 64 bits on values exact in 32."""
    g = _gen(7)
    rows, dim, n = 23, 12, 400
    ids = _ids("any", n, rows, g)
    dt = torch.randint(-8, 9, (rows, dim), generator=g, device="cuda").float()
    dout = torch.randint(-8, 9, (n, dim), generator=g, device="cuda").float()
    ws = torch.empty(gs.gs_embedding_workspace_bytes(n, rows, dim), dtype=torch.uint8, device="cuda")
    left = (gs.gs_embedding_lookup(dt, ids, scale=0.5).double() * dout.double()).sum()
    right = (gs.gs_embedding_backward(dout, ids, rows, ws, scale=0.5).double() * dt.double()).sum()
    assert left == right


def test_refusals():
    table = torch.zeros(4, 8, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(gs.gs_embedding_workspace_bytes(3, 4, 8), dtype=torch.uint8, device="cuda")
    dout = torch.zeros(3, 8, device="cuda")
    with pytest.raises(TypeError):
        gs.gs_embedding_lookup(table.half(), ids)
    with pytest.raises(TypeError):
        gs.gs_embedding_lookup(table, ids.long())
    with pytest.raises(TypeError):
        gs.gs_embedding_lookup(table.t(), ids)
    with pytest.raises(ValueError):
        gs.gs_embedding_lookup(table, ids, out=torch.zeros(2, 8, device="cuda"))
    with pytest.raises(gs.GsError) as e:
        gs.gs_embedding_backward(dout, ids, 4, ws[:256])
    assert e.value.status == 4
    with pytest.raises(gs.GsError) as e:
        gs.gs_embedding_backward(dout, ids, 4, torch.empty(ws.numel() + 256, dtype=torch.uint8, device="cuda")[1:])
    assert e.value.status == 2
    with pytest.raises(gs.GsError) as e:
        gs.gs_embedding_backward(dout, ids, 0, ws)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        gs.gs_embedding_backward(dout[:2], ids, 4, ws)
