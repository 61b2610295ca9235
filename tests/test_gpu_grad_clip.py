"""The norm over many gradients and their scaling, against 64 bits.  u = 2^-24, h half a step of a type: squares are added eight
at a time in 32 bits (8 u of their sum, 4 u of its root), then in 64; the norm is rounded once (u); the factor is off by 5 u, a
scaled number by 7 u + h."""
import math

import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F, B = torch.float32, torch.bfloat16
LISTS = {
    "one": [((1,), F)], "few": [((5, 3), F), ((7,), B), ((1, 1), B)], "tile": [((8192,), F), ((8193,), B), ((8191,), F)],
    "tables": [((1000, 64), F), ((50, 192), B), ((2000003,), B), ((64, 64), F)], "many": [((i % 37 + 1, i % 11 + 1), (F, B)[i % 2]) for i in range(70)],
    "very many": [((i % 5 + 1, 3), (F, B)[i % 3 == 0]) for i in range(1200)], "with empty": [((0, 8), F), ((3, 8), F), ((0,), B)], "large": [((3000, 4096), F), ((10_000_001,), B)],
}


def _grads(kind, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(len(kind))
    return [(torch.randn(s, generator=g, device="cuda") * size).to(t) for s, t in LISTS[kind]]


def _norm(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


def _ws(n):
    return torch.randint(0, 256, (gs.gs_grad_workspace_bytes(n),), dtype=torch.uint8, device="cuda")


def _near_scaled(got, g, norm, max_norm):
    c = min(1.0, max_norm / (norm + 1e-6))
    want = g.double() * c
    assert ((got.double() - want).abs() <= (7 * U + HALF[g.dtype]) * want.abs() + 1e-45).all()


@pytest.mark.parametrize("kind", sorted(LISTS))
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_norm_and_clip(kind, max_norm):
    grads = _grads(kind)
    norm = _norm(grads)
    before = [g.clone() for g in grads]
    got = gs.gs_grad_norm(grads, _ws(len(grads)))
    assert got.shape == (1,) and got.dtype == F and abs(float(got) - norm) <= 5 * U * norm
    out = [torch.full_like(g, 9.0) for g in grads]
    again = gs.gs_grad_clip(grads, max_norm, _ws(len(grads)), out=out)
    assert torch.equal(again, got) and all(torch.equal(a, b) for a, b in zip(grads, before))
    for o, g in zip(out, grads):
        _near_scaled(o, g, norm, max_norm)
    assert torch.equal(gs.gs_grad_clip(grads, max_norm, _ws(len(grads))), got)
    for o, g in zip(out, grads):
        assert torch.equal(o, g)
    if norm < max_norm:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_unaligned_and_permuted_gradients():
    g = torch.Generator(device="cuda").manual_seed(1)
    pool = torch.randn(100_003, generator=g, device="cuda")
    half = torch.randn(70_001, generator=g, device="cuda").to(B)
    grads = [pool[1:20_000], pool[20_001:20_002], half[3:60_000], torch.randn(48, 40, generator=g, device="cuda").t(), torch.randn(6, 5, 4, generator=g, device="cuda").permute(2, 0, 1)]
    norm = _norm(grads)
    out = [torch.empty_like(x) if i > 2 else torch.empty(x.numel() + 5, dtype=x.dtype, device="cuda")[5:] for i, x in enumerate(grads)]
    got = gs.gs_grad_clip(grads, 1.0, _ws(5), out=out)
    assert abs(float(got) - norm) <= 5 * U * norm
    for o, x in zip(out, grads):
        _near_scaled(o, x, norm, 1.0)
    edge = pool[0].clone()
    gs.gs_grad_clip(grads, 1.0, _ws(5))
    assert all(torch.equal(o, x) for o, x in zip(out, grads)) and torch.equal(pool[0], edge)


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("live", [0, 1, 33, 100, 500, -3])
def test_touched_rows(t, live):
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = torch.randn(100, 96, generator=g, device="cuda").to(t)
    n = max(0, min(live, 100))
    rows[n:] = float("nan")
    rest = torch.randn(300, generator=g, device="cuda")
    count = torch.tensor([live], dtype=torch.int32, device="cuda")
    norm = _norm([rows[:n], rest])
    assert abs(float(gs.gs_grad_norm([rows, rest], _ws(2), counts=[count, None])) - norm) <= 5 * U * norm
    out = [torch.full_like(rows, 4.0), torch.empty_like(rest)]
    gs.gs_grad_clip([rows, rest], 2.0, _ws(2), out=out, counts=[count, None])
    _near_scaled(out[0][:n], rows[:n], norm, 2.0)
    _near_scaled(out[1], rest, norm, 2.0)
    assert (out[0][n:] == 4).all()
    gs.gs_grad_clip([rows, rest], 2.0, _ws(2), counts=[count, None])
    assert torch.equal(rows[:n], out[0][:n]) and torch.isnan(rows[n:]).all()


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e18, 1e30])
@pytest.mark.parametrize("t", [F, B])
def test_squares_beyond_32_bits(size, t):
    g = torch.Generator(device="cuda").manual_seed(3)
    grads = [(torch.randn(5000, generator=g, device="cuda") * size).to(t), torch.zeros(999, device="cuda")]
    norm = _norm(grads)
    got = gs.gs_grad_clip(grads, 0.0, _ws(2), norm=torch.empty(1, device="cuda"))
    assert abs(float(got) - norm) <= 5 * U * norm
    assert all((x == 0).all() for x in grads)                # a largest norm of zero


def test_what_is_not_finite_shows():
    """The formula's factor: 0 for an infinite norm (0 times infinity is NaN), NaN for NaN."""
    a, b = torch.ones(70, device="cuda"), torch.ones(9, device="cuda")
    a[3] = float("inf")
    norm = gs.gs_grad_clip([a, b], 1.0, _ws(2))
    assert torch.isinf(norm).all() and (b == 0).all() and torch.isnan(a[3]) and (a[:3] == 0).all()
    a, b = torch.ones(70, device="cuda"), torch.ones(9, device="cuda")
    a[5] = float("nan")
    norm = gs.gs_grad_clip([a, b], 1.0, _ws(2))
    assert torch.isnan(norm).all() and torch.isnan(a).all() and torch.isnan(b).all()


def test_no_gradients():
    assert float(gs.gs_grad_norm([], _ws(0))) == 0.0
    assert float(gs.gs_grad_clip([torch.empty(0, 4, device="cuda")], 1.0, _ws(1))) == 0.0


def test_same_bits_again_and_on_a_small_grid():
    grads = _grads("tables")
    a = gs.gs_grad_norm(grads, _ws(4))
    assert torch.equal(a, gs.gs_grad_norm(grads, _ws(4)))
    gs.gs_debug_set_grid_cap(2)
    try:
        b = gs.gs_grad_clip(grads, 0.1, _ws(4))
    finally:
        gs.gs_debug_set_grid_cap(0)
    assert abs(float(a) - float(b)) <= 2 * U * float(a)
    assert abs(_norm(grads) - 0.1) <= 0.1 * 2.0 ** -9


def test_refusals():
    a, b = torch.ones(8, 6, device="cuda"), torch.ones(40, device="cuda")
    ws = _ws(2)
    with pytest.raises(gs.GsError, match="overlap"):
        gs.gs_grad_clip([a, a], 1.0, ws)
    with pytest.raises(gs.GsError, match="overlap"):
        gs.gs_grad_clip([b[:20], b[10:30]], 1.0, ws)
    with pytest.raises(gs.GsError, match="overlap"):
        gs.gs_grad_clip([b[:20]], 1.0, ws, out=[b[10:30]])
    with pytest.raises(gs.GsError, match="overlap"):
        gs.gs_grad_clip([b[:20], b[20:]], 1.0, ws, out=[torch.empty(20, device="cuda"), b[:20]])
    assert float(gs.gs_grad_norm([a, a], ws)) > 0             # nothing is written
    with pytest.raises(TypeError, match="gaps"):
        gs.gs_grad_norm([a[:, :4]], ws)
    with pytest.raises(TypeError, match="gaps"):
        gs.gs_grad_norm([torch.ones(1, device="cuda").expand(5)], ws)
    with pytest.raises(TypeError, match="contiguous"):
        gs.gs_grad_norm([a.t()], ws, counts=[torch.ones(1, dtype=torch.int32, device="cuda")])
    with pytest.raises(TypeError):
        gs.gs_grad_norm([a.half()], ws)
    with pytest.raises(TypeError):
        gs.gs_grad_clip([a], 1.0, ws, out=[a.to(B)])
    with pytest.raises(ValueError):
        gs.gs_grad_clip([a, b], 1.0, ws, out=[a])
    with pytest.raises(ValueError):
        gs.gs_grad_norm([a.cpu()], ws)
    with pytest.raises(gs.GsError, match="max_norm"):
        gs.gs_grad_clip([a], -1.0, ws)
    with pytest.raises(gs.GsError, match="max_norm"):
        gs.gs_grad_clip([a], float("nan"), ws)
    with pytest.raises(gs.GsError, match="workspace"):
        gs.gs_grad_norm([a], ws[:256])
    assert (a == 1).all() and (b == 1).all()
