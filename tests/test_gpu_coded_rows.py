"""Rows in 8 bits against their definition: every code and scale has to be equal, and what is read back is code times scale."""
import pytest
import torch

import paper_2406_17918_b200 as gs
from coded_reference import Store

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(n, heads, dim, t, g, spread=6.0):
    size = torch.exp2((torch.rand(n, heads, 1, generator=g, device="cuda") - 0.5) * 2 * spread)
    x = torch.randn(n, heads, dim, generator=g, device="cuda") * size
    x[torch.rand(n, heads, generator=g, device="cuda") < 0.1] = 0
    return x.to(t)


def _dirty(rows, heads, dim, block):
    """A store of zero rows whose bytes behind head_dim hold what was there before."""
    store = gs.gs_coded_rows(rows, heads, dim, block)
    store.codes.view(torch.uint8)[:, :, dim:] = 0x7F
    return store


def _same(store, want, written=None):
    got = store.codes.view(torch.uint8)[:, :, :want.dim]
    nan = (got & 127) == 127
    assert torch.equal(nan, (want.codes & 127) == 127)
    assert torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, want.codes))
    assert torch.equal(store.scales, want.scales)
    assert (store.claims == -1).all()
    if written is not None:
        assert (store.codes.view(torch.uint8)[written][:, :, want.dim:] == 0).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block", [1, 2, 16, 64])
@pytest.mark.parametrize("heads,dim", [(1, 1), (4, 32), (8, 16), (3, 33), (2, 24), (5, 100), (1, 257), (2, 128), (33, 4)])
def test_writes_and_reads(t, block, heads, dim):
    g = _gen(heads * 100 + dim + block)
    rows = 203
    store, want = _dirty(rows, heads, dim, block), Store(rows, heads, dim, block)
    for n, spread in ((1, 2.0), (40, 6.0), (203, 1.0), (90, 12.0)):
        ids = torch.randint(-5, rows + 9, (n,), generator=g, device="cuda", dtype=torch.int32)      # some outside, some twice
        x = _rows(n, heads, dim, t, g, spread)
        gs.gs_coded_write(store, x, ids=ids)
        want.write(x, ids.tolist())
        _same(store, want, [r for r in set(ids.tolist()) if 0 <= r < rows])
    some = torch.randint(-3, rows + 5, (97,), generator=g, device="cuda", dtype=torch.int32)
    for out_t in (torch.float32, torch.bfloat16):
        assert torch.equal(gs.gs_coded_read(store, ids=some, out_dtype=out_t).double(), want.read(some.tolist()))
    assert torch.equal(gs.gs_coded_read(store, first=3, num_rows=11, out_dtype=torch.float32).double(), want.read(range(3, 14)))
    assert torch.equal(gs.gs_coded_read(store).double(), want.read(range(rows)))


@pytest.mark.parametrize("block", [1, 4, 16, 64])
@pytest.mark.parametrize("first,n", [(0, 1), (0, 100), (37, 60), (99, 1), (16, 32), (5, 0)])
def test_ranges(block, first, n):
    g = _gen(first + n)
    store, want = _dirty(100, 3, 20, block), Store(100, 3, 20, block)
    for k in range(2):
        old = _rows(100, 3, 20, torch.float32, g)
        gs.gs_coded_write(store, old)
        want.write(old, range(100))
    _same(store, want, slice(0, 100))
    x = _rows(n, 3, 20, torch.bfloat16, g, 10.0)
    gs.gs_coded_write(store, x, first=first)
    want.write(x, range(first, first + n))
    _same(store, want)


def test_a_row_listed_often_holds_the_last():
    g = _gen(1)
    for block in (1, 16):
        store, want = gs.gs_coded_rows(64, 2, 32, block), Store(64, 2, 32, block)
        ids = torch.randint(0, 6, (5000,), generator=g, device="cuda", dtype=torch.int32)
        x = _rows(5000, 2, 32, torch.float32, g)
        gs.gs_coded_write(store, x, ids=ids)
        want.write(x, ids.tolist())
        _same(store, want)


def test_scales_at_their_borders():
    """Largest magnitudes at 448 * 2^k and next to it, in every binade of f32, subnormal numbers among them."""
    tops = [0.0]
    for k in range(-149, 128):
        for m in (1.0, 1.75, 1.75 + 2.0 ** -23, 1.75 - 2.0 ** -23, 2 - 2.0 ** -23):
            v = torch.tensor(m * 2.0 ** k, dtype=torch.float64).float()
            if torch.isfinite(v):
                tops.append(float(v))
    x = torch.zeros(len(tops), 1, 8, device="cuda")
    x[:, 0, 3] = torch.tensor(tops, dtype=torch.float64).float().cuda()
    x[:, 0, 5] = -x[:, 0, 3] * 0.3
    x[:, 0, 6] = x[:, 0, 3] * 2.0 ** -12
    store, want = gs.gs_coded_rows(len(tops), 1, 8, 1), Store(len(tops), 1, 8, 1)
    gs.gs_coded_write(store, x)
    want.write(x, range(len(tops)))
    _same(store, want)
    values = gs.gs_coded_read(store, out_dtype=torch.float32)
    # what is read is rounded to its type: the largest f32 has the code of 256 with the scale 2^120, and 2^128 is infinite in f32
    assert torch.equal(values, want.read(range(len(tops))).float())
    # half a step of a normal code is 2^-4 of it
    big = (x[:, 0, 3] > 2.0 ** -118) & torch.isfinite(values[:, 0, 3])
    assert ((values - x)[:, 0, 3].abs() <= 2.0 ** -4 * x[:, 0, 3])[big].all()


def test_every_tie_goes_to_the_even_code():
    """Halfway between two neighbouring codes, both signs, beside 448 (which keeps the scale at one)."""
    from coded_reference import e4m3_values

    v = e4m3_values()
    mid = ((v[1:] + v[:-1]) / 2).float()
    x = torch.cat([mid, -mid, torch.tensor([448.0])]).cuda().view(1, 1, -1)
    n = x.shape[2]
    store, want = gs.gs_coded_rows(1, 1, n, 1), Store(1, 1, n, 1)
    gs.gs_coded_write(store, x)
    want.write(x, [0])
    assert int(store.scales[0, 0]) == 127
    _same(store, want)


@pytest.mark.parametrize("block", [1, 8])
def test_infinities_and_nan(block):
    """They become NaN, have no part in the scale, and leave the other values what they are without them."""
    g = _gen(3)
    x = _rows(16, 2, 32, torch.float32, g)
    x[3, 0, 5], x[4, 1, 0], x[9, 0, 31], x[9, 0, 30] = INF, -INF, NAN, -NAN
    x[12] = NAN
    store, want = gs.gs_coded_rows(16, 2, 32, block), Store(16, 2, 32, block)
    gs.gs_coded_write(store, x)
    want.write(x, range(16))
    _same(store, want)
    got = gs.gs_coded_read(store, out_dtype=torch.float32)
    assert torch.equal(torch.isnan(got), ~torch.isfinite(x))
    y = _rows(3, 2, 32, torch.float32, g, 14.0) * 1e4              # requantises rows that hold NaN
    gs.gs_coded_write(store, y, first=6)
    want.write(y, range(6, 9))
    _same(store, want)


def test_a_scale_never_falls_while_rows_stay_and_starts_afresh_otherwise():
    store = gs.gs_coded_rows(20, 1, 16, 8)
    gs.gs_coded_write(store, torch.full((20, 1, 16), 448.0, device="cuda"))
    assert store.scales.flatten().tolist() == [127, 127, 127]
    gs.gs_coded_write(store, torch.full((7, 1, 16), 1.0, device="cuda"), first=0)
    assert store.scales.flatten().tolist() == [127, 127, 127]
    gs.gs_coded_write(store, torch.full((8, 1, 16), 1.75, device="cuda"), first=0)
    gs.gs_coded_write(store, torch.full((4, 1, 16), 3.5, device="cuda"), first=16)                  # the last block has four rows
    assert store.scales.flatten().tolist() == [119, 127, 120]


def test_strides_counts_parts_and_streams():
    """A slice of a fused projection into part of a store, the number of rows on the device, on another stream."""
    g = _gen(5)
    fused = torch.randn(50, 3, 4, 24, generator=g, device="cuda")
    store, want = gs.gs_coded_rows(300, 8, 24, 16), Store(300, 8, 24, 16)
    before = store.codes.view(torch.uint8).clone()
    ids = torch.randperm(300, generator=g, device="cuda")[:50].int()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    count = torch.tensor([31], dtype=torch.int32, device="cuda")
    gs.gs_coded_write(store.heads(2, 6), fused[:, 1], ids=ids, count=count, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    x = torch.zeros(50, 8, 24, device="cuda")
    x[:, 2:6] = fused[:, 1]
    want.write(x[:31], ids[:31].tolist())
    _same(store, want)
    assert torch.equal(store.codes.view(torch.uint8)[:, :2], before[:, :2]) and torch.equal(store.codes.view(torch.uint8)[:, 6:], before[:, 6:])
    out = torch.full((50, 4, 29), 7.0, device="cuda")
    got = gs.gs_coded_read(store.heads(2, 6), ids=ids, out=out[:, :, 2:26], count=count)
    assert torch.equal(got[:31].double(), want.read(ids[:31].tolist())[:, 2:6]) and (out[31:] == 7).all() and (out[:, :, :2] == 7).all() and (out[:, :, 26:] == 7).all()
    for live in (0, -4, 80):
        count.fill_(live)
        got = gs.gs_coded_read(store, ids=ids, count=count, out_dtype=torch.float32)
        n = max(0, min(live, 50))
        assert torch.equal(got[:n].double(), want.read(ids[:n].tolist())) and (got[n:] == 0).all()


@pytest.mark.parametrize("cap", [1, 2])
def test_any_grid_gives_the_same(cap):
    g = _gen(6)
    ids = torch.randint(0, 3000, (4000,), generator=g, device="cuda", dtype=torch.int32)
    x = _rows(4000, 4, 32, torch.bfloat16, g)
    stores = []
    for c in (0, cap):
        gs.gs_debug_set_grid_cap(c)
        try:
            s = gs.gs_coded_rows(3000, 4, 32, 16)
            gs.gs_coded_write(s, x[:2000], first=500)
            gs.gs_coded_write(s, x, ids=ids)
            stores.append((s, gs.gs_coded_read(s)))
        finally:
            gs.gs_debug_set_grid_cap(0)
    a, b = stores
    assert torch.equal(a[0].codes.view(torch.uint8), b[0].codes.view(torch.uint8)) and torch.equal(a[0].scales, b[0].scales) and torch.equal(a[1], b[1])


def test_rows_beyond_2_31_bytes():
    """Byte offsets of the codes pass 32 bits."""
    rows, heads, dim = (1 << 32) // 512 + 4000, 4, 128
    store = gs.gs_coded_rows(rows, heads, dim, 16)
    ids = torch.tensor([rows - 1, 5, rows - 3000, (1 << 31) // 512, rows - 17], dtype=torch.int32, device="cuda")
    x = _rows(5, heads, dim, torch.bfloat16, _gen(7))
    gs.gs_coded_write(store, x, ids=ids)
    small = gs.gs_coded_rows(5, heads, dim, 1)
    gs.gs_coded_write(small, x)
    assert torch.equal(gs.gs_coded_read(store, ids=ids), gs.gs_coded_read(small))
    assert int((store.scales != 0).any(1).sum()) == 5 - 1 * (int(ids[0]) // 16 == int(ids[4]) // 16)
