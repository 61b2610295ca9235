"""Attention over rows in 8 bits against the definition in 64 bits, on the values that the store holds.

Bounds as for the attention over typed rows (u = 2^-24, h half a step of the output's type): a score is off by at most
(D + 6) u scale sum|q||k| (two more products, by the scales), an exponential by 2^-21 relative, a sum of n terms by n u of its
magnitudes: E = 4 ((D + 6) u max_e scale sum|q||k| + 2^-21 + (n + 6) u) relative for a probability;
  out: E sum p|v| + h |out|;  lse: E + 2^-23 |lse|."""
import math

import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24
F, B = torch.float32, torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _block(lengths, src, g, masked=0.0):
    indptr = torch.zeros(len(lengths) + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = torch.tensor(lengths, device="cuda").cumsum(0).int()
    e = int(indptr[-1])
    idx = (torch.rand(e, generator=g, device="cuda") ** 2 * src).int().clamp_(max=src - 1)
    off = torch.rand(e, generator=g, device="cuda") < masked
    idx[off] = torch.where(torch.rand(e, generator=g, device="cuda") < 0.5, -1, src + 5).int()[off]
    return indptr, idx


def _store(rows, heads, dim, block, g):
    s = gs.gs_coded_rows(rows, heads, dim, block)
    size = torch.exp2(torch.rand(rows, heads, 1, generator=g, device="cuda") * 4 - 2)
    gs.gs_coded_write(s, torch.randn(rows, heads, dim, generator=g, device="cuda") * size)
    return s


def _reference(indptr, idx, q, k, v, scale, t, sources=None, rows=None):
    """k, v: the values [rows, heads, dim] in 64 bits."""
    h = HALF_ULP[t]
    n, hq, d = q.shape
    hk = k.shape[1]
    src = sources if sources is not None else k.shape[0]
    keep = (idx >= 0) & (idx < src)
    at = idx.clamp(0, max(src - 1, 0)).long()
    if rows is not None:
        at = rows.long()[at]
        keep &= (at >= 0) & (at < k.shape[0])
    dst = torch.repeat_interleave(torch.arange(n, device="cuda"), (indptr[1:] - indptr[:-1]).long())[keep]
    j = at[keep]
    q = q.double()
    kx, vx = k[j].repeat_interleave(hq // hk, 1), v[j].repeat_interleave(hq // hk, 1)
    add = lambda x: torch.zeros((n,) + x.shape[1:], dtype=torch.float64, device="cuda").index_add_(0, dst, x)  # noqa: E731
    cnt = add(torch.ones(len(dst), 1, dtype=torch.float64, device="cuda"))
    s = (q[dst] * kx).sum(-1) * scale
    smag = (q[dst].abs() * kx.abs()).sum(-1) * abs(scale)
    top = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce(0, dst[:, None].expand_as(s), s, "amax")
    tmag = torch.zeros((n, hq), dtype=torch.float64, device="cuda").scatter_reduce(0, dst[:, None].expand_as(s), smag, "amax")
    w = torch.exp(s - top[dst])
    tot = add(w)
    p = w / tot[dst]
    lse, out = top + torch.log(tot), add(p[..., None] * vx)
    E = 4 * ((d + 6) * U * tmag + 2.0 ** -21 + (cnt + 6) * U)
    return {"out": (out, E[..., None] * add(p[..., None] * vx.abs()) + h * out.abs()), "lse": (lse, E + 2.0 ** -23 * lse.abs())}


def _check(name, got, want):
    ref, slack = want
    got = got.double()
    if name == "lse":
        empty = torch.isinf(ref)
        assert torch.equal(torch.isneginf(got), empty)
        got, ref, slack = got[~empty], ref[~empty], slack[~empty]
    off = (got - ref).abs()
    assert (off <= slack * 1.01 + 1e-30).all(), "%s: worst %g" % (name, float((off / (slack + 1e-30)).max()))


def _ws(n, e, hq, d):
    return torch.randint(0, 256, (gs.gs_coded_attention_workspace_bytes(n, e, hq, d),), dtype=torch.uint8, device="cuda")


def _values(store):
    return gs.gs_coded_read(store, out_dtype=F).double()


LENGTHS = {
    "one": [1], "empty": [0, 0, 0], "few": [5, 0, 3, 1, 0, 4], "fan": [(i * 7) % 21 for i in range(300)],
    "hub": [0, 700, 3, 256, 257, 64, 65, 1, 5000], "long": [9000], "even": [20] * 5000,
}
SHAPES = [(1, 1, 8, 1), (4, 4, 16, 16), (4, 2, 32, 16), (8, 1, 24, 64), (8, 8, 16, 1), (3, 3, 33, 4), (6, 2, 20, 2), (2, 1, 128, 16), (1, 1, 256, 8),
          (5, 1, 7, 1), (4, 4, 100, 16), (2, 2, 130, 32), (12, 3, 64, 16), (4, 4, 32, 16), (2, 2, 1, 1), (16, 2, 256, 16)]


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("hq,hk,d,block", SHAPES)
@pytest.mark.parametrize("kind", sorted(LENGTHS))
def test_against_definition(t, hq, hk, d, block, kind):
    g = _gen(hq * 1000 + d)
    lengths = LENGTHS[kind]
    src = 37 if kind in ("few", "one", "empty") else 403
    indptr, idx = _block(lengths, src, g, masked=0.15 if kind != "one" else 0.0)
    store = _store(src, 2 * hk, d, block, g)
    q = torch.randn(len(lengths), hq, d, generator=g, device="cuda").to(t)
    longest = max(lengths)
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :hk], both[:, hk:], d ** -0.5, t)
    for max_row in (0, longest, 1):                           # a bound that is too small is slower, not wrong
        out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, hk), store.heads(hk, 2 * hk), _ws(len(lengths), idx.numel(), hq, d), max_row=max_row)
        _check("out", out, want["out"])
        _check("lse", lse, want["lse"])


@pytest.mark.parametrize("t", [F, B])
def test_sources_through_their_rows(t):
    """A block of local indices, the cache by node id; rows outside the store are masked."""
    g = _gen(1)
    indptr, idx = _block([(i * 5) % 17 for i in range(120)] + [300], 90, g, masked=0.1)
    store = _store(1000, 4, 32, 16, g)
    rows = torch.randint(0, 1000, (90,), generator=g, device="cuda", dtype=torch.int32)
    rows[4], rows[17], rows[50] = -1, 1000, 2_000_000_000
    q = torch.randn(121, 8, 32, generator=g, device="cuda").to(t)
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 2), store.heads(2, 4), _ws(121, idx.numel(), 8, 32), rows=rows, scale=0.3)
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :2], both[:, 2:], 0.3, t, sources=90, rows=rows)
    _check("out", out, want["out"])
    _check("lse", lse, want["lse"])


def test_masked_rows_are_not_read():
    """NaN in rows that no edge names, or only masked ones; a row with a NaN key is NaN itself."""
    g = _gen(2)
    store = _store(40, 2, 16, 1, g)
    bad = torch.full((1, 2, 16), float("nan"), device="cuda")
    for r in (0, 7, 39):
        gs.gs_coded_write(store, bad, first=r)
    idx = torch.tensor([1, -1, 40, 5, 6, 2, 7], dtype=torch.int32, device="cuda")
    indptr = torch.tensor([0, 3, 3, 6, 7], dtype=torch.int32, device="cuda")
    q = torch.randn(4, 1, 16, generator=g, device="cuda")
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 1), store.heads(1, 2), _ws(4, 7, 1, 16))
    assert torch.isfinite(out[:3]).all() and (out[1] == 0).all() and torch.isneginf(lse[1]).all() and torch.isnan(out[3]).all()


@pytest.mark.parametrize("t", [F, B])
def test_all_edges_masked_in_a_long_row(t):
    g = _gen(3)
    store = _store(10, 2, 32, 2, g)
    indptr = torch.tensor([0, 500, 501], dtype=torch.int32, device="cuda")
    idx = torch.full((501,), -1, dtype=torch.int32, device="cuda")
    idx[500] = 3
    q = torch.randn(2, 4, 32, generator=g, device="cuda").to(t)
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 1), store.heads(1, 2), _ws(2, 501, 4, 32))
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()
    want = _values(store)[3, 1].to(t)
    assert (out[1] == want).all()


@pytest.mark.parametrize("t", [F, B])
@pytest.mark.parametrize("d", [32, 33])
def test_strides_counts_and_offsets(t, d):
    """q and out inside wider arrays, sizes on the device, a block that begins at a later destination."""
    g = _gen(4)
    lengths = [(i * 7) % 90 for i in range(60)]
    indptr, idx = _block(lengths, 200, g, masked=0.1)
    store = _store(200, 4, d, 4, g)
    k, v = store.heads(0, 2), store.heads(2, 4)
    q = torch.randn(60, 4, d, generator=g, device="cuda").to(t)
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, k, v, _ws(60, idx.numel(), 4, d))
    wide = torch.full((60, 7, d + 3), 5.0, dtype=t, device="cuda")
    wq = torch.randn(60, 5, d + 3, generator=g, device="cuda").to(t)
    wq[:, 1:, 2:d + 2] = q
    got, _ = gs.gs_coded_attention_forward(indptr, idx, wq[:, 1:, 2:d + 2], k, v, _ws(60, idx.numel(), 4, d), out=wide[:, 2:6, 1:d + 1])
    assert torch.equal(got, out) and (wide[:, :2] == 5).all() and (wide[:, 6:] == 5).all() and (wide[:, :, 0] == 5).all()
    part, plse = gs.gs_coded_attention_forward(indptr[20:], idx, q[20:], k, v, _ws(40, idx.numel(), 4, d))
    assert torch.equal(part, out[20:]) and torch.equal(plse, lse[20:])
    counts = tuple(torch.tensor(c, dtype=torch.int32, device="cuda") for c in (41, 200, int(indptr[41])))
    some, slse = gs.gs_coded_attention_forward(indptr, idx, q, k, v, _ws(60, idx.numel(), 4, d), counts=counts)
    assert torch.equal(some[:41], out[:41]) and (some[41:] == 0).all() and torch.isneginf(slse[41:]).all()
    fewer = tuple(torch.tensor(c, dtype=torch.int32, device="cuda") for c in (60, 120, idx.numel()))
    some, _ = gs.gs_coded_attention_forward(indptr, idx, q, k, v, _ws(60, idx.numel(), 4, d), counts=fewer)
    want = _reference(indptr, idx, q, _values(k), _values(v), d ** -0.5, t, sources=120)
    _check("out", some, want["out"])


@pytest.mark.parametrize("cap", [1, 3])
def test_any_grid(cap):
    g = _gen(5)
    indptr, idx = _block([0, 700, 3] + [11] * 200 + [1500], 300, g)
    store = _store(300, 4, 32, 16, g)
    q = torch.randn(204, 4, 32, generator=g, device="cuda")
    args = (indptr, idx, q, store.heads(0, 2), store.heads(2, 4))
    out, lse = gs.gs_coded_attention_forward(*args, _ws(204, idx.numel(), 4, 32))
    gs.gs_debug_set_grid_cap(cap)
    try:
        again, alse = gs.gs_coded_attention_forward(*args, _ws(204, idx.numel(), 4, 32))
    finally:
        gs.gs_debug_set_grid_cap(0)
    assert torch.equal(out, again) and torch.equal(lse, alse)


def test_values_of_every_size():
    """Scales from 2^-100 to 2^60: scores of nothing, scores in the thousands, sums that do not overflow on the way."""
    g = _gen(6)
    store = gs.gs_coded_rows(64, 2, 32, 1)
    x = torch.randn(64, 2, 32, generator=g, device="cuda")
    x[:, 0] *= torch.exp2(torch.linspace(-100, 9, 64, device="cuda"))[:, None]
    x[:, 1] *= torch.exp2(torch.linspace(60, -100, 64, device="cuda"))[:, None]
    gs.gs_coded_write(store, x)
    indptr = torch.tensor([0, 64, 84, 100], dtype=torch.int32, device="cuda")
    idx = torch.cat([torch.randperm(64, generator=g, device="cuda"), torch.arange(0, 20, device="cuda"), torch.arange(40, 56, device="cuda")]).int()
    q = torch.randn(3, 2, 32, generator=g, device="cuda")
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 1), store.heads(1, 2), _ws(3, 100, 2, 32))
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :1], both[:, 1:], 32 ** -0.5, F)
    _check("out", out, want["out"])
    _check("lse", lse, want["lse"])


def test_no_rows_no_edges():
    store = _store(5, 2, 16, 1, _gen(7))
    k, v = store.heads(0, 1), store.heads(1, 2)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    out, lse = gs.gs_coded_attention_forward(zero, none, torch.empty(0, 2, 16, device="cuda"), k, v, _ws(0, 0, 2, 16))
    assert out.shape == (0, 2, 16)
    out, lse = gs.gs_coded_attention_forward(zero.repeat(3), none, torch.randn(2, 2, 16, device="cuda"), k, v, _ws(2, 0, 2, 16))
    assert (out == 0).all() and torch.isneginf(lse).all()


# Four query heads that share a key head, bf16: the products of the tensor cores.  A weight is held in 22 bits (2^-22 of itself, or
# 2^-49 of the largest) and what is 2^-31 below a query row's largest element in fewer than its 8: both within the bounds above.
@pytest.mark.parametrize("cap", [1, 3])
@pytest.mark.parametrize("d", [16, 64, 100])
def test_any_grid_shared_heads(cap, d):
    g = _gen(8)
    indptr, idx = _block([0, 700, 3] + [11] * 200 + [1500, 16, 17, 32, 33, 0], 300, g, masked=0.1)
    n = indptr.numel() - 1
    store = _store(300, 4, d, 16, g)
    q = torch.randn(n, 8, d, generator=g, device="cuda").to(B)
    args = (indptr, idx, q, store.heads(0, 2), store.heads(2, 4))
    out, lse = gs.gs_coded_attention_forward(*args, _ws(n, idx.numel(), 8, d))
    gs.gs_debug_set_grid_cap(cap)
    try:
        again, alse = gs.gs_coded_attention_forward(*args, _ws(n, idx.numel(), 8, d))
    finally:
        gs.gs_debug_set_grid_cap(0)
    assert torch.equal(out, again) and torch.equal(lse, alse)


def test_values_of_every_size_shared_heads():
    g = _gen(9)
    store = gs.gs_coded_rows(64, 2, 32, 1)
    x = torch.randn(64, 2, 32, generator=g, device="cuda")
    x[:, 0] *= torch.exp2(torch.linspace(-100, 9, 64, device="cuda"))[:, None]
    x[:, 1] *= torch.exp2(torch.linspace(60, -100, 64, device="cuda"))[:, None]
    gs.gs_coded_write(store, x)
    indptr = torch.tensor([0, 64, 84, 100, 101], dtype=torch.int32, device="cuda")
    idx = torch.cat([torch.randperm(64, generator=g, device="cuda"), torch.arange(0, 20, device="cuda"), torch.arange(40, 56, device="cuda"),
                     torch.tensor([63], device="cuda")]).int()
    q = torch.randn(4, 4, 32, generator=g, device="cuda")
    q[:, 1] *= 2.0 ** 20
    q[:, 2] *= 2.0 ** -90
    q[:, 3, 1:] *= 2.0 ** -28
    q = q.to(B)
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 1), store.heads(1, 2), _ws(4, 101, 4, 32))
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :1], both[:, 1:], 32 ** -0.5, B)
    _check("out", out, want["out"])
    _check("lse", lse, want["lse"])
    # one edge: its value as it is, however small
    assert torch.equal(out[3], both[63, 1].to(B).expand(4, 32)) and (out[3] != 0).any()


@pytest.mark.parametrize("hq", [4, 2])
def test_nan_stays_in_its_place(hq):
    """A NaN key makes the rows that meet it NaN in its own key head, a NaN value in its own column; zero queries are no special case."""
    g = _gen(10)
    x = torch.randn(50, 4, 32, generator=g, device="cuda")
    x[7, 0, 3] = float("nan")                                # a key of key head 0
    x[9, 3, 5] = float("inf")                                # a value of key head 1
    store = gs.gs_coded_rows(50, 4, 32, 1)
    gs.gs_coded_write(store, x)
    indptr = torch.tensor([0, 20, 40, 40, 180], dtype=torch.int32, device="cuda")
    idx = (torch.arange(180, device="cuda") % 6 + 10).int()
    idx[5], idx[25], idx[100], idx[101] = 7, 9, 7, 9
    q = torch.randn(4, 2 * hq, 32, generator=g, device="cuda").to(B)
    q[:, hq + 1] = 0
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 2), store.heads(2, 4), _ws(4, 180, 2 * hq, 32))
    bad = torch.isnan(out)
    want = torch.zeros_like(bad)
    want[0, :hq] = want[3, :hq] = True
    want[1, hq:, 5] = want[3, hq:, 5] = True
    assert torch.equal(bad, want) and (out[2] == 0).all()
    sums = torch.zeros(4, 2 * hq, dtype=torch.bool, device="cuda")
    sums[0, :hq] = sums[3, :hq] = True
    assert torch.equal(torch.isnan(lse), sums) and torch.isneginf(lse[2]).all()


@pytest.mark.parametrize("t,hq,hk,d", [(F, 4, 4, 8), (B, 8, 2, 16), (B, 4, 4, 8)])
def test_chunks_of_a_whole_neighbourhood(t, hq, hk, d):
    """So many edges that the chunks are longer than the shortest; rows of a few chunks and of very many beside one another."""
    g = _gen(11)
    indptr, idx = _block([500000, 0, 65, 400, 30000, 1, 120000], 5000, g, masked=0.1)
    n = indptr.numel() - 1
    store = _store(5000, 2 * hk, d, 16, g)
    q = torch.randn(n, hq, d, generator=g, device="cuda").to(t)
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, hk), store.heads(hk, 2 * hk), _ws(n, idx.numel(), hq, d))
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :hk], both[:, hk:], d ** -0.5, t)
    _check("out", out, want["out"])
    _check("lse", lse, want["lse"])


def test_two_captured_graphs_with_one_workspace():
    """Graphs replayed one after the other share a workspace; new inputs in the same places count."""
    g = _gen(12)
    ws = _ws(6, 1500, 8, 32)
    store = _store(300, 4, 32, 16, g)
    calls = []
    for lengths in ([700, 3, 0], [5, 130, 64, 65]):
        indptr, idx = _block(lengths, 300, g)
        calls.append((indptr, idx, torch.randn(len(lengths), 8, 32, generator=g, device="cuda").to(B), store.heads(0, 2), store.heads(2, 4), ws))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs, results = [], []
    with torch.cuda.stream(stream):
        for args in calls:
            gs.gs_coded_attention_forward(*args)
        for args in calls:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                results.append(gs.gs_coded_attention_forward(*args))
            graphs.append(graph)
    torch.cuda.synchronize()
    for again in range(2):
        for args in calls:
            args[2].copy_(torch.randn(args[2].shape, generator=g, device="cuda").to(B))
        ws.fill_(255)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for args, got in zip(calls, results):
            out, lse = gs.gs_coded_attention_forward(*args)
            assert torch.equal(out, got[0]) and torch.equal(lse, got[1])


@pytest.mark.parametrize("hq", [2, 8])
def test_more_chunks_than_edges_allow(hq):
    """Offsets that do not ascend name edges more than once.  The lists have room for the edges once: what does not fit is left out, rows
    that are not cut are as ever, and nothing else is touched."""
    g = _gen(13)
    store = _store(300, 4, 32, 16, g)
    idx = torch.randint(0, 300, (1000,), generator=g, device="cuda", dtype=torch.int32)
    indptr = torch.tensor(([0, 1000] * 40) + [990, 1000], dtype=torch.int32, device="cuda")
    n = indptr.numel() - 1
    q = torch.randn(n, hq, 32, generator=g, device="cuda").to(B)
    need = gs.gs_coded_attention_workspace_bytes(n, 1000, hq, 32)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 2), store.heads(2, 4), ws[:need])
    assert (ws[need:] == 77).all()
    one, _ = gs.gs_coded_attention_forward(indptr[-2:], idx, q[-1:], store.heads(0, 2), store.heads(2, 4), _ws(1, 1000, hq, 32))
    assert torch.equal(out[-1:], one)
