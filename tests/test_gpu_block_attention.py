"""Attention over a block, forward and backward, against 64-bit references.

Bounds, derived from the 32-bit arithmetic (u = 2^-24; h: half an ulp of the output type, 2^-8 for bf16):
a score is off by at most (D + 4) u scale sum|q||k|, an exponential by 2^-21 relative, a sum of n terms by n u of its
magnitudes.  With E = 4 ((D + 4) u max_e scale sum|q||k| + 2^-21 + (n + 4) u) bounding a probability's relative error:
  out: E sum p|v| + h |out|;  lse: E + 2^-23 |lse|
  delta: sum|do| (E sum p|v| + h |out|) + D u sum |do||out|;  ds: scale p (E (|dp| + |delta|) + D u sum|do||v| + delta's)
  dq, dk: sum of ds's |k| (|q|) + (n + 2) u sum|ds||k|, + h |.|;  dv: sum E p |do| + (n + 2) u sum p|do| + h |dv|."""
import math

import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _block(lengths, src, g, masked=0.0):
    indptr = torch.zeros(len(lengths) + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = torch.tensor(lengths, device="cuda").cumsum(0).int()
    e = int(indptr[-1])
    idx = (torch.rand(e, generator=g, device="cuda") ** 2 * src).int().clamp_(max=src - 1)
    off = torch.rand(e, generator=g, device="cuda") < masked
    idx[off] = torch.where(torch.rand(e, generator=g, device="cuda") < 0.5, -1, src + 5).int()[off]
    return indptr, idx


def _reference(indptr, idx, q, k, v, do, scale, t):
    h = HALF_ULP[t]
    n, hq, d = q.shape
    src, hk = k.shape[0], k.shape[1]
    keep = (idx >= 0) & (idx < src)
    dst = torch.repeat_interleave(torch.arange(n, device="cuda"), (indptr[1:] - indptr[:-1]).long())[keep]
    j = idx[keep].long()
    q, do = q.double(), do.double()
    kx = k.double()[j].repeat_interleave(hq // hk, 1)
    vx = v.double()[j].repeat_interleave(hq // hk, 1)
    cnt = torch.zeros(n, 1, dtype=torch.float64, device="cuda").index_add_(0, dst, torch.ones(len(dst), 1, dtype=torch.float64, device="cuda"))

    def rows(x):
        return torch.zeros((n,) + x.shape[1:], dtype=torch.float64, device="cuda").index_add_(0, dst, x)

    def cols(x):                                     # sums over destinations and over the heads that share a source head
        x = x.view(x.shape[0], hk, hq // hk, d).sum(2)
        return torch.zeros(src, hk, d, dtype=torch.float64, device="cuda").index_add_(0, j, x)

    s = (q[dst] * kx).sum(-1) * scale
    smag = (q[dst].abs() * kx.abs()).sum(-1) * abs(scale)
    top = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce(0, dst[:, None].expand_as(s), s, "amax")
    tmag = torch.zeros((n, hq), dtype=torch.float64, device="cuda").scatter_reduce(0, dst[:, None].expand_as(s), smag, "amax")
    w = torch.exp(s - top[dst])
    tot = rows(w)
    p = w / tot[dst]
    lse = top + torch.log(tot)
    out = rows(p[..., None] * vx)
    E = 4 * ((d + 4) * U * tmag + 2.0 ** -21 + (cnt + 4) * U)
    pv = rows(p[..., None] * vx.abs())
    r = {"out": (out, E[..., None] * pv + h * out.abs()), "lse": (lse, E + 2.0 ** -23 * lse.abs())}
    delta = (do * out).sum(-1)
    derr = (do.abs() * (E[..., None] * pv + h * out.abs())).sum(-1) + d * U * (do.abs() * out.abs()).sum(-1)
    dp = (do[dst] * vx).sum(-1)
    ds = p * (dp - delta[dst]) * scale
    dserr = abs(scale) * p * (E[dst] * (dp.abs() + delta[dst].abs()) + d * U * (do[dst].abs() * vx.abs()).sum(-1) + derr[dst])
    deg = torch.zeros(src, 1, 1, dtype=torch.float64, device="cuda").index_add_(0, j, torch.ones(len(j), 1, 1, dtype=torch.float64, device="cuda")) * (hq // hk)
    dq, dk, dv = rows(ds[..., None] * kx), cols(ds[..., None] * q[dst]), cols(p[..., None] * do[dst])
    r["dq"] = (dq, rows(dserr[..., None] * kx.abs()) + (cnt[..., None] + 2) * U * rows((ds[..., None] * kx).abs()) + h * dq.abs())
    r["dk"] = (dk, cols(dserr[..., None] * q[dst].abs()) + (deg + 2) * U * cols((ds[..., None] * q[dst]).abs()) + h * dk.abs())
    r["dv"] = (dv, cols(E[dst][..., None] * p[..., None] * do[dst].abs()) + (deg + 2) * U * cols((p[..., None] * do[dst]).abs()) + h * dv.abs())
    return r


def _check(name, got, want):
    ref, slack = want
    got = got.double()
    if name == "lse":
        empty = torch.isinf(ref)
        assert torch.equal(torch.isneginf(got), empty)
        got, ref, slack = got[~empty], ref[~empty], slack[~empty]
    bad = (got - ref).abs() > slack * 1.01 + 1e-30
    assert not bad.any(), "%s: %d off, worst %g" % (name, int(bad.sum()), float(((got - ref).abs() / (slack + 1e-30)).max()))


def _run(indptr, idx, q, k, v, do, scale=None, max_row=0, **kw):
    ws = torch.randint(0, 256, (gs.gs_block_attention_workspace_bytes(q.shape[0], k.shape[0], idx.numel(), q.shape[1], k.shape[1], q.shape[2]),),
                       dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, idx, q, k, v, ws, scale=scale, max_row=max_row, **kw)
    rev = gs.gs_block_reverse(indptr, idx, k.shape[0], ws, **kw)
    dq, dk, dv = gs.gs_block_attention_backward(indptr, idx, rev, q, k, v, out, lse, do, ws, scale=scale, max_row=max_row, **kw)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv), rev


def _inputs(n, src, hq, hk, d, t, g):
    mk = lambda r, h: torch.randn(r, h, d, generator=g, device="cuda").to(t)  # noqa: E731
    return mk(n, hq), mk(src, hk), mk(src, hk), mk(n, hq)


LENGTHS = {
    "one": [1], "empty": [0, 0, 0], "few": [5, 0, 3, 1, 0, 4], "fan": None,
    "hub": [0, 700, 3, 256, 257, 1, 5000], "long": [9000],
}
SHAPES = [(1, 1, 8), (4, 4, 16), (4, 2, 32), (8, 1, 24), (8, 8, 16), (3, 3, 33), (6, 2, 20), (2, 1, 128), (1, 1, 256), (5, 1, 7), (4, 4, 100), (2, 2, 130), (12, 3, 64)]


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hk,d", SHAPES)
@pytest.mark.parametrize("kind", sorted(LENGTHS))
def test_against_definition(t, hq, hk, d, kind):
    g = _gen(hq * 1000 + d)
    lengths = LENGTHS[kind] or [(i * 7) % 21 for i in range(300)]
    src = 37 if kind in ("few", "one", "empty") else 400
    indptr, idx = _block(lengths, src, g, masked=0.15 if kind != "one" else 0.0)
    q, k, v, do = _inputs(len(lengths), src, hq, hk, d, t, g)
    scale = 0.7 / math.sqrt(d)
    ref = _reference(indptr, idx, q, k, v, do, scale, t)
    got, rev = _run(indptr, idx, q, k, v, do, scale)
    for name, want in ref.items():
        _check(name, got[name], want)
    # the reversed block, exactly
    keep = (idx >= 0) & (idx < src)
    dst = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), (indptr[1:] - indptr[:-1]).long())[keep]
    order = torch.argsort(idx[keep].long(), stable=True)
    assert torch.equal(rev[1][:len(order)].long(), dst[order])
    assert torch.equal(rev[0].long(), torch.searchsorted(idx[keep].long()[order], torch.arange(src + 1, device="cuda")))
    again, _ = _run(indptr, idx, q, k, v, do, scale)
    assert all(torch.equal(got[n], again[n]) for n in got)           # same bits every time
    hinted, _ = _run(indptr, idx, q, k, v, do, scale, max_row=max(max(lengths), 1))
    for name, want in ref.items():
        _check(name, hinted[name], want)
    # a promise that does not hold costs time, not correctness
    if kind == "hub":
        wrong, _ = _run(indptr, idx, q, k, v, do, scale, max_row=4)
        for name, want in ref.items():
            _check(name, wrong[name], want)
    gs.gs_train_status()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_strided_operands(t):
    """Slices of fused projections: [rows, 3, heads, dim] and [rows, heads, 3 dim], odd row pitches."""
    g = _gen(3)
    lengths = [(i * 5) % 17 for i in range(70)]
    indptr, idx = _block(lengths, 90, g, 0.1)
    for d in (16, 24, 15):
        fused = torch.randn(90, 3, 4, d, generator=g, device="cuda").to(t)
        wide = torch.randn(90, 4, 3 * d + 1, generator=g, device="cuda").to(t)
        for q, k, v in ((fused[:70, 0], fused[:, 1], fused[:, 2]), (wide[:70, :, :d], wide[:, :, d:2 * d], wide[:, :, 2 * d:3 * d])):
            do = torch.randn(70, 4, d + 3, generator=g, device="cuda").to(t)[:, :, :d]
            a, _ = _run(indptr, idx, q, k, v, do)
            b, _ = _run(indptr, idx, q.contiguous(), k.contiguous(), v.contiguous(), do.contiguous())
            ref = _reference(indptr, idx, q, k, v, do, d ** -0.5, t)
            for name, want in ref.items():
                _check(name, a[name], want)
                _check(name, b[name], want)


def test_masked_rows_are_not_read_and_extremes():
    """NaN and infinity where only masked edges point; scores of -inf among finite ones; a row of -inf alone."""
    d = 8
    q = torch.ones(4, 1, d, device="cuda")
    k = torch.zeros(6, 1, d, device="cuda")
    v = torch.arange(6, device="cuda").float().view(6, 1, 1).expand(6, 1, d).contiguous()
    k[5], v[5] = float("nan"), float("inf")
    k[4] = -float("inf")
    indptr = torch.tensor([0, 3, 5, 6, 8], dtype=torch.int32, device="cuda")
    idx = torch.tensor([1, -1, 3, 4, 2, -7, 4, 4], dtype=torch.int32, device="cuda")
    ws = torch.empty(gs.gs_block_attention_workspace_bytes(4, 6, 8, 1, 1, d), dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, idx, q, k, v, ws)
    assert torch.equal(out[0], torch.full((1, d), 2.0, device="cuda")) and torch.equal(out[1], torch.full((1, d), 2.0, device="cuda"))
    assert (out[2] == 0).all() and torch.isneginf(lse[2]).all()
    assert (out[3] == 0).all() and torch.isneginf(lse[3]).all()
    assert abs(float(lse[0]) - math.log(2)) < 1e-6 and abs(float(lse[1])) < 1e-6
    low = torch.finfo(torch.float32).min
    k[1], k[3] = low / d, low / d                     # scores near the type's lowest value: still a uniform softmax
    out, lse = gs.gs_block_attention_forward(indptr, idx, q, k, v, ws, scale=0.5)
    assert torch.equal(out[0], torch.full((1, d), 2.0, device="cuda")) and torch.isfinite(lse[0]).all()


def test_device_counts_and_capped_grids():
    g = _gen(9)
    lengths = [(i * 11) % 40 for i in range(200)] + [900]
    indptr, idx = _block(lengths, 333, g, 0.05)
    q, k, v, do = _inputs(201, 333, 4, 2, 16, torch.float32, g)
    whole, rev = _run(indptr, idx, q, k, v, do)
    # the same block at the front of larger arrays whose tails hold anything
    ip = torch.cat([indptr, torch.randint(-5, 1 << 20, (40,), device="cuda", dtype=torch.int32)])
    ix = torch.cat([idx, torch.randint(-5, 400, (77,), device="cuda", dtype=torch.int32)])
    big = lambda x, r: torch.cat([x, torch.full((r,) + x.shape[1:], float("nan"), device="cuda")])  # noqa: E731
    counts = tuple(torch.tensor(c, dtype=torch.int32, device="cuda") for c in (201, 333, idx.numel()))
    try:
        for cap in (0, 1, 3):
            gs.gs_debug_set_grid_cap(cap)
            got, r2 = _run(ip, ix, big(q, 40), big(k, 60), big(v, 60), big(do, 40), counts=counts)
            assert torch.equal(r2[0][:334], rev[0]) and torch.equal(r2[1][:int(rev[0][-1])], rev[1][:int(rev[0][-1])])
            for n, rows in (("out", 201), ("lse", 201), ("dq", 201), ("dk", 333), ("dv", 333)):
                assert torch.allclose(got[n][:rows], whole[n], rtol=1e-5, atol=1e-6), n
    finally:
        gs.gs_debug_set_grid_cap(0)


def test_sampled_block_end_to_end():
    """A block as gs_sample_batch leaves it (device counts, arrays at their bounds) goes straight in."""
    from workloads import batch_seeds, build_graph, get_config, seed_permutation

    cfg = get_config("tiny")
    gr = build_graph(cfg).to("cuda")
    G = gs.gs_graph_create(gr.indptr, gr.indices, None)
    cache = gs.gs_cache_init(G, cfg["fanouts"], cfg["cache_width"], 7, False)
    sws = torch.empty(gs.gs_workspace_bytes(G, cfg["fanouts"], cfg["batch"]), dtype=torch.uint8, device="cuda")
    seeds = batch_seeds(seed_permutation(cfg), 0, cfg["batch"]).to("cuda")
    blocks, _, _ = gs.gs_sample_batch(cache, seeds, gs.GS_MODE_OTF, 0.25, 1, sws)
    g = _gen(1)
    for b in blocks:
        counts = b.counts_device()
        n, s, e = (int(c) for c in counts)
        q, k, v, do = _inputs(b.max_dst, b.max_src, 4, 4, 16, torch.float32, g)
        got, _ = _run(b.indptr(b.max_dst), b.indices(b.max_edges), q, k, v, do, max_row=max(cfg["fanouts"]), counts=counts)
        ref = _reference(b.indptr(n), b.indices(e), q[:n], k[:s], v[:s], do[:n], 0.25, torch.float32)
        for name, want in ref.items():
            _check(name, got[name][:want[0].shape[0]], want)


def test_gradients_are_the_derivatives():
    """Central differences of the 64-bit loss <out, do> along random directions, step 1e-6: truncation is of order
    1e-12, so the directional derivatives agree to the 32-bit bounds (1e-4 relative is ten times those here)."""
    g = _gen(12)
    lengths = [4, 0, 7, 2, 9, 1]
    indptr, idx = _block(lengths, 11, g, 0.1)
    q, k, v, do = _inputs(6, 11, 4, 2, 12, torch.float32, g)
    got, _ = _run(indptr, idx, q, k, v, do)

    def loss(q, k, v):
        return (_reference(indptr, idx, q, k, v, do, 12 ** -0.5, torch.float32)["out"][0] * do.double()).sum()

    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        way = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        args = {"dq": q.double(), "dk": k.double(), "dv": v.double()}
        plus, minus = dict(args), dict(args)
        plus[name], minus[name] = args[name] + 1e-6 * way, args[name] - 1e-6 * way
        slope = (loss(*plus.values()) - loss(*minus.values())) / 2e-6
        mine = (got[name].double() * way).sum()
        assert abs(slope - mine) <= 1e-4 * (got[name].double() * way).abs().sum()


def test_refusals():
    g = _gen(2)
    indptr, idx = _block([2, 1], 5, g)
    q, k, v, do = _inputs(2, 5, 4, 2, 16, torch.float32, g)
    ws = torch.empty(gs.gs_block_attention_workspace_bytes(2, 5, 3, 4, 2, 16), dtype=torch.uint8, device="cuda")
    fwd = lambda *a, **kw: gs.gs_block_attention_forward(*a, **kw)  # noqa: E731
    with pytest.raises(TypeError):
        fwd(indptr.long(), idx, q, k, v, ws)
    with pytest.raises(TypeError):
        fwd(indptr, idx, q, k.bfloat16(), v, ws)
    with pytest.raises(TypeError):
        fwd(indptr, idx, q.half(), k.half(), v.half(), ws)
    with pytest.raises(TypeError):
        fwd(indptr, idx, q, k, v[:4], ws)
    with pytest.raises(ValueError):
        fwd(indptr, idx, q[:1], k, v, ws)
    for bad, status in ((dict(q=q[:, :3]), 1), (dict(ws=ws[:256]), 4), (dict(ws=torch.empty(ws.numel() + 8, dtype=torch.uint8, device="cuda")[8:]), 2), (dict(max_row=-1), 1)):
        args = dict(q=q, ws=ws, max_row=0, **{})
        args.update(bad)
        with pytest.raises(gs.GsError) as e:
            fwd(indptr, idx, args["q"], k, v, args["ws"], max_row=args["max_row"])
        assert e.value.status == status
    wide = torch.zeros(2, 1, 257, device="cuda")
    with pytest.raises(gs.GsError):
        fwd(indptr, idx, wide, torch.zeros(5, 1, 257, device="cuda"), torch.zeros(5, 1, 257, device="cuda"), ws)
