"""dq and dk of bf16 operands: delta = do . o does not take over the rounding of `out` to bf16, which rows of one or two edges,
or with one probability near 1, would show in full (a row of one edge has no gradient through its score at all).

The bounds are those of the 32-bit arithmetic alone (test_gpu_block_attention.py, without its term h |out| in delta).  The
sums run over p (dp - delta') with delta' off by up to t = h sum|do||o|, and over p k, and are corrected by
r = sum p (dp - delta'): each of these adds (n + 4) u p t per edge, and r lacks t |1 - sum p| <= t E."""
import math

import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8


def _reference(indptr, idx, q, k, v, do, scale):
    n, hq, d = q.shape
    src, hk = k.shape[0], k.shape[1]
    dst = torch.repeat_interleave(torch.arange(n, device="cuda"), (indptr[1:] - indptr[:-1]).long())
    j = idx.long()
    q, do = q.double(), do.double()
    kx, vx = (x.double()[j].repeat_interleave(hq // hk, 1) for x in (k, v))
    rows = lambda x: torch.zeros((n,) + x.shape[1:], dtype=torch.float64, device="cuda").index_add_(0, dst, x)  # noqa: E731
    cols = lambda x: torch.zeros(src, hk, d, dtype=torch.float64, device="cuda").index_add_(0, j, x.view(-1, hk, hq // hk, d).sum(2))  # noqa: E731
    cnt = rows(torch.ones(len(j), 1, dtype=torch.float64, device="cuda"))
    s = (q[dst] * kx).sum(-1) * scale
    top = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce(0, dst[:, None].expand_as(s), s, "amax")
    tmag = torch.zeros((n, hq), dtype=torch.float64, device="cuda").scatter_reduce(0, dst[:, None].expand_as(s), (q[dst].abs() * kx.abs()).sum(-1) * scale, "amax")
    w = torch.exp(s - top[dst])
    p = w / rows(w)[dst]
    out, pv = rows(p[..., None] * vx), rows(p[..., None] * vx.abs())
    E = 4 * ((d + 4) * U * tmag + 2.0 ** -21 + (cnt + 4) * U)
    delta, mag = (do * out).sum(-1), (do.abs() * out.abs()).sum(-1)
    t = H * mag
    dp = (do[dst] * vx).sum(-1)
    ds = p * (dp - delta[dst]) * scale
    derr = E * (do.abs() * pv).sum(-1) + d * U * mag + t * (E + (cnt + 4) * U)
    dserr = scale * p * (E[dst] * (dp.abs() + delta[dst].abs() + t[dst]) + d * U * (do[dst].abs() * vx.abs()).sum(-1) + derr[dst] + (cnt[dst] + 4) * U * t[dst])
    deg = torch.zeros(src, 1, 1, dtype=torch.float64, device="cuda").index_add_(0, j, torch.ones(len(j), 1, 1, dtype=torch.float64, device="cuda")) * (hq // hk)
    dq, dk = rows(ds[..., None] * kx), cols(ds[..., None] * q[dst])
    return {"dq": (dq, rows(dserr[..., None] * kx.abs()) + (cnt[..., None] + 2) * U * rows((ds[..., None] * kx).abs()) + H * dq.abs()),
            "dk": (dk, cols(dserr[..., None] * q[dst].abs()) + (deg + 2) * U * cols((ds[..., None] * q[dst]).abs()) + H * dk.abs())}


@pytest.mark.parametrize("hq,hk,d", [(1, 1, 8), (4, 4, 32), (8, 2, 24), (2, 1, 128), (3, 3, 33), (6, 2, 20), (2, 1, 7), (1, 1, 256), (4, 2, 100), (12, 3, 64)])
@pytest.mark.parametrize("kind", ["one", "two", "peaked", "long"])
def test_gradients_do_not_show_the_rounding_of_out(hq, hk, d, kind):
    g = torch.Generator(device="cuda").manual_seed(d + hq)
    lengths = {"one": [1] * 60, "two": [1, 2] * 40, "peaked": [(i * 7) % 21 for i in range(80)], "long": [1, 700, 2, 65, 64, 300]}[kind]
    src, t = 90, torch.bfloat16
    indptr = torch.zeros(len(lengths) + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = torch.tensor(lengths, device="cuda").cumsum(0).int()
    idx = torch.randint(0, src, (int(indptr[-1]),), generator=g, device="cuda", dtype=torch.int32)
    mk = lambda r, h: torch.randn(r, h, d, generator=g, device="cuda")  # noqa: E731
    q, k, v, do = (x.to(t) for x in (mk(len(lengths), hq) * (4.0 if kind in ("peaked", "long") else 1.0), mk(src, hk), mk(src, hk), mk(len(lengths), hq)))
    scale = d ** -0.5
    for max_row in (0, max(lengths)):
        ws = torch.randint(0, 256, (gs.gs_block_attention_workspace_bytes(len(lengths), src, idx.numel(), hq, hk, d),), dtype=torch.uint8, device="cuda")
        out, lse = gs.gs_block_attention_forward(indptr, idx, q, k, v, ws, max_row=max_row)
        rev = gs.gs_block_reverse(indptr, idx, src, ws)
        dq, dk, _ = gs.gs_block_attention_backward(indptr, idx, rev, q, k, v, out, lse, do, ws, max_row=max_row)
        for name, got, (ref, slack) in zip(("dq", "dk"), (dq, dk), _reference(indptr, idx, q, k, v, do, scale).values()):
            off = (got.double() - ref).abs()
            assert (off <= slack * 1.01 + 1e-30).all(), "%s: %d off, worst %g of the bound" % (name, int((off > slack * 1.01).sum()), float((off / (slack + 1e-30)).max()))
