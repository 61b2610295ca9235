"""Backward pass of rows with scores of -inf: rows that have nothing else have no part in any gradient, as masked rows have none;
an edge with such a score beside finite ones has no part either.  The gradients are bit for bit those of the block whose
edges of these scores are masked."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
INF = float("inf")


def _pass(indptr, idx, q, k, v, do, **kw):
    n, hq, d = q.shape
    ws = torch.empty(gs.gs_block_attention_workspace_bytes(n, k.shape[0], idx.numel(), hq, k.shape[1], d), dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, idx, q, k, v, ws, **kw)
    rev = gs.gs_block_reverse(indptr, idx, k.shape[0], ws)
    dq, dk, dv = gs.gs_block_attention_backward(indptr, idx, rev, q, k, v, out, lse, do, ws, **kw)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hk,d", [(1, 1, 8), (4, 2, 16), (8, 2, 24), (3, 3, 33), (2, 1, 100), (2, 1, 7), (1, 1, 256)])
@pytest.mark.parametrize("long_row", [0, 300])
def test_scores_of_minus_infinity(t, hq, hk, d, long_row):
    g = torch.Generator(device="cuda").manual_seed(d + long_row)
    src = 40                                          # sources 30 .. 39 have keys of -inf
    lengths = [5, 7, 4, 0, 6, 3 + long_row, 2 + long_row, 9]
    indptr = torch.zeros(len(lengths) + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = torch.tensor(lengths, device="cuda").cumsum(0).int()
    idx = torch.randint(0, 30, (int(indptr[-1]),), generator=g, device="cuda", dtype=torch.int32)
    row = lambda i: slice(int(indptr[i]), int(indptr[i + 1]))  # noqa: E731
    dead = [1, 5]                                     # all scores -inf, by the keys
    for i in dead:
        idx[row(i)] = torch.randint(30, 40, (lengths[i],), generator=g, device="cuda", dtype=torch.int32)
    idx[row(4)][::2] = 33                             # some scores -inf
    idx[row(6)][::3] = 31
    mk = lambda r, h: torch.randn(r, h, d, generator=g, device="cuda").to(t)  # noqa: E731
    q, k, v, do = mk(len(lengths), hq).abs() + 0.1, mk(src, hk), mk(src, hk), mk(len(lengths), hq)
    k[30:] = -INF
    for kw in (dict(), dict(max_row=max(lengths))):
        got = _pass(indptr, idx, q, k, v, do, **kw)
        masked = idx.clone()
        masked[idx >= 30] = -1
        want = _pass(indptr, masked, q, k, v, do, **kw)
        for name in got:
            assert torch.equal(got[name], want[name]), name
        for i in dead:
            assert (got["out"][i] == 0).all() and torch.isneginf(got["lse"][i]).all() and (got["dq"][i] == 0).all()
        assert (got["dk"][30:] == 0).all() and (got["dv"][30:] == 0).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [16, 7])
def test_query_and_upstream_gradient_of_a_dead_row_may_be_infinite(t, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    indptr = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    idx = torch.tensor([0, 1, 2, 2, 1, 3], dtype=torch.int32, device="cuda")
    mk = lambda r: torch.randn(r, 2, d, generator=g, device="cuda").to(t)  # noqa: E731
    q, k, v, do = mk(2), mk(4).abs() + 0.1, mk(4), mk(2)
    q[1], do[1] = -INF, INF                           # the second row's scores are all -inf
    got = _pass(indptr, idx, q, k, v, do)
    idx[3:] = -1
    want = _pass(indptr, idx, q, k, v, do)
    for name in got:
        assert torch.equal(got[name], want[name]), name
    assert all(torch.isfinite(got[n]).all() for n in ("dq", "dk", "dv"))
