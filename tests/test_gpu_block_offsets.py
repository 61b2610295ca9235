"""A block whose first offset is not 0 - some destinations of a larger block, with its whole array of indices - gives the bits of
the same destinations as a block of their own, forward, reversed and backward."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu


def _pass(indptr, idx, src, q, k, v, do, counts=None):
    ws = torch.randint(0, 256, (gs.gs_block_attention_workspace_bytes(q.shape[0], src, idx.numel(), q.shape[1], k.shape[1], q.shape[2]),),
                       dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, idx, q, k, v, ws, counts=counts)
    ws.random_(0, 256)
    rev = gs.gs_block_reverse(indptr, idx, src, ws, counts=counts)
    ws.random_(0, 256)
    return (out, lse) + gs.gs_block_attention_backward(indptr, idx, rev, q, k, v, out, lse, do, ws, counts=counts), rev


@pytest.mark.parametrize("t,hq,hk,d", [(torch.float32, 4, 2, 16), (torch.bfloat16, 2, 1, 24), (torch.float32, 2, 2, 7)])
@pytest.mark.parametrize("rows,longest,src", [(60, 9, 100), (2000, 12, 700), (20000, 10, 9000), (300, 200, 100), (50, 5, 3000)])
@pytest.mark.parametrize("device_counts", [False, True])
def test_part_of_a_block(t, hq, hk, d, rows, longest, src, device_counts):
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    indptr = torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = torch.randint(0, longest + 1, (rows,), generator=g, device="cuda").cumsum(0).int()
    idx = torch.randint(-1, src + 1, (int(indptr[-1]),), generator=g, device="cuda", dtype=torch.int32)
    a, b = rows // 3, rows - rows // 5
    n, first, last = b - a, int(indptr[a]), int(indptr[b])
    mk = lambda r, h: torch.randn(r, h, d, generator=g, device="cuda").to(t)  # noqa: E731
    q, k, v, do = mk(n, hq), mk(src, hk), mk(src, hk), mk(n, hq)
    want, rev = _pass(indptr[a:b + 1] - first, idx[first:last].clone(), src, q, k, v, do)
    counts = tuple(torch.tensor(c, dtype=torch.int32, device="cuda") for c in (n, src, idx.numel())) if device_counts else None
    got, part = _pass(indptr[a:b + 1].clone(), idx, src, q, k, v, do, counts)
    live = int(rev[0][-1])
    assert torch.equal(part[0], rev[0]) and torch.equal(part[1][:live], rev[1][:live]) and torch.equal(part[2][:live] - first, rev[2][:live])
    assert all(torch.equal(x, y) for x, y in zip(got, want))
