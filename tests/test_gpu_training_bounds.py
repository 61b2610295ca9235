"""Arrays at their bounds, with the actual sizes on the device, through autograd: rows behind the sizes are zeros in results
and gradients, so that what stands in front (a projection, here) gets the gradient of the rows that exist.  The memory the
results are made in is filled with NaN first."""
import pytest
import torch

import paper_2406_17918_b200 as gs
from paper_2406_17918_b200.autograd import block_attention, embedding

pytestmark = pytest.mark.gpu
N, SRC, HEADS, DIM = 50, 130, 4, 16            # what the block has
MORE_N, MORE_SRC, MORE_E = 70, 190, 60         # what the arrays hold beyond it


@pytest.fixture
def nan_memory():
    """Freed memory of every size that is used here holds NaN."""
    torch.cuda.empty_cache()
    for shift in range(8, 25):
        held = [torch.full((1 << shift >> 2,), float("nan"), device="cuda") for _ in range(12 if shift < 20 else 3)]
        del held
    torch.cuda.synchronize()


def _block():
    g = torch.Generator(device="cuda").manual_seed(2)
    lengths = torch.randint(0, 9, (N,), generator=g, device="cuda")
    lengths[7] = 100                                          # a row that is split
    indptr = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = lengths.cumsum(0).int()
    e = int(indptr[-1])
    indices = torch.randint(-1, SRC, (e,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn(SRC, 24, generator=g, device="cuda")
    weight = torch.randn(24, 3 * HEADS * DIM, generator=g, device="cuda") * 0.2
    do = torch.randn(N, HEADS, DIM, generator=g, device="cuda")
    return indptr, indices, x, weight, do


def _grads(indptr, indices, x, weight, do, rows, t, **kw):
    x, weight = x.clone().to(t).requires_grad_(), weight.clone().to(t).requires_grad_()
    qkv = (x @ weight).view(x.shape[0], 3, HEADS, DIM)
    out = block_attention(qkv[:rows, 0], qkv[:, 1], qkv[:, 2], indptr, indices, **kw)
    out.backward(do.to(t))
    return out.detach(), x.grad, weight.grad


def _tail(x, rows, value):
    return torch.cat([x, torch.full((rows,) + x.shape[1:], value, dtype=x.dtype, device="cuda")])


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_device_counts(t, nan_memory):
    indptr, indices, x, weight, do = _block()
    want, want_x, want_w = _grads(indptr, indices, x, weight, do, N, t)
    counts = tuple(torch.tensor(c, dtype=torch.int32, device="cuda") for c in (N, SRC, indices.numel()))
    # the upstream rows behind the sizes may hold anything finite: they meet gradients of zero
    out, dx, dw = _grads(_tail(indptr, MORE_N, 5), _tail(indices, MORE_E, 3), _tail(x, MORE_SRC, 1e3), weight, _tail(do, MORE_N, 1e3), N + MORE_N, t,
                         counts=counts)
    assert torch.equal(out[:N], want) and (out[N:] == 0).all()
    assert torch.equal(dx[:SRC], want_x) and (dx[SRC:] == 0).all()
    tol = 1e-5 if t == torch.float32 else 2e-2                # the projection's product has other tiles
    assert torch.isfinite(dw).all() and (dw - want_w).norm() <= tol * want_w.norm()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_more_query_rows_than_destinations(t, nan_memory):
    indptr, indices, x, weight, do = _block()
    _, want_x, want_w = _grads(indptr, indices, x, weight, do, N, t)
    x2, w2 = x.clone().to(t).requires_grad_(), weight.clone().to(t).requires_grad_()
    qkv = (x2 @ w2).view(SRC, 3, HEADS, DIM)
    out = block_attention(qkv[:, 0], qkv[:, 1], qkv[:, 2], indptr, indices)
    assert out.shape[0] == SRC and (out[N:] == 0).all()
    out[:N].backward(do.to(t))
    assert torch.equal(x2.grad, want_x) and torch.equal(w2.grad, want_w)


def test_binding_with_more_rows(nan_memory):
    indptr, indices, x, _, do = _block()
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(r, HEADS, DIM, generator=g, device="cuda") for r in (N + 9, SRC, SRC + 11))
    ws = torch.empty(gs.gs_block_attention_workspace_bytes(N, SRC, indices.numel(), HEADS, HEADS, DIM), dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, indices, q, k, v, ws)
    assert (out[N:] == 0).all() and torch.isneginf(lse[N:]).all()
    rev = gs.gs_block_reverse(indptr, indices, SRC, ws)
    dq, dk, dv = gs.gs_block_attention_backward(indptr, indices, rev, q, k, v, out, lse, _tail(do, 9, 7.0), ws)
    assert (dq[N:] == 0).all() and (dv[SRC:] == 0).all()
    assert all(torch.isfinite(d).all() for d in (dq, dk, dv))


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("live", [0, 1, 77, 100])
def test_embedding_count(t, live, nan_memory):
    g = torch.Generator(device="cuda").manual_seed(4)
    ids = torch.randint(0, 40, (100,), generator=g, device="cuda", dtype=torch.int32)
    leaf = torch.randn(40, 24, generator=g, device="cuda").to(t)
    weight = torch.randn(24, 8, generator=g, device="cuda").to(t).requires_grad_()
    table = leaf.clone().requires_grad_()
    x = embedding(table, ids, scale=2.0, count=torch.tensor(live, dtype=torch.int32, device="cuda"))
    assert (x[live:] == 0).all()
    (x @ weight).sum().backward()
    # all upstream gradients are one: sums over the live rows, exact to a few roundings
    rows = (leaf.double()[ids[:live].long()] * 2.0).to(t).double().sum(0)
    assert torch.isfinite(weight.grad).all() and torch.isfinite(table.grad).all()
    assert ((weight.grad.double() - rows[:, None]).abs() <= (1e-4 if t == torch.float32 else 0.5) + 1e-2 * rows.abs()[:, None]).all()
    hit = torch.zeros(40, dtype=torch.bool, device="cuda")
    hit[ids[:live].long()] = True
    assert (table.grad[~hit] == 0).all()
