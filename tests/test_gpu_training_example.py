"""The operators together: the example's model against the same model in elementary operations, and a short training."""
import os
import sys

import pytest
import torch

import paper_2406_17918_b200 as gs
from paper_2406_17918_b200.autograd import block_attention, embedding, table_cross_entropy

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _plain_attention(q, k, v, indptr, indices):
    n, heads, dim = q.shape
    dst = torch.repeat_interleave(torch.arange(n, device=q.device), (indptr[1:] - indptr[:-1]).long())
    src = indices.long()
    s = (q[dst] * k[src]).sum(-1) / dim ** 0.5
    p = torch.zeros(n, heads, dtype=q.dtype, device=q.device)
    top = torch.full_like(p, -float("inf")).scatter_reduce(0, dst[:, None].expand_as(s), s.detach(), "amax")
    w = torch.exp(s - top[dst])
    total = p.index_add(0, dst, w)
    return torch.zeros(n, heads, dim, dtype=q.dtype, device=q.device).index_add(0, dst, (w / total[dst])[..., None] * v[src])


def test_functions_compose_like_elementary_operations():
    """One layer and the loss, f32: gradients of every parameter against 64-bit autograd.  A gradient passes through three
    32-bit operators of at most a few hundred terms each: 1e-4 of its norm is a hundred times their rounding."""
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    n, src, edges, width, vocab = 30, 80, 300, 32, 90
    dst = torch.randint(0, n, (edges,), generator=g, device="cuda").sort().values
    indptr = torch.searchsorted(dst, torch.arange(n + 1, device="cuda")).int()
    indices = torch.randint(0, src, (edges,), generator=g, device="cuda", dtype=torch.int32)
    ids = torch.randint(0, vocab, (src,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(-1, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    leaves = [torch.randn(s, generator=g, device="cuda") * 0.3 for s in ((vocab, width), (width, 3 * width), (vocab, width))]
    mine = [x.clone().requires_grad_() for x in leaves]
    ref = [x.double().requires_grad_() for x in leaves]

    x = embedding(mine[0], ids, scale=2.0)
    qkv = (x @ mine[1]).view(src, 3, 4, 8)
    h = block_attention(qkv[:n, 0], qkv[:, 1], qkv[:, 2], indptr, indices, max_row=64)
    loss = table_cross_entropy(x[:n] + h.reshape(n, width), mine[2], labels).sum()
    loss.backward()

    xr = ref[0][ids.long()] * 2.0
    qr = (xr @ ref[1]).view(src, 3, 4, 8)
    hr = xr[:n] + _plain_attention(qr[:n, 0], qr[:, 1], qr[:, 2], indptr, indices).reshape(n, width)
    z = hr @ ref[2].t()
    keep = labels >= 0
    lr = torch.nn.functional.cross_entropy(z[keep], labels[keep].long(), reduction="sum")
    lr.backward()
    assert abs(loss.double() - lr) <= 1e-5 * lr
    for a, b in zip(mine, ref):
        assert (a.grad.double() - b.grad).norm() <= 1e-4 * b.grad.norm()


def test_short_training_learns():
    from train_context_nodes import train

    before = gs.gs_kernel_launches()
    history = train("tiny", steps=40, log=lambda *a: None)
    assert all(x == x and x < 50 for x in history)
    assert sum(history[-5:]) < sum(history[:5]) - 1.0        # forty steps over the same few thousand nodes
    assert gs.gs_kernel_launches() > before + 40 * 10
