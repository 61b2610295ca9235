"""The differentiable wrappers on the CPU, over stand-ins for the library's calls: gradients are first derivatives, and asking
for a second one is an error, not a constant."""
import types

import pytest
import torch

from paper_2406_17918_b200 import autograd


def _stand_ins():
    """Elementwise cubes in the places of the operators: their second derivatives are not zero."""
    f = types.SimpleNamespace()
    f.gs_embedding_workspace_bytes = f.gs_block_attention_workspace_bytes = f.gs_xent_workspace_bytes = lambda *a: 8
    f.gs_embedding_lookup = lambda table, ids, **kw: table.detach() ** 3
    f.gs_embedding_backward = lambda dout, ids, rows, ws, **kw: dout.detach() * 7
    f.gs_block_attention_forward = lambda indptr, indices, q, k, v, ws, **kw: (q.detach() ** 3, q.detach()[..., 0])
    f.gs_block_reverse = lambda *a, **kw: None
    f.gs_block_attention_backward = lambda indptr, indices, rev, q, k, v, out, lse, dout, ws, **kw: (3 * q.detach() ** 2 * dout.detach(), 0 * k, 0 * v)
    f.gs_xent_forward = lambda h, w, y, ws, **kw: (h.detach().pow(3).sum(1), h.detach()[:, 0])
    f.gs_xent_backward = lambda h, w, y, lse, dl, ws, **kw: (3 * h.detach() ** 2 * dl.detach()[:, None], 0 * w)
    return f


def _calls():
    ids = torch.zeros(3, dtype=torch.int32)
    return {
        "embedding": lambda x: autograd.embedding(x, ids),
        "block_attention": lambda x: autograd.block_attention(x.view(3, 1, 4), x.detach().view(3, 1, 4), x.detach().view(3, 1, 4), ids, ids),
        "table_cross_entropy": lambda x: autograd.table_cross_entropy(x, torch.ones(5, 4), ids),
    }


@pytest.mark.parametrize("name", sorted(_calls()))
def test_second_derivatives_are_refused(name, monkeypatch):
    monkeypatch.setattr(autograd, "gs", _stand_ins())
    x = torch.arange(1.0, 13.0).view(3, 4).requires_grad_()
    call = _calls()[name]
    loss = lambda: (call(x) ** 2).sum()  # noqa: E731
    loss().backward()
    first = x.grad.clone()
    assert (first != 0).all()
    value = loss()
    grad, = torch.autograd.grad(value, x, create_graph=True)
    assert torch.equal(grad, first)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        (value + (grad ** 2).sum()).backward()                # a gradient penalty beside the loss


@pytest.mark.parametrize("name", ["block_attention", "table_cross_entropy"])
def test_operands_count_too(name, monkeypatch):
    """The incoming gradient is a constant, the gradient still depends on what was saved."""
    monkeypatch.setattr(autograd, "gs", _stand_ins())
    x = torch.arange(1.0, 13.0).view(3, 4).requires_grad_()
    value = _calls()[name](x).sum()
    grad, = torch.autograd.grad(value, x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        (value + (grad ** 2).sum()).backward()


def test_a_linear_operator_s_gradient_may_be_a_constant(monkeypatch):
    """The rows' gradient by the table does not depend on the table: nothing is tied, nothing refused."""
    monkeypatch.setattr(autograd, "gs", _stand_ins())
    x = torch.ones(3, 4, requires_grad=True)
    value = _calls()["embedding"](x).sum()
    grad, = torch.autograd.grad(value, x, create_graph=True)
    assert not grad.requires_grad
    value.backward()
