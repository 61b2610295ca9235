"""The training operators as differentiable PyTorch functions.

Thin ``torch.autograd.Function`` wrappers over the library's calls: what is saved, recomputed and returned is what the
C ABI documents (``include/gs.h``).  Workspaces come from PyTorch's caching allocator for the length of a call.  Arrays
at their bounds (``count``, ``counts``, more query rows than the block has destinations): rows behind the actual sizes are
zeros, in results and in gradients.  The gradients are not differentiable: second derivatives raise an error.
"""
from __future__ import annotations

import functools

import torch

from . import binding as gs

__all__ = ["embedding", "block_attention", "rms_norm", "table_cross_entropy"]


def _workspace(nbytes: int, like: torch.Tensor) -> torch.Tensor:
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device)


class _NotTwice(torch.autograd.Function):
    """A gradient that depends on `on`, which it cannot be differentiated by."""

    @staticmethod
    def forward(ctx, grad, *on):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the training operators have first derivatives only: a gradient taken with create_graph=True was differentiated")


def _first_order(backward):
    """With create_graph, the gradients of `backward` are tied to all that they depend on, saved operands included
    (once_differentiable looks at the incoming gradients alone), so that a second derivative is an error and not zero."""

    @functools.wraps(backward)
    def checked(ctx, *incoming):
        with torch.no_grad():
            grads = backward(ctx, *incoming)
        on = [t for t in (*incoming, *ctx.saved_tensors) if t is not None and t.requires_grad] if torch.is_grad_enabled() else []
        return tuple(g if g is None else _NotTwice.apply(g, *on) for g in grads) if on else grads

    return checked


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, out_dtype, count):
        ctx.save_for_backward(ids, count)
        ctx.shape, ctx.dtype, ctx.scale = table.shape, table.dtype, scale
        return gs.gs_embedding_lookup(table, ids, scale=scale, out_dtype=out_dtype, count=count)

    @staticmethod
    @_first_order
    def backward(ctx, dout):
        ids, count = ctx.saved_tensors
        rows, dim = ctx.shape
        ws = _workspace(gs.gs_embedding_workspace_bytes(ids.numel(), rows, dim), dout)
        grad = gs.gs_embedding_backward(dout.contiguous(), ids, rows, ws, scale=ctx.scale, out_dtype=ctx.dtype, count=count)
        return grad, None, None, None, None


def embedding(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out_dtype: torch.dtype = None, count: torch.Tensor = None):
    """scale * table[ids] (zeros for ids outside the table); the gradient is the whole table's."""
    return _Embedding.apply(table, ids, float(scale), out_dtype, count)


class _BlockAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, indptr, indices, scale, max_row, counts):
        n, heads, dim = q.shape
        ws = _workspace(gs.gs_block_attention_workspace_bytes(n, k.shape[0], indices.numel(), heads, k.shape[1], dim), q)
        out, lse = gs.gs_block_attention_forward(indptr, indices, q, k, v, ws, scale=scale, max_row=max_row, counts=counts)
        ctx.save_for_backward(q, k, v, indptr, indices, out, lse)
        ctx.scale, ctx.max_row, ctx.counts = scale, max_row, counts
        return out

    @staticmethod
    @_first_order
    def backward(ctx, dout):
        q, k, v, indptr, indices, out, lse = ctx.saved_tensors
        n, heads, dim = q.shape
        ws = _workspace(gs.gs_block_attention_workspace_bytes(n, k.shape[0], indices.numel(), heads, k.shape[1], dim), q)
        reverse = gs.gs_block_reverse(indptr, indices, k.shape[0], ws, counts=ctx.counts)
        dq, dk, dv = gs.gs_block_attention_backward(indptr, indices, reverse, q, k, v, out, lse, dout.contiguous(), ws, scale=ctx.scale,
                                                    max_row=ctx.max_row, counts=ctx.counts)
        return dq, dk, dv, None, None, None, None, None


def block_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, indptr: torch.Tensor, indices: torch.Tensor,
                    scale: float = None, max_row: int = 0, counts=None):
    """Attention of a block's destinations (q [dst, q_heads, dim]) over their sources (k, v [src, kv_heads, dim])."""
    return _BlockAttention.apply(q, k, v, indptr, indices, scale, max_row, counts)


class _TableCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, table, labels, scale):
        ws = _workspace(gs.gs_xent_workspace_bytes(hidden.shape[0], table.shape[0], hidden.shape[1], hidden.dtype), hidden)
        loss, lse = gs.gs_xent_forward(hidden, table, labels, ws, scale=scale)
        ctx.save_for_backward(hidden, table, labels, lse)
        ctx.scale = scale
        return loss

    @staticmethod
    @_first_order
    def backward(ctx, dloss):
        hidden, table, labels, lse = ctx.saved_tensors
        ws = _workspace(gs.gs_xent_workspace_bytes(hidden.shape[0], table.shape[0], hidden.shape[1], hidden.dtype), hidden)
        dhidden, dtable = gs.gs_xent_backward(hidden, table, labels, lse, dloss.float().contiguous(), ws, scale=ctx.scale)
        return dhidden, dtable, None, None


def table_cross_entropy(hidden: torch.Tensor, table: torch.Tensor, labels: torch.Tensor, scale: float = 1.0):
    """Cross entropy per row of softmax(scale * hidden table^T); labels outside the table give 0 and no gradient.  Results of
    bf16 operands hold if ``gs_train_status()`` passes after them (it synchronises: call it where a step is kept anyway)."""
    return _TableCrossEntropy.apply(hidden, table, labels, float(scale))


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps, count):
        ctx.set_materialize_grads(False)
        out, hidden = gs.gs_rms_norm_forward(x, weight, residual=residual, eps=eps, count=count)
        ctx.save_for_backward(hidden, weight, count)
        ctx.eps, ctx.with_residual = eps, residual is not None
        return (out, hidden) if residual is not None else out

    @staticmethod
    @_first_order
    def backward(ctx, dout, dhidden=None):
        hidden, weight, count = ctx.saved_tensors
        if dout is None:                                     # the norm's result has no part in what is differentiated
            dout = torch.zeros_like(hidden)
        ws = _workspace(gs.gs_rms_norm_workspace_bytes(*hidden.shape), hidden)
        dx, dweight = gs.gs_rms_norm_backward(hidden, dout.contiguous(), ws, weight=weight, dhidden=None if dhidden is None else dhidden.contiguous(),
                                              eps=ctx.eps, count=count)
        return dx, dweight, dx if ctx.with_residual else None, None, None


def rms_norm(x: torch.Tensor, weight: torch.Tensor = None, residual: torch.Tensor = None, eps: float = 1e-6, count: torch.Tensor = None):
    """weight * h / sqrt(mean(h^2) + eps) for the rows of h = x + residual.  With a residual returns (that, h), both differentiable."""
    return _RmsNorm.apply(x, weight, residual, float(eps), count)
