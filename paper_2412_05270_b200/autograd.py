"""The two ends of a language model as autograd functions: token embedding and token log probabilities.

Both call the library's kernels in either direction (no PyTorch arithmetic in between); see `binding` for the shapes
and types they take.  They have first derivatives; differentiating one of those raises."""
from __future__ import annotations

import torch

from . import binding as B


class _FirstOrder(torch.autograd.Function):
    """Hands a gradient on as a function of the tensors it was computed from, and refuses to be differentiated: without it a
    term made of the gradient (create_graph=True) would count as constant and drop out of another loss's backward pass."""

    @staticmethod
    def forward(ctx, grad, *sources):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("embedding and token_logprobs have a first derivative only")


def _first_order(grad, *sources):
    return _FirstOrder.apply(grad, *sources) if torch.is_grad_enabled() else grad          # enabled: create_graph=True


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, index, scale):
        ctx.save_for_backward(index)
        ctx.rows, ctx.dim, ctx.scale = *table.shape, scale
        return B.embedding(table, index, scale)

    @staticmethod
    def backward(ctx, d_out):
        index, = ctx.saved_tensors
        d_out = d_out.reshape(index.numel(), ctx.dim)
        # (a gradient that was broadcast or transposed: the kernels read contiguous rows that do not overlap)
        if (ctx.dim > 1 and d_out.stride(1) != 1) or (d_out.shape[0] > 1 and d_out.stride(0) < ctx.dim):
            d_out = d_out.contiguous()
        return _first_order(B.embedding_grad(d_out, index, ctx.rows, scale=ctx.scale), d_out), None, None


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, scale):
        r = B.token_logprobs(logits, targets, scale=scale)
        ctx.save_for_backward(logits, targets, r.lse, r.entropy)
        ctx.set_materialize_grads(False)               # an output that no loss uses: None, no entropy term
        ctx.scale = scale
        return r.logprob, r.entropy

    @staticmethod
    def backward(ctx, d_logprob, d_entropy):
        logits, targets, lse, entropy = ctx.saved_tensors
        if d_logprob is None:
            d_logprob = torch.zeros_like(lse)
        grad = B.token_logprobs_grad(logits, targets, lse, entropy, d_logprob.contiguous(),
                                     None if d_entropy is None else d_entropy.contiguous(), scale=ctx.scale)
        return _first_order(grad, logits, d_logprob, d_entropy), None, None


def embedding(table: torch.Tensor, index: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """scale * table[index] with the gradient for the table (a zero row and no gradient for indices outside it)."""
    return _Embedding.apply(table, index, float(scale))


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, scale: float = 1.0):
    """(log probability of the target, entropy) per row of `logits`, with the gradient for the logits."""
    return _TokenLogprobs.apply(logits, targets, float(scale))
