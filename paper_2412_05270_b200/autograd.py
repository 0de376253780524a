"""The two ends of a language model as autograd functions: token embedding, adjusted logits and token log probabilities.

All call the library's kernels in either direction (no PyTorch arithmetic in between); see `binding` for the shapes
and types they take.  They have first derivatives; differentiating one of those raises.

Forward and backward pass can be captured into a CUDA graph together.  No graph of autograd's that was made outside the capture may then
hold the same leaves: PyTorch would add up their gradients on the stream of that one."""
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
        raise RuntimeError("embedding, adjust_logits and token_logprobs have a first derivative only")


def _first_order(grad, *sources):
    return _FirstOrder.apply(grad, *sources) if torch.is_grad_enabled() else grad          # enabled: create_graph=True


def _rows(d_out):
    """A gradient that was broadcast or transposed as the kernels read it: contiguous rows that do not overlap."""
    if (d_out.shape[1] > 1 and d_out.stride(1) != 1) or (d_out.shape[0] > 1 and d_out.stride(0) < d_out.shape[1]):
        return d_out.contiguous()
    return d_out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, index, scale):
        ctx.save_for_backward(index)
        ctx.rows, ctx.dim, ctx.scale = *table.shape, scale
        return B.embedding(table, index, scale)

    @staticmethod
    def backward(ctx, d_out):
        index, = ctx.saved_tensors
        d_out = _rows(d_out.reshape(index.numel(), ctx.dim))
        return _first_order(B.embedding_grad(d_out, index, ctx.rows, scale=ctx.scale), d_out), None, None


class _AdjustLogits(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, bias, bias_value, bias_index, history, lengths, start, repetition, frequency, presence, mask):
        ctx.set_materialize_grads(False)
        ctx.bias = "none" if bias is None else "shared" if bias.dim() == 1 else "row"
        kept = (history, lengths, repetition, bias_index, mask)        # what the backward pass reads: tensors are watched for changes in place
        ctx.kept = [None if isinstance(x, torch.Tensor) else x for x in kept]
        # (without a history the gradient does not ask for the logits' signs)
        ctx.save_for_backward(logits if history is not None else None, *(x if isinstance(x, torch.Tensor) else None for x in kept))
        return B.adjust_logits(logits, history, lengths, start, repetition, frequency, presence, bias, bias_index, bias_value, mask)

    @staticmethod
    def backward(ctx, d_out):
        if d_out is None:
            return (None,) * 11
        logits, *tensors = ctx.saved_tensors
        history, lengths, repetition, bias_index, mask = (x if x is not None else k for x, k in zip(tensors, ctx.kept))
        d = _rows(d_out)
        need_logits, need_bias, need_value = ctx.needs_input_grad[:3]
        r = B.adjust_logits_grad(d if logits is None else logits, d, history, lengths, repetition, mask, ctx.bias if need_bias else "none",
                                 bias_index if need_value else None)
        given = [_first_order(x, d_out, *([] if logits is None else [logits])) if x is not None and need else None
                 for x, need in zip(r, (need_logits, need_bias, need_value))]
        return (*given, *(None,) * 8)


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


def adjust_logits(logits: torch.Tensor, history=None, lengths=None, start=None, repetition=1.0, frequency=0.0, presence=0.0, bias=None,
                  bias_index=None, bias_value=None, mask=None) -> torch.Tensor:
    """`binding.adjust_logits` (penalties, biases, mask) out of place, with the gradients for logits, bias and bias_value."""
    return _AdjustLogits.apply(logits, bias, bias_value, bias_index, history, lengths, start, repetition, frequency, presence, mask)
