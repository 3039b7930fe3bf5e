"""torch.autograd front ends of the losses over a vocabulary.

`linear_cross_entropy` and `linear_distillation` take hidden states (..., h) and an output head (v, h), both bfloat16 or
both float32, and return the scalar loss, on torch's current stream. The logits are never held as a whole, so the
forward pass computes the gradients as well where they are wanted (the backward pass multiplies them by the incoming
gradient, in place, and hands them out: it can run once). That factor rounds bfloat16 gradients a second time unless it is a
power of two; a factor that is known beforehand is better given as `scale`. `token_losses` is the loss of every token,
without gradients. These functions only marshal arguments: the arithmetic runs in libmfsdp.so, and there is no CPU path.

Forward and backward passes can be captured into a graph. As with any torch function, let no loss of an eager pass over the
same leaves live on while their backward pass is captured: torch ties a leaf's gradient to the stream of the pass that it first
met, and waiting for that stream during a capture is an error that can end the process.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import native


def _dense(t: torch.Tensor) -> torch.Tensor:
    """t contiguous and 16-byte aligned, as the library takes it (labels shifted by one, ids[1:], are not)."""
    t = t.detach().contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _rows(t: torch.Tensor, tail: int, what: str) -> torch.Tensor:
    """t with its leading dimensions as one; `tail` dimensions stay."""
    if t.dim() <= tail:
        raise ValueError(f"{what}: at least {tail + 1} dimensions are required, got shape {tuple(t.shape)}")
    return _dense(t.reshape(-1, *t.shape[t.dim() - tail:]))


class _HeadLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, grads, call):
        with torch.cuda.device(hidden.device):
            x, w = _rows(hidden, 1, "hidden"), _dense(weight)
            loss = torch.empty((), dtype=torch.float32, device=hidden.device)
            dx = torch.empty_like(x) if grads and ctx.needs_input_grad[0] else None
            dw = torch.empty_like(w) if grads and ctx.needs_input_grad[1] else None
            call(x, w, loss=loss, dx=dx, dw=dw)
        ctx.grads = (dx, dw)
        ctx.shape = hidden.shape
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        if ctx.grads is None:
            raise RuntimeError("the gradients of this loss have been handed out: its backward pass runs once")
        (dx, dw), ctx.grads = ctx.grads, None
        with torch.cuda.device(grad.device):
            factor = grad.to(torch.float32).contiguous()
            for g in (dx, dw):
                if g is not None:
                    native.scale_grad_t(g, factor)
        return dx.view(ctx.shape) if dx is not None else None, dw, None, None


def _weights(token_weight: Optional[torch.Tensor], shape: torch.Size) -> Optional[torch.Tensor]:
    """One weight per token, in the tokens' own shape or as one dimension (any other of as many elements, a transposed one
    for instance, would give tokens each other's weights)."""
    if token_weight is None:
        return None
    if token_weight.shape not in (shape, (shape.numel(),)):
        raise ValueError(f"token_weight: shape {tuple(token_weight.shape)} where {tuple(shape)} is required")
    return _dense(token_weight.reshape(-1))


def _check_head(hidden: torch.Tensor, weight: torch.Tensor) -> None:
    if not hidden.is_cuda or not weight.is_cuda:
        raise ValueError(f"the losses run on the GPU only; got {hidden.device} and {weight.device} tensors")
    if hidden.device != weight.device:
        raise ValueError(f"hidden and weight must be on one GPU; got {hidden.device} and {weight.device}")


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, ignore_index: int = -100,
                         reduction: str = "mean", token_weight: Optional[torch.Tensor] = None, z_loss: float = 0.0,
                         scale: float = 1.0, chunk_rows: int = 0) -> torch.Tensor:
    """Softmax cross entropy of hidden @ weight.T with the labels `targets` (hidden's shape without its last dimension):
    scale / D sum_r a_r (lse_r - z_{r, t_r} + z_loss lse_r^2), D = 1 ("sum") or the sum of the a_r of the labelled
    tokens ("mean"). token_weight: a_r (targets' shape, float32; no gradient). A call with all labels ignored gives 0."""
    _check_head(hidden, weight)
    if targets.shape != hidden.shape[:-1]:
        raise ValueError(f"targets: shape {tuple(targets.shape)} where {tuple(hidden.shape[:-1])} is required")
    t, a = _dense(targets.reshape(-1)), _weights(token_weight, targets.shape)

    def call(x, w, **out):
        native.linear_xent_t(x, w, t, ignore_index=ignore_index, reduction=reduction, scale=scale, token_weight=a,
                             z_loss=z_loss, chunk_rows=chunk_rows, **out)

    return _HeadLoss.apply(hidden, weight, torch.is_grad_enabled(), call)


def linear_distillation(hidden: torch.Tensor, weight: torch.Tensor, top_ids: torch.Tensor, top_logits: torch.Tensor,
                        temperature: float = 1.0, reduction: str = "mean", token_weight: Optional[torch.Tensor] = None,
                        scale: float = 1.0, chunk_rows: int = 0) -> torch.Tensor:
    """KL divergence from a teacher's top logits (top_ids, top_logits: (..., k); a negative id is an empty slot) to the
    softmax of hidden @ weight.T / temperature over the whole vocabulary, reduced as linear_cross_entropy's. Pass
    scale=temperature ** 2 for gradients of the size of the hard labels'. The teacher gets no gradient."""
    _check_head(hidden, weight)
    want = (*hidden.shape[:-1], top_ids.shape[-1] if top_ids.dim() else 0)
    for t, what in ((top_ids, "top_ids"), (top_logits, "top_logits")):
        if t.shape != want:
            raise ValueError(f"{what}: shape {tuple(t.shape)} where {want} is required")
    ids, logits = _rows(top_ids, 1, "top_ids"), _rows(top_logits, 1, "top_logits")
    a = _weights(token_weight, hidden.shape[:-1])

    def call(x, w, **out):
        native.linear_distill_t(x, w, ids, logits, temperature=temperature, reduction=reduction, scale=scale,
                                token_weight=a, chunk_rows=chunk_rows, **out)

    return _HeadLoss.apply(hidden, weight, torch.is_grad_enabled(), call)


@torch.no_grad()
def token_losses(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                 ignore_index: int = -100) -> torch.Tensor:
    """-log p(target) of every token (float32, targets' shape; 0 where ignored): scoring, down to a single token."""
    _check_head(hidden, weight)
    if targets.shape != hidden.shape[:-1]:
        raise ValueError(f"targets: shape {tuple(targets.shape)} where {tuple(hidden.shape[:-1])} is required")
    with torch.cuda.device(hidden.device):
        out = torch.empty(targets.shape, dtype=torch.float32, device=hidden.device)
        native.linear_xent_t(_rows(hidden, 1, "hidden"), _dense(weight), _dense(targets.reshape(-1)),
                             token_loss=out.view(-1), ignore_index=ignore_index)
    return out
