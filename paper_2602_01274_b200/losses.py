"""The operators on rows of logits as differentiable PyTorch functions, for training programs.

Every function takes logits [..., vocab] (f32, bf16 or f16, on the GPU) and runs the library's kernels in both directions
(``binding.pacer_logprobs``, ``binding.pacer_distill``); gradients come in the logits' type.  A second derivative is not
defined.  What a training step needs of loss and gradient in one pass, with the gradient written over the logits if
wanted, is ``binding.pacer_distill_grad``.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, top):
        rows, f32 = logits.shape[0], dict(dtype=torch.float32, device=logits.device)
        logp, entropy, lse = (torch.empty(rows, **f32) for _ in range(3))      # (no views of one tensor: they may be changed in place)
        ids, top_logp = torch.empty(rows, top, dtype=torch.int32, device=logits.device), torch.empty(rows, top, **f32)
        binding.pacer_logprobs(logits, tokens, top, out=(logp, entropy, lse, ids, top_logp))
        ctx.save_for_backward(logits, tokens, lse, entropy)
        ctx.mark_non_differentiable(ids, top_logp)
        ctx.set_materialize_grads(False)
        return logp, entropy, lse, ids, top_logp

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logp, g_entropy, g_lse, *_):
        if g_logp is None and g_entropy is None and g_lse is None:
            return None, None, None
        logits, tokens, lse, entropy = ctx.saved_tensors
        return binding.pacer_logprobs_backward(logits, tokens, lse, entropy, g_logp, g_entropy, g_lse), None, None


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0):
    """(logp, entropy, lse, top_ids, top_logp) of int32 tokens [...] under logits [..., vocab]; the first three are
    differentiable.  A token outside the vocabulary (-1: padding) has logp 0 and passes no gradient.  logp may be changed in
    place; entropy and lse are kept for the backward pass, as the logits are."""
    shape = tokens.shape
    assert logits.shape[:-1] == shape, "tokens: the logits' leading shape"
    logp, entropy, lse, ids, top_logp = _TokenLogprobs.apply(logits.reshape(-1, logits.shape[-1]), tokens.reshape(-1), top)
    return logp.view(shape), entropy.view(shape), lse.view(shape), ids.view(*shape, top), top_logp.view(*shape, top)


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, teacher, teacher_lse, temperature):
        loss, lse, tail_lse = binding.pacer_distill(logits, ids, teacher, temperature, teacher_lse)
        ctx.save_for_backward(logits, ids, teacher, teacher_lse, lse, tail_lse)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, g_loss):
        logits, ids, teacher, teacher_lse, lse, tail_lse = ctx.saved_tensors
        return (binding.pacer_distill_backward(logits, ids, teacher, lse, tail_lse, g_loss, ctx.temperature, teacher_lse),
                None, None, None, None)


def distill_loss(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, temperature: float = 1.0,
                 teacher_lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    """KL from a teacher's top logits (ids int32 and teacher [..., k]; teacher_lse [...] or None, see
    ``binding.pacer_distill``) to the student's logits [..., vocab], per position [...].  The teacher gets no gradient."""
    lead = logits.shape[:-1]
    assert ids.shape[:-1] == lead and teacher.shape == ids.shape, "ids and teacher: the logits' leading shape, then the list"
    k = ids.shape[-1]
    loss = _Distill.apply(logits.reshape(-1, logits.shape[-1]), ids.reshape(-1, k), teacher.detach().reshape(-1, k),
                          None if teacher_lse is None else teacher_lse.detach().reshape(-1), temperature)
    return loss.view(lead)
