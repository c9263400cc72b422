"""The operators on rows of logits as differentiable PyTorch functions, for training programs.

Every function takes logits [..., vocab] (f32, bf16 or f16, on the GPU) and runs the library's kernels in both directions
(``binding.pacer_logprobs``, ``binding.pacer_distill``); gradients come in the logits' type.  A second derivative is not
defined.  What a training step needs of loss and gradient in one pass, with the gradient written over the logits if
wanted, is ``binding.pacer_distill_grad``.

``head_logprobs`` and ``head_nll`` take hidden rows [..., d] and the LM head [vocab, d] (bf16) instead, and never write the logits:
``head_nll`` computes the gradients in its forward pass, together with the loss.
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


class _HeadLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, head, tokens, bias_ids, bias):
        # (clones: logp may be changed in place where the three are views of one allocation)
        logp, entropy, lse = (x.clone() for x in binding.pacer_head_logprobs(hidden, head, tokens, bias_ids, bias))
        ctx.save_for_backward(hidden, head, tokens, bias_ids, logp, entropy, lse)
        ctx.bias = bias
        ctx.set_materialize_grads(False)
        return logp, entropy, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logp, g_entropy, g_lse):
        if g_logp is None and g_entropy is None and g_lse is None:
            return (None,) * 5
        hidden, head, tokens, bias_ids, logp, entropy, lse = ctx.saved_tensors
        return (*binding.pacer_head_logprobs_backward(hidden, head, tokens, logp, lse, entropy, g_logp, g_entropy, g_lse, bias_ids, ctx.bias,
                                                      grads=ctx.needs_input_grad[:2]), None, None, None)


def _flat_rows(hidden, tokens, bias_ids):
    shape = tokens.shape
    assert hidden.shape[:-1] == shape and (bias_ids is None or bias_ids.shape == shape), "tokens and bias_ids: the hidden rows' leading shape"
    return hidden.reshape(-1, hidden.shape[-1]), tokens.reshape(-1), None if bias_ids is None else bias_ids.reshape(-1)


def head_logprobs(hidden: torch.Tensor, head: torch.Tensor, tokens: torch.Tensor, bias_ids: Optional[torch.Tensor] = None, bias: float = 0.0):
    """(logp, entropy, lse) [...] of int32 tokens [...] under hidden @ head.T (see ``binding.pacer_head_logprobs``), differentiable in
    hidden and head; the logits are computed again in the backward pass.  A token outside the vocabulary has logp 0 and passes
    no gradient.  All three outputs are kept for the backward pass."""
    h, t, i = _flat_rows(hidden, tokens, bias_ids)
    return tuple(x.view(tokens.shape) for x in _HeadLogprobs.apply(h, head, t, i, bias))


class _HeadNll(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, head, tokens, weight, bias_ids, bias, train):
        grads = ctx.needs_input_grad[:2] if train else (False, False)
        loss, dhidden, dhead = binding.pacer_head_nll_grad(hidden, head, tokens, weight, bias_ids, bias, grads=grads)
        ctx.save_for_backward(dhidden, dhead, loss if ctx.needs_input_grad[3] else None)        # (freed by the backward pass)
        return (loss * weight).sum()

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        dhidden, dhead, loss = (None if x is None else x * g for x in ctx.saved_tensors)
        return dhidden, dhead, None, loss, None, None, None


def head_nll(hidden: torch.Tensor, head: torch.Tensor, tokens: torch.Tensor, weight: torch.Tensor, bias_ids: Optional[torch.Tensor] = None,
             bias: float = 0.0) -> torch.Tensor:
    """sum(weight * negative log-likelihood) of int32 tokens [...] under hidden @ head.T, weight f32 [...]: a scalar, whose gradients the forward
    pass computes (``binding.pacer_head_nll_grad``); the backward pass multiplies them by the incoming scalar, which rounds them once more
    unless it is a power of 2.  A token outside the vocabulary (-1: padding) adds nothing."""
    h, t, i = _flat_rows(hidden, tokens, bias_ids)
    assert weight.shape == tokens.shape, "weight: the hidden rows' leading shape"
    return _HeadNll.apply(h, head, t, weight.reshape(-1), i, bias, torch.is_grad_enabled())     # (inside the function it never is)
