"""Gradients of the fused head where the logits of a row are far apart: each row of dhead is one token, so that the gradients of rare tokens have to
be right by themselves, and where dz comes with its rounding remainders (up to 128 rows).

Tolerances as in test_gpu_head_grads (its `slack`), with the shares that dz is held to: the one call keeps 11 bits of each share, half a step is 2^-11,
of all that is within 2^-62 of its half tile's largest; up to 128 rows dz and its remainder are two bf16 numbers, 2^-16, above that one, 2^-8."""
import math

import pytest
import torch

from tests import logit_refs as ref
from tests.test_gpu_head_grads import BF16, DEV, F32, logits, slack, weights

pytestmark = pytest.mark.gpu


def close(got, dz, size, other, by_rows, share, slack_z, slack_k, least):
    """got bf16 against dz @ other (by_rows) or dz.T @ other, whose dz are off by `share` of themselves and by `least`."""
    a, s = (dz, size) if by_rows else (dz.T, size.T)
    want = a @ other
    terms = (a.abs() * (share + slack_k) + s * slack_z + least) @ other.abs()
    bound = 1.01 * terms + BF16 * (want.abs() + terms) + 1e-38
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= bound).all(), (float((off / bound).max()), float((off / want.abs().clamp(min=1e-300)).max()))


def spread(rows, vocab, d, nats):
    """Rows that are nearly alike, so that a rare token is rare in all of them; logits with a standard deviation of `nats`."""
    g = torch.Generator(device=DEV).manual_seed(rows + vocab)
    h = (torch.randn(1, d, generator=g, device=DEV) + 0.05 * torch.randn(rows, d, generator=g, device=DEV)).to(torch.bfloat16)
    w = (torch.randn(vocab, d, generator=g, device=DEV) * nats / math.sqrt(d)).to(torch.bfloat16)
    tok = torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    tok[1::5] = -1
    return h, w, tok


def gradient(h, w, tok, ids, bias, weight):
    z = logits(h, w, ids, bias)
    lp, _ = ref.softmax_parts(z)
    named = tok >= 0
    at, g = torch.where(named, tok, 0).long()[:, None], torch.where(named, weight, 0.0).double()[:, None]
    own = g * torch.where(named, torch.expm1(lp.gather(1, at)[:, 0]) - lp.gather(1, at)[:, 0].exp(), 0.0)[:, None]
    return z, (lp.exp() * g).scatter_add(1, at, own), (lp.exp() * g.abs()).scatter_add(1, at, own.abs())


@pytest.mark.parametrize("rows,vocab,d", [(1, 4000, 64), (6, 4099, 64), (130, 8003, 128), (300, 1000, 72)])
@pytest.mark.parametrize("planted", [False, True])
def test_far_apart(rows, vocab, d, planted):
    from paper_2602_01274_b200 import binding as b
    h, w, tok = spread(rows, vocab, d, 3.0 if planted else 6.0)
    ids = (tok + 1) % vocab if planted else None                            # (a planted bias on a token that is not the row's)
    weight = weights(rows)[0]
    z, dz, size = gradient(h, w, tok, ids, 18.0, weight)
    assert float(z.max() - z.min()) > 30
    sz, _ = slack(h, w, z, 0)
    least = float(weight.abs().max()) * 2.0 ** -62
    for grads in ((True, True), (False, True)):
        _, dh, dw = b.pacer_head_nll_grad(h, w, tok, weight, ids, 18.0, grads=grads)
        share = 2.0 ** -11 + (2.0 ** -16 if rows <= 128 else BF16)
        close(dw, dz, size, h.double(), False, share, sz, (rows / 16 + 1) * 2 * F32, least)
        if dh is not None:
            close(dh, dz, size, w.double(), True, share, sz, (vocab / 16 + 1) * 2 * F32, least)
    logp, ent, lse = b.pacer_head_logprobs(h, w, tok, ids, 18.0)
    dh, dw = b.pacer_head_logprobs_backward(h, w, tok, logp, lse, ent, -weight, None, None, ids, 18.0)
    close(dw, dz, size, h.double(), False, 2.0 ** -16 if rows <= 128 else BF16, sz, (rows / 16 + 1) * 2 * F32, 1e-37)
    close(dh, dz, size, w.double(), True, 2.0 ** -16 if rows <= 128 else BF16, sz, (vocab / 16 + 1) * 2 * F32, 1e-37)


def confident(bias, rows=40, vocab=500):
    """All logits 0 but the row's token's: (h, w, tokens, the rest's mass over the token's, dz of the loss)."""
    g = torch.Generator(device=DEV).manual_seed(3)
    h = torch.randn(rows, 64, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.zeros(vocab, 64, device=DEV, dtype=torch.bfloat16)
    tok = torch.arange(rows, device=DEV, dtype=torch.int32)
    rest = (vocab - 1) * math.exp(-bias)
    dz = torch.full((rows, vocab), math.exp(-bias) / (1 + rest), device=DEV, dtype=torch.float64)
    dz[torch.arange(rows), torch.arange(rows)] = -rest / (1 + rest)
    return h, w, tok, rest, dz


@pytest.mark.parametrize("bias", [8.0, 14.0, 20.0, 40.0, 60.0])
@pytest.mark.parametrize("rows", [40, 200])
def test_confident_rows_of_the_loss(bias, rows):
    """1 - p of the token is the others' share: no difference of numbers near 1."""
    from paper_2602_01274_b200 import binding as b
    h, w, tok, rest, dz = confident(bias, rows)
    loss, _, dw = b.pacer_head_nll_grad(h, w, tok, torch.ones(rows, device=DEV), tok, bias)
    assert ((loss.double() - math.log1p(rest)).abs() <= 32 * F32 * (1 + bias) * math.log1p(rest)).all()
    share = 2.0 ** -11 + (2.0 ** -16 if rows <= 128 else BF16) + 32 * F32 * (1 + bias)
    close(dw, dz, dz.abs(), h.double(), False, share, 0.0, (rows / 16 + 1) * 2 * F32, 1e-37)


@pytest.mark.parametrize("bias", [8.0, 14.0, 20.0, 40.0])
def test_confident_rows_of_log_probabilities(bias):
    """1 - p out of logp, whose error is that of the f32 sum of all shares: some roundings of 2^-24 of 1, whatever 1 - p is."""
    from paper_2602_01274_b200 import binding as b
    h, w, tok, rest, dz = confident(bias)
    one = torch.ones(40, device=DEV)
    logp, ent, lse = b.pacer_head_logprobs(h, w, tok, tok, bias)
    _, dw = b.pacer_head_logprobs_backward(h, w, tok, logp, lse, ent, -one, None, None, tok, bias)
    at_token = torch.zeros_like(dz)
    at_token[torch.arange(40), torch.arange(40)] = 1.0
    # (p of the others: lse is off by half a step of bias + log S)
    close(dw, dz, at_token, h.double(), False, 2.0 ** -16 + 8 * F32 * (1 + bias), 16 * F32, 4 * 2 * F32, 1e-37)
