"""Rows of logits that share an offset or are masked with finite values: what is computed of a row goes by the differences of its
logits, whatever they have in common.

Bounds, row by row.  EPS (tests/test_gpu_logits.py) is what fp32 arithmetic may change of a row's log sum of exponentials, taken over
differences.  A log probability is an exponent (one fused multiply-add, with a constant of half a step), minus the sum's logarithm,
times a constant: six half steps of its own size.  A log-sum-exp has the logits' size and is rounded there: two half steps."""
import math

import pytest
import torch

from tests import logit_refs as ref
from tests.test_gpu_logits import DEV, EPS, TYPES, close, gen, make_logits, make_tokens

pytestmark = pytest.mark.gpu

OFFSETS = [("f32", o) for o in (-9e7, -1e7, -1e5, -1e3, 0.0, 1e2, 1e3, 1e4, 1e5, 1e6, 1e7, 5e7, 9e7)] + \
    [("bf16", o) for o in (-9e7, -1e4, 1e4, 5e7)] + [("f16", o) for o in (-6e4, -2e4, 2e4, 6e4)]


def shifted(rows, vocab, dtype, offset, seed=50, pad=0):
    """Noise a few steps of the type wide (two at least) around the offset."""
    step = 2.0 ** math.floor(math.log2(max(abs(offset), 1.0))) * torch.finfo(TYPES[dtype]).eps
    z = make_logits(rows, vocab, "f32", pad, seed=seed) * max(1.0, 0.7 * step if step < 16 else 0.1 * step)
    z = z + offset
    return z.to(TYPES[dtype])


def size(x):
    return x.abs().nan_to_num(0, 0, 0)


def check_rows(z, tokens, top):
    from paper_2602_01274_b200 import binding as b
    got = b.pacer_logprobs(z, tokens, top)
    logp, ent, lse, ids, tlp = got
    want_logp, want_ent, want_lse, lp = ref.logprobs(z, tokens)
    close(logp, want_logp, EPS + 6 * ref.F32 * size(want_logp), "logp")
    close(lse, want_lse, EPS + 2 * ref.F32 * size(want_lse), "lse")
    close(ent, want_ent, 40 * EPS, "entropy")
    best = ref.order_rows(z, top)
    assert torch.equal(ids.long(), best)
    want = lp.gather(1, best)
    close(tlp, want, EPS + 6 * ref.F32 * size(want), "alternatives")
    return got


@pytest.mark.parametrize("dtype,offset", OFFSETS)
@pytest.mark.parametrize("rows,vocab", [(1, 32003), (3, 4096), (600, 4099)])
def test_logprobs_with_an_offset(dtype, offset, rows, vocab):
    check_rows(shifted(rows, vocab, dtype, offset), make_tokens(rows, vocab), 20)


@pytest.mark.parametrize("rows,vocab", [(9, 1000), (600, 32000), (4, 151936)])
@pytest.mark.parametrize("value", [-1e7, -9e7, -2e8, 5e7, 1e3])
def test_rows_of_one_value_are_uniform(rows, vocab, value):
    from paper_2602_01274_b200 import binding as b
    z = torch.full((rows, vocab), value, device=DEV)
    logp, ent, _, ids, tlp = b.pacer_logprobs(z, torch.arange(rows, dtype=torch.int32, device=DEV), 5)
    want = torch.full((rows,), -math.log(vocab), dtype=torch.float64, device=DEV)
    close(logp, want, EPS, "logp")
    close(tlp, want[:, None].expand(rows, 5), EPS, "alternatives")
    close(ent, -want, 2 * EPS, "entropy")
    assert (ids == torch.arange(5, device=DEV)).all()


@pytest.mark.parametrize("rows", [30, 600])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_finite_masks_row_by_row(rows, dtype):
    """A row masked with finite values has the results of the row masked with -inf."""
    vocab, top = 32003, 20
    z = make_logits(rows, vocab, dtype, seed=51)
    low = torch.finfo(z.dtype).min
    masks = (low,) if dtype == "f16" else (low, -3e38, -1e20, -1e10, -1e8, -1e7, -1e6, -1e5)
    hidden = torch.zeros(rows, vocab, dtype=torch.bool, device=DEV)
    finite = z.clone()
    for i, m in enumerate(masks):
        for j, keep in enumerate((slice(0, 700), slice(vocab - 700, vocab), slice(4000, 4700))):
            hidden[3 * i + j] = True
            hidden[3 * i + j, keep] = False
            finite[3 * i + j] = torch.where(hidden[3 * i + j], torch.full_like(z[0], m), z[3 * i + j])
    tokens = make_tokens(rows, vocab)
    first = hidden.long().argmin(1).to(torch.int32)     # a token that is left
    tokens = torch.where(tokens >= 0, first, tokens)
    got = check_rows(finite, tokens, top)
    plain = check_rows(z.masked_fill(hidden, -math.inf), tokens, top)
    assert torch.equal(got[3], plain[3])
    for i, name in ((0, "logp"), (1, "entropy"), (2, "lse"), (4, "alternatives")):
        close(got[i], plain[i], (80 if name == "entropy" else 2) * EPS, name)


@pytest.mark.parametrize("dtype,offset", OFFSETS)
@pytest.mark.parametrize("rows,vocab", [(3, 4096), (600, 4099)])
def test_the_gradient_of_rows_with_an_offset(dtype, offset, rows, vocab):
    """From the forward call's own lse and entropy.  An lse below 1024 has an error of two half steps of its size, which each
    probability shares; larger ones are taken anew."""
    from paper_2602_01274_b200 import binding as b
    z, tokens = shifted(rows, vocab, dtype, offset), make_tokens(rows, vocab)
    _, ent, lse, _, _ = b.pacer_logprobs(z, tokens)
    g = [torch.randn(rows, generator=gen(52 + i), device=DEV) for i in range(3)]
    _, want_ent, want_lse, _ = ref.logprobs(z, tokens)
    want, terms = ref.logprobs_grad(z, tokens, want_lse, want_ent, *g)
    got = b.pacer_logprobs_backward(z, tokens, lse, ent, *g)
    half, least = ref.rounding(z.dtype)
    shared = torch.where(want_lse.abs() < 1024, 2 * ref.F32 * want_lse.abs(), 0.0)[:, None]
    # the entropy's error, 40 EPS, and that of log p itself, times g_entropy p
    gh, p = g[1].double().abs()[:, None], torch.softmax(z.double(), 1)
    # the exponential flushes what lies below 2^-126 to 0; log p is -87.3 there and the factor of g_entropy p at most 87.3 + H, H < 9
    # (further down p falls faster than its logarithm grows)
    flushed = 2.0 ** -126 * 100 * sum(x.double().abs() for x in g)[:, None]
    close(got, want, half * 1.01 * want.abs() + (180 * ref.F32 + EPS + shared) * terms + gh * p * (41 * EPS + shared) + least + flushed, "dlogits")
