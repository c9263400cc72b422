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
    """Noise around the offset: of width 2, or more where the type's steps there are coarser (some then tell hardly any logits apart)."""
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


def make_list(z, k, temperature, tail, seed=60):
    """A teacher's list without repetitions, and its log-sum-exp with three tenths to a half of the mass outside."""
    rows, vocab = z.shape
    ids = torch.rand(rows, vocab, generator=gen(seed), device=DEV).topk(k, 1).indices.to(torch.int32)
    t = torch.randn(rows, k, generator=gen(seed + 1), device=DEV) * 2
    lse = torch.logsumexp(t / temperature, 1) + 0.4 + 0.2 * torch.rand(rows, generator=gen(seed + 2), device=DEV) if tail else None
    return ids, t, lse


def check_distill(z, ids, t, temperature, tl):
    """Loss, one-pass and two-call gradient against 64 bits and against each other.  log p of a listed token, and of the tail, is right to
    EPS and six half steps of its size, and comes in times q, which is right to 100 half steps (exponents of the teacher's values below 30,
    four roundings of half a step of at most 32 * 0.7, a sum of 20, two exponentials); with a tail, q_t = 1 - sum q is right to 2 EPS, times a logarithm of at most 30 for p_t of the
    rows here that have one (or of log p_t's size, which the six half steps of the loss's size and 2 EPS of it cover).  The
    gradient's terms: 4 EPS as in tests/test_gpu_logits.py (exponents down to -126 with five half steps each are 2.6 EPS), what the exponential
    flushes below 2^-126 (p and w, each times at most 1), and for the second call what its lse below 1024 is off, two half steps."""
    from paper_2602_01274_b200 import binding as b
    rows, vocab = z.shape
    w = torch.randn(rows, generator=gen(63), device=DEV)
    loss0, lse0, tail0, d0, terms = ref.distill(z, ids, t, temperature, tl, w)
    top = z.double().amax(1, keepdim=True)
    logs = size(ref.softmax_parts((z.double() - top) / temperature)[0].gather(1, ids.long())).amax(1)
    loss, lse, tail = b.pacer_distill(z, ids, t, temperature, tl)
    close(loss, loss0, (4 if tl is None else 64) * EPS + 106 * ref.F32 * logs + (0 if tl is None else (2 * EPS + 6 * ref.F32) * size(loss0)), "loss")
    close(lse, lse0, EPS + 4 * ref.F32 * size(lse0), "lse")
    if tl is not None:
        close(tail, tail0, EPS + 4 * ref.F32 * size(tail0), "tail")
    half, least = ref.rounding(z.dtype)
    flushed = (2 * 2.0 ** -126 * w.double().abs() / temperature)[:, None]
    loss1, d1 = b.pacer_distill_grad(z, ids, t, w, temperature, tl)
    assert torch.equal(loss1, loss)
    close(d1, d0, half * 1.01 * d0.abs() + 4 * EPS * terms + least + flushed, "one pass")
    shared = torch.where(lse0.abs() < 1024, 2 * ref.F32 * lse0.abs(), 0.0)
    if tl is not None:
        shared = shared + torch.where(tail0.abs() < 1024, 2 * ref.F32 * tail0.abs(), 0.0)
    d2 = b.pacer_distill_backward(z, ids, t, lse, tail, w, temperature, tl)
    close(d2, d0, half * 1.01 * d0.abs() + (4 * EPS + shared[:, None]) * terms + least + flushed, "two calls")
    if z.dtype == torch.float32:                        # a row's gradient sums to 0
        for d, more in ((d1, 0.0), (d2, shared)):
            assert (d.double().sum(1).abs() <= (4 * EPS + more) * terms.sum(1) + vocab * flushed[:, 0]).all()
    copy = z.clone()
    assert torch.equal(b.pacer_distill_grad(copy, ids, t, w, temperature, tl, out=copy)[1], d1)
    copy = z.clone()
    assert torch.equal(b.pacer_distill_backward(copy, ids, t, lse, tail, w, temperature, tl, out=copy), d2)


@pytest.mark.parametrize("dtype,offset", OFFSETS)
@pytest.mark.parametrize("temperature", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("tail", [False, True])
def test_distillation_of_a_student_with_an_offset(dtype, offset, temperature, tail):
    for rows, vocab, k in ((3, 4096, 20), (600, 1031, 5)):
        z = shifted(rows, vocab, dtype, offset)
        check_distill(z, *make_list(z, k, temperature, tail)[:2], temperature, make_list(z, k, temperature, tail)[2])


@pytest.mark.parametrize("offset", [0.0, 20.0, -500.0])
def test_distillation_at_the_lowest_temperature(offset):
    z = make_logits(6, 2000, "f32", seed=64) + offset
    ids, t, _ = make_list(z, 9, 1e-3, False)
    check_distill(z, ids, t * 1e-3, 1e-3, None)


@pytest.mark.parametrize("mask", [-1e3, -1e5, -1e6, -1e7, -9e7])
def test_distillation_with_a_masked_tail(mask):
    """All tokens outside the list masked with one finite value: they share the tail's part evenly."""
    z = make_logits(6, 3001, "f32", seed=65)
    ids, t, tl = make_list(z, 12, 1.0, True)
    z = torch.full_like(z, mask).scatter(1, ids.long(), z.gather(1, ids.long()))
    check_distill(z, ids, t, 1.0, tl)


@pytest.mark.parametrize("teacher,offset", [("f32", o) for o in (-3e38, -9e7, -1e5, 1e3, 1e5, 1e6, 9e7, 3e38)] +
                         [("bf16", -3e38), ("bf16", 1e4), ("f16", -6e4), ("f16", 6e4)])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 3.0])
def test_a_teacher_with_an_offset(teacher, offset, temperature):
    """Values that share an offset: the renormalised list is that of their differences."""
    z = make_logits(40, 3001, "f32", seed=66)
    ids = make_list(z, 20, 1.0, False)[0]
    t = shifted(40, 20, teacher, offset, seed=67) if abs(offset) < 1e30 else torch.full((40, 20), offset, device=DEV).to(TYPES[teacher])
    t[:20, ::3] = torch.finfo(t.dtype).min if offset > -1e30 else -math.inf       # some that the teacher masks
    t[7] = torch.finfo(t.dtype).min                                               # ... and all of them alike
    check_distill(z, ids, t, temperature, None)


@pytest.mark.parametrize("teacher,offset", [("f32", -1e6), ("f32", -1e4), ("f32", 1e3), ("f32", 1e5), ("bf16", 1e4), ("f16", 6e4)])
@pytest.mark.parametrize("temperature", [0.5, 0.7, 1.0, 3.0])
def test_a_teacher_with_an_offset_and_a_tail(teacher, offset, temperature):
    """q from the given values, the given log-sum-exp, which f32 holds to 0.03 at 1e6, and the given temperature, an f32 number too."""
    temperature = float(torch.tensor(temperature, dtype=torch.float32))
    z = make_logits(40, 3001, "f32", seed=66)
    ids = make_list(z, 20, 1.0, False)[0]
    t = (shifted(40, 20, "f32", 0.0, seed=67) + offset).to(TYPES[teacher])
    check_distill(z, ids, t, temperature, (torch.logsumexp(t.double() / temperature, 1) + 0.5).float())


@pytest.mark.parametrize("k", [1, 5, 64, 256])
@pytest.mark.parametrize("level", [0.0, 20.0, -100.0, 1000.0])
@pytest.mark.parametrize("outside", [None, -math.inf, -1e9, -3e38, -300.0])
def test_no_tail_of_either_has_a_finite_loss(k, level, outside):
    """A list that holds all of the teacher's and all of the student's mass: 1 - sum q is a rounding, not a tail."""
    from paper_2602_01274_b200 import binding as b
    rows, vocab = 500, k if outside is None else k + 300
    inside = torch.randn(rows, k, generator=gen(70), device=DEV)
    z = torch.full((rows, vocab), outside or 0.0, device=DEV)
    ids = torch.rand(rows, vocab, generator=gen(71), device=DEV).topk(k, 1).indices
    z.scatter_(1, ids, inside)
    ids = ids.to(torch.int32)
    t = torch.randn(rows, k, generator=gen(72), device=DEV) * 2 + level
    tl, w = torch.logsumexp(t, 1), torch.ones(rows, device=DEV)
    want, _, _, d0, terms = ref.distill(z, ids, t, 1.0, None, w)       # (the list renormalised)
    logs = size(ref.softmax_parts(z.double())[0].gather(1, ids.long())).amax(1)
    # the q sum to 1 but for the log-sum-exp's own rounding and the list's: 2^-24 (40 + 4 |lse|), times logarithms of at most logs + 20
    rest = ref.F32 * (40 + 4 * tl.double().abs())
    loss, d = b.pacer_distill_grad(z, ids, t, w, 1.0, tl)
    close(loss, want, 4 * EPS + 106 * ref.F32 * logs + rest * (logs + 20), "loss")
    others = torch.ones_like(z, dtype=torch.bool).scatter(1, ids.long(), False)
    close(d, d0, 4 * EPS * terms + 2 * rest[:, None] * torch.where(others, 1.0, terms), "gradient")
    # what is more than a rounding is a tail
    loss, _, tail = b.pacer_distill(z, ids, t, 1.0, tl + 0.05 * max(1.0, abs(level)))
    assert (loss > 5.0).all() and (outside is not None and outside > -1e38 or (loss > 1e30).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,k", [(64, 64), (256, 256), (3, 3), (4099, 20)])
def test_rows_with_nan_are_nan_whatever_the_list_holds(dtype, vocab, k):
    """NaN inside the list, outside it and everywhere, beside -inf and beside numbers, with a tail and without."""
    from paper_2602_01274_b200 import binding as b
    z = make_logits(7, vocab, dtype, seed=80)
    ids = torch.arange(k, device=DEV, dtype=torch.int32).flip(0).repeat(7, 1)
    z[0] = math.nan
    z[1] = -math.inf
    z[1, k - 1] = math.nan                              # one listed NaN, nothing else left
    z[2, 0] = math.nan
    z[3, -1] = math.nan
    z[4, k:] = math.nan                                 # (nothing where the list is the whole vocabulary)
    t = torch.randn(7, k, generator=gen(81), device=DEV)
    w = torch.ones(7, device=DEV)
    bad = [0, 1, 2, 3] + ([4] if vocab > k else [])
    good = [r for r in range(7) if r not in bad]
    for tl in (None, torch.logsumexp(t, 1) + 0.3):
        loss, lse, tail = b.pacer_distill(z, ids, t, 1.0, tl)
        _, d = b.pacer_distill_grad(z, ids, t, w, 1.0, tl)
        d2 = b.pacer_distill_backward(z, ids, t, lse, tail, w, 1.0, tl)
        for r in bad:
            assert torch.isnan(loss[r]) and torch.isnan(lse[r]) and torch.isnan(d[r]).all() and torch.isnan(d2[r]).all(), (r, tl is None)
        for r in good:
            assert not torch.isnan(loss[r]) and torch.isfinite(lse[r]) and torch.isfinite(d[r]).all() and torch.isfinite(d2[r]).all(), (r, tl is None)


@pytest.mark.parametrize("rows,vocab", [(2000, 1), (2000, 7), (2000, 1000), (300, 32003), (40, 151936)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_no_probability_above_one(rows, vocab, dtype):
    """Rows that are sure of one token: no log probability above 0, no entropy below."""
    from paper_2602_01274_b200 import binding as b
    z = torch.randn(rows, vocab, generator=gen(90), device=DEV) * 10
    at = torch.randint(0, vocab, (rows, 1), generator=gen(91), device=DEV)
    z.scatter_(1, at, z.amax(1, keepdim=True) + 40 * torch.rand(rows, 1, generator=gen(92), device=DEV))
    logp, ent, _, _, tlp = check_rows(z.to(TYPES[dtype]), at[:, 0].to(torch.int32), min(vocab, 3))
    assert (logp <= 0).all() and (tlp <= 0).all() and (ent >= 0).all()
    h, w = torch.zeros(rows, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(min(vocab, 4099), 64, dtype=torch.bfloat16, device=DEV)
    h[:, 0] = 1 + torch.rand(rows, generator=gen(93), device=DEV)
    w[:, 0] = z[0, :len(w)]
    logp, ent, _ = b.pacer_head_logprobs(h, w, w[:, 0].argmax().to(torch.int32).expand(rows))
    assert (logp <= 0).all() and (ent >= 0).all()
