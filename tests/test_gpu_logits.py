"""Log probabilities of given tokens, entropy and alternatives, their gradients, and distillation from a teacher's top logits,
against plain 64-bit forms on the same inputs.

Tolerances.  A row's sum of exponentials in fp32: an exponent |t| <= 40 is off by at most 3 |t| half steps (difference, scaling,
product's operand), ex2 itself by four, a thread's two running sums (even and odd elements) of at most 150 terms each (the largest
vocabulary over 8 blocks of 256 threads, or 70 001 over one) by 150: S, and each p, are right to
EPS = (3 * 40 * ln 2 + 4 + 150) half steps < 240 * 2^-24 = 1.5e-5, and so is its logarithm, absolutely.  lse and logp add roundings of their own size, four half steps at most."""
import math

import pytest
import torch

from tests import logit_refs as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 240 * ref.F32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def make_logits(rows, vocab, dtype, pad=0, offset=0, seed=0, spread=2.0):
    """[rows][vocab] with `pad` elements between rows, beginning `offset` elements into its storage."""
    flat = torch.randn(rows * (vocab + pad) + offset, generator=gen(seed), device=DEV) * spread
    return flat.to(TYPES[dtype])[offset:].view(rows, vocab + pad)[:, :vocab]


def make_tokens(rows, vocab, seed=1):
    t = torch.randint(0, vocab, (rows,), generator=gen(seed), device=DEV, dtype=torch.int32)
    t[::5] = -1
    return t


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf]), what
    fine = torch.isfinite(want)
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or over.max() <= 0, (what, float(over.max()))


def check_logprobs(z, tokens, top):
    from paper_2602_01274_b200 import binding as b
    logp, ent, lse, ids, tlp = b.pacer_logprobs(z, tokens, top)
    want_logp, want_ent, want_lse, lp = ref.logprobs(z, tokens)
    size = z.double().abs().nan_to_num(0, 0, 0).max() + want_lse.abs().nan_to_num(0, 0, 0)
    close(lse, want_lse, EPS + 4 * ref.F32 * size, "lse")
    close(logp, want_logp, EPS + 4 * ref.F32 * size, "logp")
    # each p_v off by EPS, its exponent's distance from the mean at most 40
    close(ent, want_ent, 40 * EPS, "entropy")
    want_ids = ref.order_rows(z, top)
    assert torch.equal(ids.long(), want_ids)
    close(tlp, lp.gather(1, want_ids), (EPS + 4 * ref.F32 * size)[:, None], "alternatives")
    again = b.pacer_logprobs(z, tokens, top)
    assert all(torch.equal(x, y) for x, y in zip(again, (logp, ent, lse, ids, tlp)))


@pytest.mark.parametrize("rows,vocab,pad,offset,dtype,top", [
    (1, 1, 0, 0, "f32", 1), (3, 2, 0, 0, "bf16", 2), (2, 7, 0, 1, "bf16", 7), (5, 3, 1, 3, "f16", 0),
    (4, 8, 0, 0, "bf16", 3), (7, 33, 0, 0, "f32", 20), (6, 100, 4, 0, "f16", 100), (9, 127, 0, 5, "bf16", 127),
    (11, 2048, 0, 0, "f32", 128),                      # fewer whole vectors a thread than alternatives
    (17, 4096, 0, 0, "f32", 5), (600, 4099, 0, 0, "bf16", 20), (2, 4097, 0, 3, "f32", 64),
    (1, 32000, 0, 0, "bf16", 20), (25, 32256, 0, 0, "f32", 1), (136, 32003, 61, 0, "bf16", 64), (700, 32003, 0, 0, "f16", 20),
    (1, 151936, 0, 0, "f32", 20), (1, 151936, 0, 0, "f32", 128), (33, 151936, 0, 0, "bf16", 128), (3, 151937, 2, 1, "f16", 64),
    # rows of one warp each
    (1024, 1, 0, 0, "f32", 1), (1025, 7, 0, 1, "bf16", 7), (2000, 127, 0, 5, "f16", 127), (5000, 300, 3, 0, "f32", 128),
    (1100, 4099, 61, 0, "bf16", 64), (1024, 32003, 0, 0, "f16", 20), (1500, 2048, 0, 0, "f32", 0), (1030, 70001, 0, 3, "bf16", 128),
])
def test_logprobs(rows, vocab, pad, offset, dtype, top):
    check_logprobs(make_logits(rows, vocab, dtype, pad, offset, seed=vocab + rows), make_tokens(rows, vocab), top)


@pytest.mark.parametrize("rows", [1, 40, 600, 1100])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprobs_of_masked_rows(rows, dtype):
    vocab, top = 32003, 20
    z = make_logits(rows, vocab, dtype, seed=3)
    z[:, 1000:] = -math.inf                             # a grammar leaves a part
    z[0] = -math.inf                                    # ... nothing
    if rows > 1:
        z[1, 5:] = -math.inf                            # ... fewer than the alternatives
        z[2] = torch.finfo(z.dtype).min                 # a mask of the type's lowest value, everywhere
        z[3, 7:] = torch.finfo(z.dtype).min
        z[4] = 1.0                                      # ties, and zeros of both signs
        z[5] = 0.0
        z[5, ::2] = -0.0
        z[6, :] = -1e9 if dtype == "f32" else -1e4
        z[7] = -math.inf
        z[7, -1] = 3.0                                  # one token is left: the last
        if dtype != "f16":                              # finite masks of any size, in front of what is left and behind it
            for r, v in enumerate((-1e8, -1e10, -1e20, -3e38)):
                z[8 + 2 * r, :-500] = v
                z[9 + 2 * r, 500:] = v
                z[16 + r] = v
    tokens = make_tokens(rows, vocab)
    tokens[0] = 17
    check_logprobs(z, tokens, top)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 151936, "f32"), (300, 32000, "bf16"), (1024, 32000, "bf16")])
def test_alternatives_that_sit_in_few_threads(rows, vocab, dtype):
    """The best elements all in vectors that one thread reads: more candidates than the block keeps at a time."""
    z = make_logits(rows, vocab, dtype, seed=4)
    z[:, :] = z.abs().neg()
    E = 16 // z.element_size()
    for step in (256, 32, 8):                           # vectors of one thread of a block, of one lane, of an eighth of the threads
        z.view(rows, -1, E)[:, ::step] += 64.0
        check_logprobs(z, make_tokens(rows, vocab), 64)
    z = (torch.arange(vocab, device=DEV) // 50).float().expand(rows, vocab).contiguous()   # ascending, ties of 50
    check_logprobs(z / z.max() * 20, make_tokens(rows, vocab), 128)
    check_logprobs(-z / z.max() * 20, make_tokens(rows, vocab), 128)


@pytest.mark.parametrize("rows", [6, 1030])
def test_logprobs_of_rows_with_nan_and_inf(rows):
    from paper_2602_01274_b200 import binding as b
    z = make_logits(rows, 5000, "f32", seed=5)
    z[0, 17] = math.nan
    z[1] = math.nan
    z[2, 4:] = math.nan
    z[2, :2] = -math.inf
    z[3, 100] = math.inf
    z[4] = -math.inf
    z[4, 3000:] = math.nan
    tokens = torch.arange(rows, dtype=torch.int32, device=DEV)
    logp, ent, lse, ids, tlp = b.pacer_logprobs(z, tokens, 100)
    for r in range(5):
        assert torch.isnan(lse[r]) and torch.isnan(ent[r]) and torch.isnan(logp[r]) and torch.isnan(tlp[r]).all()
    for r in range(6):
        assert ids[r].tolist() == ref.order(z[r], 100), r
    # a row's neighbours are as without it
    one = b.pacer_logprobs(z[5:], tokens[5:], 100)
    assert torch.equal(one[3], ids[5:]) and torch.isfinite(lse[5:]).all()


@pytest.mark.parametrize("rows,vocab,pad,offset,dtype,use", [
    (1, 1, 0, 0, "f32", "lhs"), (3, 5, 0, 1, "bf16", "lhs"), (5, 7, 3, 0, "f16", "l"), (17, 4096, 0, 0, "f32", "h"),
    (1, 151936, 0, 0, "f32", "lh"), (25, 32003, 0, 0, "bf16", "lhs"), (600, 4099, 61, 0, "f32", "s"), (33, 32256, 0, 3, "f16", "lhs"),
])
def test_logprobs_backward(rows, vocab, pad, offset, dtype, use):
    from paper_2602_01274_b200 import binding as b
    z = make_logits(rows, vocab, dtype, pad, offset, seed=7)
    if vocab > 100:
        z[:, 50:60] = -math.inf
        z[-1] = -math.inf if rows > 1 else z[-1]
    tokens = make_tokens(rows, vocab)
    tokens[-1] = 0
    g = {k: torch.randn(rows, generator=gen(8 + i), device=DEV) if k in use else None for i, k in enumerate("lhs")}
    _, ent, lse, _ = ref.logprobs(z, tokens)
    lse, ent = lse.float(), ent.float()
    want, size = ref.logprobs_grad(z, tokens, lse, ent, g["l"], g["h"], g["s"])
    args = (tokens if "l" in use else None, lse, ent if "h" in use else None, g["l"], g["h"], g["s"])
    got = b.pacer_logprobs_backward(z, *args)
    # p from the given lse: the exponent (at most 40) is off by 4 * 40 half steps, ex2 by four, the terms by a few more; then one
    # rounding to the type
    half, least = ref.rounding(z.dtype)
    close(got, want, half * want.abs() * 1.01 + (1 + half) * 180 * ref.F32 * size + least, "dlogits")
    # other rows than the logits' (shifted by one element), and in place
    other = torch.full((rows, vocab + 3), 7.0, device=DEV, dtype=z.dtype)
    b.pacer_logprobs_backward(z, *args, out=other[:, 1:vocab + 1])
    assert torch.equal(other[:, 1:vocab + 1], got) and (other[:, 0] == 7).all() and (other[:, vocab + 1:] == 7).all()
    base = z._base if z._base is not None else z
    rest = base.clone()
    b.pacer_logprobs_backward(z, *args, out=z)
    assert torch.equal(z, got)
    z.copy_(torch.as_strided(rest, z.shape, z.stride(), z.storage_offset()))
    assert torch.equal(base, rest)                       # nothing between the rows was touched


def test_logprobs_backward_of_rows_that_f32_lse_cannot_tell_apart():
    from paper_2602_01274_b200 import binding as b
    for dtype, rows in (("f32", 3), ("bf16", 700)):
        z = make_logits(rows, 8192, dtype, seed=9)
        z[0] = torch.finfo(z.dtype).min
        z[1] = -1e9
        tokens = torch.zeros(rows, dtype=torch.int32, device=DEV)
        _, ent, lse, _, _ = b.pacer_logprobs(z, tokens)
        one = torch.ones(rows, device=DEV)
        want = torch.full((2, 8192), -1 / 8192.0, dtype=torch.float64)
        want[:, 0] += 1
        half, least = ref.rounding(z.dtype)
        got = b.pacer_logprobs_backward(z, tokens, lse, ent, one)
        close(got[:2].cpu(), want, (half + 2 * EPS) * want.abs() + least, "uniform rows")
        b.pacer_logprobs_backward(z, tokens, lse, ent, one, out=z)
        assert torch.equal(z, got)


def test_gradients_against_differences():
    """Directional differences of the operators' own fp32 values: error h^2 / 6 times the third derivative (of order one) and the
    values' own 2e-5 over h."""
    from paper_2602_01274_b200 import binding as b
    rows, vocab, h = 6, 67, 0.02
    z = make_logits(rows, vocab, "f32", seed=10)
    tokens = torch.tensor([3, -1, 66, 0, 5, 9], dtype=torch.int32, device=DEV)
    u = torch.randn(rows, vocab, generator=gen(11), device=DEV)
    u /= u.norm(dim=1, keepdim=True)
    _, ent, lse, _, _ = b.pacer_logprobs(z, tokens)
    one, none = torch.ones(rows, device=DEV), None
    up, down = b.pacer_logprobs(z + h * u, tokens), b.pacer_logprobs(z - h * u, tokens)
    bound = h * h * 2 + 2 * EPS * 40 / h
    for i, g in enumerate([(one, none, none), (none, one, none), (none, none, one)]):
        d = (b.pacer_logprobs_backward(z, tokens, lse, ent, *g) * u).sum(1)
        close(d, (up[i] - down[i]) / (2 * h), bound, i)
    ids = torch.randint(0, vocab, (rows, 9), generator=gen(12), device=DEV, dtype=torch.int32)
    t = torch.randn(rows, 9, generator=gen(13), device=DEV)
    for tl in (None, torch.logsumexp(t / 1.5, 1) + 0.3):
        _, d = b.pacer_distill_grad(z, ids, t, one, 1.5, tl)
        du, dd = b.pacer_distill(z + h * u, ids, t, 1.5, tl)[0], b.pacer_distill(z - h * u, ids, t, 1.5, tl)[0]
        close((d * u).sum(1), (du - dd) / (2 * h), bound, "distill")


def make_teacher(rows, vocab, k, tail, temperature, dtype="f32", seed=20, spoil=True):
    g = gen(seed)
    ids = torch.randint(0, vocab, (rows, k), generator=g, device=DEV, dtype=torch.int32)
    t = (torch.randn(rows, k, generator=g, device=DEV) * 2 + 3).to(TYPES[dtype])
    if spoil and rows > 3:
        ids[1] = -1                                     # no entry at all
        if k > 2:
            ids[2, ::2] = -1
            ids[3, 1] = ids[3, 0]                       # listed twice
            ids[3, 2] = vocab                           # outside
            t[2, 1] = -math.inf                         # the teacher excludes it
    lse = None
    if tail:
        lse = torch.logsumexp(t.float() / temperature, 1) + 0.05 + torch.rand(rows, generator=g, device=DEV)
    return ids, t, lse


@pytest.mark.parametrize("rows,vocab,pad,offset,dtype,k,temperature,tail", [
    (1, 1, 0, 0, "f32", 1, 1.0, False), (4, 3, 0, 1, "bf16", 2, 2.0, True), (5, 17, 1, 0, "f16", 9, 0.5, True),
    (9, 1000, 0, 0, "f32", 256, 1.0, True), (17, 4096, 0, 0, "bf16", 64, 1.0, False), (17, 4096, 0, 0, "f32", 64, 3.0, True),
    (600, 4099, 61, 0, "bf16", 20, 1.0, True), (2, 32003, 0, 3, "f32", 1, 1.0, False), (25, 32003, 0, 0, "f16", 8, 2.0, True),
    (1, 151936, 0, 0, "f32", 100, 0.7, True), (33, 151937, 0, 0, "bf16", 33, 1.0, True), (300, 32256, 0, 0, "f32", 200, 1.0, False),
])
def test_distill(rows, vocab, pad, offset, dtype, k, temperature, tail):
    from paper_2602_01274_b200 import binding as b
    z = make_logits(rows, vocab, dtype, pad, offset, seed=21)
    if vocab > 100:
        z[:, 50:60] = -math.inf
    ids, t, tl = make_teacher(rows, vocab, k, tail, temperature, {"f32": "f32", "bf16": "bf16", "f16": "f32"}[dtype])
    if vocab > 100:                                     # (a listed token of probability 0 has an infinite loss: its own test below)
        ids = torch.where((ids >= 50) & (ids < 60), ids + 10, ids)
    if rows > 6:
        z[5] = -math.inf
    w = torch.randn(rows, generator=gen(22), device=DEV)
    want = ref.distill(z, ids, t, temperature, tl, w)
    loss, lse, tail_lse = b.pacer_distill(z, ids, t, temperature, tl)
    # log q, log p and their difference (magnitudes up to 100) to 8 half steps and EPS, summed with weights that add up to at most 1;
    # q_t = 1 - sum q to EPS absolutely, times the log of a ratio of at most e^30
    bound = 30 * 2 * EPS
    close(loss, want[0], bound, "loss")
    close(lse, want[1], EPS + 4 * ref.F32 * want[1].abs().nan_to_num(0, 0, 0) + 1e-6, "lse")
    if tail:
        close(tail_lse, want[2], EPS + 4 * ref.F32 * want[2].abs().nan_to_num(0, 0, 0) + 1e-6, "tail")
    else:
        assert tail_lse is None
    half, least = ref.rounding(z.dtype)
    grad_bound = half * 1.01 * want[3].abs() + 4 * EPS * want[4] + least
    loss2, d = b.pacer_distill_grad(z, ids, t, w, temperature, tl)
    assert torch.equal(loss, loss2)
    close(d, want[3], grad_bound, "dlogits")
    d2 = b.pacer_distill_backward(z, ids, t, lse, tail_lse, w, temperature, tl)
    # (from the rounded lse: 40 |lse| half steps of the exponent more)
    close(d2, want[3], grad_bound + 40 * 4 * ref.F32 * want[4], "dlogits, second call")
    other = torch.full((rows, vocab + 3), 7.0, device=DEV, dtype=z.dtype)
    b.pacer_distill_grad(z, ids, t, w, temperature, tl, out=other[:, 1:vocab + 1])
    assert torch.equal(other[:, 1:vocab + 1], d) and (other[:, 0] == 7).all() and (other[:, vocab + 1:] == 7).all()
    copy = make_logits(rows, vocab, dtype, pad, offset, seed=21)
    copy.copy_(z)
    _, inplace = b.pacer_distill_grad(z, ids, t, w, temperature, tl, out=z)
    assert torch.equal(inplace, d)
    b.pacer_distill_backward(copy, ids, t, lse, tail_lse, w, temperature, tl, out=copy)
    assert torch.equal(copy, d2)


def test_distill_at_its_limits():
    from paper_2602_01274_b200 import binding as b
    V = 64
    one = torch.ones(4, device=DEV)
    ids = torch.arange(V, device=DEV, dtype=torch.int32).repeat(4, 1)
    z = make_logits(4, V, "f32", seed=23)
    t = torch.randn(4, V, generator=gen(24), device=DEV)
    # the list is the whole vocabulary: nothing is left for the tail
    tl = torch.logsumexp(t, 1)
    loss, _, tail = b.pacer_distill(z, ids, t, 1.0, tl)
    assert (tail == -math.inf).all()
    want = ref.distill(z, ids, t, 1.0, None, one)
    _, d = b.pacer_distill_grad(z, ids, t, one, 1.0)
    close(d, want[3], 4 * EPS * want[4], "whole list")
    # q_t may be a rounding above zero, and the student has nothing there
    assert all(x == math.inf or abs(x - y) < 60 * EPS for x, y in zip(loss.tolist(), want[0].tolist()))
    # a student that is sure of the list keeps its tail
    z = torch.zeros(4, V, device=DEV)
    z[:, 0] = 30.0
    ids, t, tl = torch.zeros(4, 1, dtype=torch.int32, device=DEV), torch.zeros(4, 1, device=DEV), torch.full((4,), 0.5, device=DEV)
    want = ref.distill(z, ids, t, 1.0, tl, one)
    loss, d = b.pacer_distill_grad(z, ids, t, one, 1.0, tl)
    close(loss, want[0], 60 * EPS, "sure of the list")
    close(d, want[3], 4 * EPS * want[4], "sure of the list")
    # a listed token that the student excludes: infinite loss, finite gradient
    z[:, 0] = -math.inf
    loss, d = b.pacer_distill_grad(z, ids, t, one, 1.0)
    assert (loss == math.inf).all() and (d[:, 0] == -1).all() and torch.isfinite(d).all()
    loss, lse, tail = b.pacer_distill(z, ids, t, 1.0, tl)                # ... with a tail: all that is left is outside the list
    want = torch.full((4, V), (1 - (1 - math.exp(-0.5))) / (V - 1), dtype=torch.float64, device=DEV)      # p_v Q - q_t w_v, p_v = w_v
    want[:, 0] = -math.exp(-0.5)
    assert (loss == math.inf).all() and torch.equal(lse, tail)
    close(lse, torch.full((4,), math.log(V - 1), device=DEV), 2 * EPS, "excluded list, lse")
    close(b.pacer_distill_grad(z, ids, t, one, 1.0, tl)[1], want, 4 * EPS, "excluded list")
    close(b.pacer_distill_backward(z, ids, t, lse, tail, one, 1.0, tl), want, 4 * EPS, "excluded list, second call")
    # rows at the type's lowest value are uniform
    z[:] = torch.finfo(torch.float32).min
    loss, lse, _ = b.pacer_distill(z, ids, t, 0.7)
    _, d = b.pacer_distill_grad(z, ids, t, one, 0.7)
    d2 = b.pacer_distill_backward(z, ids, t, lse, None, one, 0.7)
    want = torch.full((4, V), 1 / V / 0.7, dtype=torch.float64, device=DEV)
    want[:, 0] -= 1 / 0.7
    close(loss, torch.full((4,), math.log(V), device=DEV), 2 * EPS, "lowest")
    close(d, want, 4 * EPS, "lowest")
    close(d2, want, 4 * EPS, "lowest, second call")
    loss, lse, tail = b.pacer_distill(z, ids, t, 0.7, tl)
    d2 = b.pacer_distill_backward(z, ids, t, lse, tail, one, 0.7, tl)
    d = b.pacer_distill_grad(z, ids, t, one, 0.7, tl)[1]
    close(d2, d, 8 * EPS, "lowest with a tail")
    z[:, 0] = 2.0                                        # ... or the others alone: they share the tail's part evenly
    want = torch.full((4, V), -(1 - math.exp(-0.5)) / (V - 1), dtype=torch.float64, device=DEV)
    want[:, 0] = 1 - math.exp(-0.5)
    z[:2, 1:] = -1e9
    loss, lse, tail = b.pacer_distill(z, ids, t, 1.0, tl)
    close(b.pacer_distill_grad(z, ids, t, one, 1.0, tl)[1], want, 4 * EPS, "others at the lowest")
    close(b.pacer_distill_backward(z, ids, t, lse, tail, one, 1.0, tl), want, 4 * EPS, "others at the lowest, second call")


@pytest.mark.parametrize("dtype,mask", [("f32", -1e8), ("f32", -1e10), ("f32", -1e20), ("f32", -3.4e38), ("bf16", -1e10),
                                        ("bf16", -3.38e38), ("f16", -65504.0)])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 10.0])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_of_rows_masked_with_finite_values(dtype, mask, temperature, tail):
    """A finite mask leaves what -inf would leave; a row of nothing else is a row of zeros."""
    from paper_2602_01274_b200 import binding as b
    rows, vocab = 6, 9001
    ids, t, tl = make_teacher(rows, vocab, 7, tail, temperature, spoil=False)
    ids = ids % 400 + vocab - 500                       # the list lies in what is left of rows 0 and 3
    z = make_logits(rows, vocab, dtype, seed=34)
    plain = z.clone()
    z[0, :-500], plain[0, :-500] = mask, -math.inf
    z[1], plain[1] = mask, 0.0
    z[3, :-500:2], plain[3, :-500:2] = mask, -math.inf
    w = torch.ones(rows, device=DEV)
    got, want = b.pacer_distill_grad(z, ids, t, w, temperature, tl), ref.distill(plain, ids, t, temperature, tl, w)
    close(got[0], want[0], 60 * EPS, "loss")
    half, least = ref.rounding(z.dtype)
    close(got[1], want[3], half * 1.01 * want[3].abs() + 4 * EPS * want[4] + least, "dlogits")
    _, lse, tail_lse = b.pacer_distill(z, ids, t, temperature, tl)
    again = b.pacer_distill_backward(z, ids, t, lse, tail_lse, w, temperature, tl)
    close(again, want[3], half * 1.01 * want[3].abs() + (4 * EPS + 160 * ref.F32) * want[4] + least, "dlogits, second call")


def test_rows_beyond_32_bit_offsets():
    from paper_2602_01274_b200 import binding as b
    rows, vocab, ld = 17000, 1000, 131072                # 2.2e9 elements from the first row to the last
    z = torch.empty(rows, ld, dtype=torch.bfloat16, device=DEV)[:, :vocab]
    z.copy_(make_logits(rows, vocab, "bf16", seed=30))
    tokens = make_tokens(rows, vocab)
    got, small = b.pacer_logprobs(z, tokens, 5), b.pacer_logprobs(z.contiguous(), tokens, 5)
    assert all(torch.equal(x, y) for x, y in zip(got, small))
    w = torch.ones(rows, device=DEV)
    ids, t, tl = make_teacher(rows, vocab, 4, True, 1.0)
    want = b.pacer_logprobs_backward(z.contiguous(), tokens, got[2], got[1], w, w)
    want2 = b.pacer_distill_grad(z.contiguous(), ids, t, w, 1.0, tl)[1]
    copy = z.contiguous()
    b.pacer_logprobs_backward(z, tokens, got[2], got[1], w, w, out=z)
    assert torch.equal(z, want)
    z.copy_(copy)
    b.pacer_distill_grad(z, ids, t, w, 1.0, tl, out=z)
    assert torch.equal(z, want2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_largest_vocabulary(dtype):
    from paper_2602_01274_b200 import binding as b
    rows, vocab = 3, b.PACER_MAX_VOCAB
    z = make_logits(rows, vocab, dtype, 0, 1, seed=32)
    check_logprobs(z, make_tokens(rows, vocab), 128)
    ids, t, tl = make_teacher(rows, vocab, 256, True, 1.0)
    ids[0, :4] = torch.tensor([0, vocab - 1, vocab - 2, 1], device=DEV)
    w = torch.ones(rows, device=DEV)
    want = ref.distill(z, ids, t, 1.0, tl, w)
    loss, d = b.pacer_distill_grad(z, ids, t, w, 1.0, tl)
    close(loss, want[0], 60 * EPS, "loss")
    half, least = ref.rounding(z.dtype)
    close(d, want[3], half * 1.01 * want[3].abs() + 4 * EPS * want[4] + least, "dlogits")
    with pytest.raises(b.PacerError, match="vocab out of range"):
        b.pacer_logprobs(torch.zeros(1, vocab + 1, device=DEV), make_tokens(1, 5))


def test_outputs_that_cannot_be_written_are_refused():
    from paper_2602_01274_b200 import binding as b
    z = make_logits(4, 50, "f32", seed=33)
    t, w = make_tokens(4, 50), torch.ones(4, device=DEV)
    _, ent, lse, _, _ = b.pacer_logprobs(z, t)
    for out in (torch.empty(1, 50, device=DEV).expand(4, 50), torch.empty(4, 50, device=DEV, dtype=torch.bfloat16), torch.empty(4, 49, device=DEV),
                torch.empty(50, 4, device=DEV).t(), torch.empty(4, 50)):
        with pytest.raises(AssertionError, match="out: like the logits"):
            b.pacer_logprobs_backward(z, t, lse, ent, w, out=out)
    with pytest.raises(b.PacerError, match="overlaps"):
        flat = torch.empty(4 * 50 + 50, device=DEV)
        b.pacer_logprobs_backward(flat[:200].view(4, 50), t, lse, ent, w, out=flat[50:].view(4, 50))
    with pytest.raises(AssertionError, match="tokens"):
        b.pacer_logprobs(z, t.long())
    with pytest.raises(AssertionError, match="tokens"):
        b.pacer_logprobs(z, t.cpu())
    with pytest.raises(AssertionError, match="logits"):
        b.pacer_logprobs(z.double(), t)


def test_no_rows():
    from paper_2602_01274_b200 import binding as b
    z = torch.empty(0, 100, device=DEV)
    e, i = torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    assert [tuple(x.shape) for x in b.pacer_logprobs(z, i, 3)] == [(0,), (0,), (0,), (0, 3), (0, 3)]
    assert b.pacer_logprobs_backward(z, i, e, e, e).shape == (0, 100)
    assert b.pacer_distill(z, i.view(0, 1), e.view(0, 1))[0].shape == (0,)
    assert b.pacer_distill_grad(z, i.view(0, 1), e.view(0, 1), e)[1].shape == (0, 100)


def test_other_streams_and_graphs():
    """Two calls at once on two streams, and a captured call replayed on new inputs, give what plain calls give."""
    from paper_2602_01274_b200 import binding as b
    z = [make_logits(n, 32003, "bf16", seed=n) for n in (9, 700)]
    tokens = [make_tokens(x.shape[0], 32003) for x in z]
    lists = [make_teacher(x.shape[0], 32003, 20, True, 1.0) for x in z]

    def both(i):
        a = b.pacer_logprobs(z[i], tokens[i], 20)
        w = torch.ones(z[i].shape[0], device=DEV)
        loss, d = b.pacer_distill_grad(z[i], lists[i][0], lists[i][1], w, 1.0, lists[i][2])
        return (*a, b.pacer_logprobs_backward(z[i], tokens[i], a[2], a[1], w, w), loss, d)

    want = [both(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            for _ in range(3):
                got[i] = both(i)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, y) for x, y in zip(got[i], want[i]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(0)
    keep = z[0].clone()
    z[0].copy_(z[0].flip(1))
    graph.replay()
    flipped = [x.clone() for x in out]
    assert all(torch.equal(x, y) for x, y in zip(flipped, both(0)))
    z[0].copy_(keep)
    graph.replay()
    assert all(torch.equal(x, y) for x, y in zip(out, want[0]))


def test_one_row_in_place_whatever_its_stride():
    from paper_2602_01274_b200 import binding as b
    z = torch.randn(1, 70, device=DEV)[:, :61].clone()       # a single row: contiguous, with a stride of 70
    t, w = make_tokens(1, 61), torch.ones(1, device=DEV)
    ids, teacher, _ = make_teacher(1, 61, 5, False, 1.0)
    _, want = b.pacer_distill_grad(z, ids, teacher, w)
    keep = z.clone()
    assert torch.equal(b.pacer_distill_grad(keep, ids, teacher, w, out=keep)[1], want)
    _, ent, lse, _, _ = b.pacer_logprobs(z, t)
    want = b.pacer_logprobs_backward(z, t, lse, ent, w, w)
    assert torch.equal(b.pacer_logprobs_backward(z, t, lse, ent, w, w, out=z), want)


def test_inputs_of_any_stride():
    from paper_2602_01274_b200 import binding as b
    z = make_logits(300, 40, "f32", seed=31)
    t = make_tokens(40, 300)
    got, want = b.pacer_logprobs(z.t(), t, 3), b.pacer_logprobs(z.t().contiguous(), t, 3)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    row = z[:1].expand(5, 40)
    t = make_tokens(5, 40)
    assert all(torch.equal(x, y) for x, y in zip(b.pacer_logprobs(row, t, 3), b.pacer_logprobs(row.contiguous(), t, 3)))
    w = torch.ones((), device=DEV).expand(5)
    _, ent, lse, _, _ = b.pacer_logprobs(row, t)
    d = b.pacer_logprobs_backward(row, t, lse, ent, w)
    assert d.shape == (5, 40) and torch.equal(d, b.pacer_logprobs_backward(row.contiguous(), t, lse, ent, w.contiguous()))
