"""The gradients of the LM head fused with the scoring, against plain 64-bit products on the same bf16 inputs.

Tolerance, per element.  The logits are off by dz <= (d / 16 + 1) 2^-23 |h| |w| (the tensor cores truncate when they add), and so is
their log-sum-exp beside its own half step; p and its factors are then off by a share of 2 dz + 16 half steps of fp32 (the exponential's two,
factors and sums).  dz is rounded to bf16 (half a step of its value), its products of K terms are added with K / 16 truncations
of 2^-23, and the result is rounded to bf16.  Everything but the last is relative to the sum of the terms' sizes."""
import math

import pytest
import torch

from tests import logit_refs as ref
from tests.test_gpu_head_logprobs import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = ref.F32, 2.0 ** -8


def weights(rows, seed=7):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + rows)
    return [torch.randn(rows, generator=g, device=DEV) for _ in range(3)]


def logits(h, w, bias_ids, bias=8.0):
    z = h.double() @ w.double().T
    if bias_ids is not None:
        ok = (bias_ids >= 0) & (bias_ids < w.shape[0])
        z.scatter_add_(1, torch.where(ok, bias_ids, 0).long()[:, None], torch.where(ok, bias, 0.0).double()[:, None])
    return z


def slack(h, w, z, K):
    """(of dz relative to its terms, of a product over K terms relative to them), beside the rounding of dz."""
    d = h.shape[1]
    off = (d / 16 + 1) * 2 * F32 * h.double().norm(dim=1).max() * w.double().norm(dim=1).max()
    lse = torch.logsumexp(z, 1).abs().max()
    return float(2 * off + 2 * F32 * lse + 16 * F32) * (1 + float((z - torch.logsumexp(z, 1)[:, None]).abs().max())), (K / 16 + 1) * 2 * F32


def check(got, dz, size, other, by_rows, slack_z, slack_k, name):
    """got bf16 against dz @ other (by_rows) or dz.T @ other."""
    a, s = (dz, size) if by_rows else (dz.T, size.T)
    want = a @ other
    terms = (a.abs() * BF16 + s * slack_z + a.abs() * slack_k) @ other.abs()
    bound = 1.01 * terms + BF16 * (want.abs() + terms) + 1e-38
    over = ((got.double() - want).abs() - bound).max()
    assert torch.isfinite(got).all() and over <= 0, (name, float(over), float((got.double() - want).norm() / want.norm()))
    return float((got.double() - want).norm() / want.norm()) if want.norm() else 0.0


SHAPES = [
    (1, 1, 8, 0), (1, 2, 64, 0), (2, 31, 72, 0), (7, 33, 128, 8), (8, 257, 64, 0), (9, 1000, 200, 0), (1, 4096, 256, 0), (33, 4099, 768, 0),
    (64, 512, 264, 0), (65, 513, 136, 64), (127, 5003, 256, 0), (128, 8000, 128, 0), (129, 8003, 1032, 0), (256, 256, 256, 0), (257, 255, 320, 8),
    (300, 32256, 512, 0), (1000, 7777, 1024, 0), (5, 40007, 64, 0), (2048, 4096, 2048, 0), (1153, 1201, 5120, 0),
    # four k blocks of rows and more, with rows of the gradient that no 32-byte stores fit
    (600, 1001, 1032, 0), (700, 2003, 264, 8), (193, 300, 24, 0),
    # the largest vocabulary
    (17, 1 << 21, 64, 0),
]


@pytest.mark.parametrize("rows,vocab,d,pad", SHAPES)
@pytest.mark.parametrize("biased", [False, True])
def test_nll_grad(rows, vocab, d, pad, biased):
    from paper_2602_01274_b200 import binding as b
    h, w, tok, bias_ids = make(rows, vocab, d, pad)
    bias_ids = bias_ids if biased else None
    weight = weights(rows)[0]
    loss, dh, dw = b.pacer_head_nll_grad(h, w, tok, weight, bias_ids, 8.0)
    z = logits(h, w, bias_ids)
    lp, lse = ref.softmax_parts(z)
    named = (tok >= 0) & (tok < vocab)
    at = torch.where(named, tok, 0).long()[:, None]
    want = torch.where(named, -lp.gather(1, at)[:, 0], 0.0)
    off = (d / 16 + 1) * 2 * F32 * h.double().norm(dim=1) * w.double().norm(dim=1).max()
    assert ((loss.double() - want).abs() <= 2 * off + 240 * F32 + 4 * F32 * (z.abs().amax(1) + lse.abs())).all()
    assert (loss[~named] == 0).all()
    g = torch.where(named, weight, 0.0).double()[:, None]
    size = lp.exp() * g.abs()
    dz = (lp.exp() * g).scatter_add(1, at, g * torch.where(named, torch.expm1(lp.gather(1, at)[:, 0]) - lp.gather(1, at)[:, 0].exp(), 0.0)[:, None])
    size = size.scatter_add(1, at, torch.where(named[:, None], g.abs(), 0.0))
    sz, _ = slack(h, w, z, 0)
    check(dh, dz, size, w.double(), True, sz, (vocab / 16 + 1) * 2 * F32, "dhidden")
    check(dw, dz, size, h.double(), False, sz, (rows / 16 + 1) * 2 * F32, "dhead")
    # one of the two alone, and the same bits again
    only_h, only_w = b.pacer_head_nll_grad(h, w, tok, weight, bias_ids, 8.0, grads=(True, False)), b.pacer_head_nll_grad(h, w, tok, weight, bias_ids, 8.0, grads=(False, True))
    assert only_h[2] is None and only_w[1] is None and torch.equal(only_w[2], dw) and torch.equal(only_w[0], loss)
    check(only_h[1], dz, size, w.double(), True, sz, (vocab / 16 + 1) * 2 * F32, "dhidden alone")
    again = b.pacer_head_nll_grad(h, w, tok, weight, bias_ids, 8.0)
    assert all(torch.equal(x, y) for x, y in zip((loss, dh, dw), again))


@pytest.mark.parametrize("rows,vocab,d,pad", SHAPES[:16])
@pytest.mark.parametrize("which", ["logp", "entropy", "lse", "all"])
def test_logprobs_backward(rows, vocab, d, pad, which):
    from paper_2602_01274_b200 import binding as b
    h, w, tok, bias_ids = make(rows, vocab, d, pad)
    bias_ids = bias_ids if which == "all" else None
    logp, ent, lse = b.pacer_head_logprobs(h, w, tok, bias_ids, 8.0)
    gl, gh, gs = (g if which in (name, "all") else None for g, name in zip(weights(rows), ("logp", "entropy", "lse")))
    dh, dw = b.pacer_head_logprobs_backward(h, w, tok if gl is not None else None, logp if gl is not None else None, lse,
                                            ent if gh is not None else None, gl, gh, gs, bias_ids, 8.0)
    z = logits(h, w, bias_ids)
    dz, size = ref.logprobs_grad(z, tok, lse, ent, gl, gh, gs)
    sz, _ = slack(h, w, z, 0)
    check(dh, dz, size, w.double(), True, sz, (vocab / 16 + 1) * 2 * F32, "dhidden")
    check(dw, dz, size, h.double(), False, sz, (rows / 16 + 1) * 2 * F32, "dhead")


def test_confident_rows():
    """1 - p of a token that has nearly all of the mass keeps its relative accuracy."""
    from paper_2602_01274_b200 import binding as b
    g = torch.Generator(device=DEV).manual_seed(3)
    h = torch.randn(40, 64, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.zeros(500, 64, device=DEV, dtype=torch.bfloat16)
    tok = torch.arange(40, device=DEV, dtype=torch.int32)
    one = torch.ones(40, device=DEV)
    for bias in (8.0, 14.0, 20.0):
        loss, _, dw = b.pacer_head_nll_grad(h, w, tok, one, tok, bias)
        rest = 499 * math.exp(-bias)
        assert ((loss.double() - math.log1p(rest)).abs() <= 4 * F32 * (1 + bias)).all()
        dz = torch.full((40, 500), math.exp(-bias) / (1 + rest), device=DEV, dtype=torch.float64)
        dz[torch.arange(40), torch.arange(40)] = -rest / (1 + rest)
        # (1 - p from logp: half a step of S = 1 + rest, and of the logarithm)
        share = BF16 + 8 * F32 * (1 + bias + 1 / rest)
        want = dz.T @ h.double()
        assert ((dw.double() - want).abs() <= 1.01 * share * (dz.abs().T @ h.double().abs()) + BF16 * want.abs()).all()


@pytest.mark.parametrize("rows,vocab,d", [(75000, 16001, 72), (300000, 4000, 64)])
def test_pieces_of_the_vocabulary(rows, vocab, d):
    """More rows than dz of the whole vocabulary is kept for."""
    from paper_2602_01274_b200 import binding as b
    assert rows * vocab * 2 > 2 << 30
    h, w, tok, bias_ids = make(rows, vocab, d)
    weight = weights(rows)[0] / rows
    loss, dh, dw = b.pacer_head_nll_grad(h, w, tok, weight, bias_ids, 8.0)
    wide = w.double()
    want_w, size_w = torch.zeros(vocab, d, dtype=torch.float64, device=DEV), torch.zeros(vocab, d, dtype=torch.float64, device=DEV)
    for lo in range(0, rows, 10000):
        r = slice(lo, lo + 10000)
        z = logits(h[r], w, bias_ids[r])
        lp, _ = ref.softmax_parts(z)
        named = (tok[r] >= 0) & (tok[r] < vocab)
        at = torch.where(named, tok[r], 0).long()[:, None]
        g = torch.where(named, weight[r], 0.0).double()[:, None]
        dz = (lp.exp() * g).scatter_add(1, at, -g)
        size = (lp.exp() * g.abs()).scatter_add(1, at, g.abs())
        sz, _ = slack(h[r], w, z, 0)
        check(dh[r], dz, size, wide, True, sz, (vocab / 16 + 1) * 2 * F32, "dhidden")
        assert ((loss[r].double() + torch.where(named, lp.gather(1, at)[:, 0], 0.0)).abs() < 1e-4).all()
        want_w += dz.T @ h[r].double()
        size_w += (size * (BF16 + sz + (rows / 16 + 1) * 2 * F32)).T @ h[r].double().abs()
    assert ((dw.double() - want_w).abs() <= 1.01 * size_w + BF16 * (want_w.abs() + size_w)).all()


def test_differences():
    """The gradients against differences of the forward's own 64-bit form along a direction, in the small."""
    from paper_2602_01274_b200 import binding as b
    h, w, tok, bias_ids = make(24, 300, 64)
    weight = weights(24)[0]
    _, dh, dw = b.pacer_head_nll_grad(h, w, tok, weight, bias_ids, 8.0)
    g = torch.Generator(device=DEV).manual_seed(9)
    u, v = torch.randn(24, 64, generator=g, device=DEV).double(), torch.randn(300, 64, generator=g, device=DEV).double()
    named = (tok >= 0) & (tok < 300)

    def total(s):
        z = (h.double() + s * u) @ (w.double() + s * v).T
        ok = (bias_ids >= 0) & (bias_ids < 300)
        z = z.scatter_add(1, torch.where(ok, bias_ids, 0).long()[:, None], torch.where(ok, 8.0, 0.0).double()[:, None])
        l = torch.logsumexp(z, 1) - z.gather(1, torch.where(named, tok, 0).long()[:, None])[:, 0]
        return (torch.where(named, weight, 0.0).double() * l).sum()

    e = 1e-5
    want = (total(e) - total(-e)) / (2 * e)
    parts = (dh.double() * u).abs().sum() + (dw.double() * v).abs().sum()
    assert abs((dh.double() * u).sum() + (dw.double() * v).sum() - want) <= 3 * BF16 * parts


def test_outputs_of_the_caller_strides_and_versions():
    from paper_2602_01274_b200 import binding as b
    h, w, tok, bias_ids = make(50, 999, 136, pad=24)
    weight = weights(50)[0]
    loss, dh, dw = b.pacer_head_nll_grad(h, w, tok, weight)
    big_h, big_w = (torch.full((n, 160), 5.0, device=DEV, dtype=torch.bfloat16) for n in (52, 1001))
    out = (big_h[1:51, 8:144], big_w[1:1000, 8:144])
    version = big_h._version
    got = b.pacer_head_nll_grad(h, w, tok, weight, out=out)
    assert torch.equal(out[0], dh) and torch.equal(out[1], dw) and got[1] is out[0] and big_h._version > version
    for big, n in ((big_h, 50), (big_w, 999)):                              # what lies around is left as it was
        edge = big.clone()
        edge[1:n + 1, 8:144] = 5.0
        assert (edge == 5.0).all()
    with pytest.raises(AssertionError, match="out"):
        b.pacer_head_nll_grad(h, w, tok, weight, out=(torch.empty(50, 136, device=DEV), None))
    with pytest.raises(b.PacerError, match="overlaps"):
        b.pacer_head_nll_grad(h, w, tok, weight, out=(h, None))
    # more rows, gradients that begin off the 32-byte grid
    h, w, tok, _ = make(400, 999, 144)
    weight = weights(400)[0]
    _, dh, dw = b.pacer_head_nll_grad(h, w, tok, weight)
    out = tuple(torch.full((n, 160), 5.0, device=DEV, dtype=torch.bfloat16) for n in (400, 999))
    b.pacer_head_nll_grad(h, w, tok, weight, out=[x[:, 8:152] for x in out])
    assert torch.equal(out[0][:, 8:152], dh) and torch.equal(out[1][:, 8:152], dw)
    assert all((x[:, :8] == 5.0).all() and (x[:, 152:] == 5.0).all() for x in out)
    both = torch.empty(1049, 136, device=DEV, dtype=torch.bfloat16)
    h, w, tok, _ = make(50, 999, 136)
    with pytest.raises(b.PacerError, match="overlaps"):
        b.pacer_head_nll_grad(h, w, tok, weights(50)[0], out=(both[:50], both[49:1048]))


def test_scratch_between_calls_graphs_and_streams():
    """Scratch full of garbage, calls on two streams, and a captured call on new inputs."""
    from paper_2602_01274_b200 import binding as b
    from tests.common import filled_workspaces
    sets = [(*make(40, 8003, 256), weights(40)[0]), (*make(300, 5000, 520), weights(300)[0])]
    call = lambda s: b.pacer_head_nll_grad(s[0], s[1], s[2], s[4], s[3], 8.0)
    want = [call(s) for s in sets]
    with filled_workspaces(0xFF) as sizes:
        got = [call(s) for s in sets]
    assert len(sizes) == 2 and all(torch.equal(x, y) for g, v in zip(got, want) for x, y in zip(g, v))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            for _ in range(4):
                got[k] = call(sets[k])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g, v in zip(got, want) for x, y in zip(g, v))
    h, w, t, i, weight = sets[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(sets[0])
    for x in (h, t, i, weight):
        x.copy_(x.flip(0))
    graph.replay()
    new = call(sets[0])
    assert all(torch.equal(x, y) for x, y in zip(out, new)) and torch.equal(out[1], want[0][1].flip(0))


def test_no_rows():
    from paper_2602_01274_b200 import binding as b
    h, w, _, _ = make(1, 100, 64)
    e, f = torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV)
    loss, dh, dw = b.pacer_head_nll_grad(h[:0], w, e, f)
    assert loss.shape == (0,) and dh.shape == (0, 64) and (dw == 0).all()
    dh, dw = b.pacer_head_logprobs_backward(h[:0], w, e, f, f, f, f)
    assert dh.shape == (0, 64) and (dw == 0).all()


def test_one_row_whatever_its_stride():
    from paper_2602_01274_b200 import binding as b
    h, w, t, _ = make(1, 300, 64)
    t[:] = 3
    odd = torch.as_strided(h, (1, 64), (67, 1))              # (no second row: the stride says nothing)
    one = torch.ones(1, device=DEV)
    assert all(torch.equal(x, y) for x, y in zip(b.pacer_head_nll_grad(odd, w, t, one), b.pacer_head_nll_grad(h, w, t, one)))
