"""The LM head fused with the scoring of given tokens, against a plain 64-bit product and softmax on the same bf16 inputs.

Tolerance.  The tensor cores truncate when they add: each of d / 16 additions to an accumulator loses at most one step (2^-23) of
the partial sum, which stays below sum |h w| <= |h| |w| (norms); the products of 16 inside an addition are held at least as well.
So |dz| <= (d / 16) 2^-23 |h| |w|, far above what is seen (the losses of a random walk).  The rest as for rows of logits: 240 half
steps of fp32 for the sums, four of the values' own size."""
import math

import pytest
import torch

from tests import logit_refs as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(rows, vocab, d, pad=0, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + rows + vocab)
    h = torch.randn(rows, d + pad, generator=g, device=DEV).to(torch.bfloat16)[:, :d]
    w = (torch.randn(vocab, d + pad, generator=g, device=DEV) * 1.5 / math.sqrt(d)).to(torch.bfloat16)[:, :d]
    tok = torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    bias_ids = torch.randint(-1, vocab + 1, (rows,), generator=g, device=DEV, dtype=torch.int32)
    tok[::3] = bias_ids[::3].clamp(0, vocab - 1)
    tok[1::4] = -1
    if rows > 2:
        tok[2] = vocab
    return h, w, tok, bias_ids


@pytest.mark.parametrize("rows,vocab,d,pad", [
    (1, 1, 8, 0), (1, 2, 64, 0), (2, 31, 72, 0), (7, 33, 128, 8), (8, 257, 64, 0), (9, 1000, 200, 0), (1, 4096, 256, 0),
    (1, 32000, 768, 0), (25, 32256, 2048, 0), (33, 4099, 768, 0), (127, 5003, 256, 0), (128, 32000, 128, 0), (129, 32003, 136, 64),
    (136, 151936, 128, 0), (300, 32256, 512, 0), (1000, 7777, 1024, 0), (5, 151937, 64, 0), (2048, 4096, 2048, 0),
    # by pairs of blocks (as are 129, 136, 1000 and 2048 rows)
    (200, 33, 72, 0), (256, 1, 8, 0), (1153, 32003, 576, 0), (500, 40000, 1536, 8),
])
@pytest.mark.parametrize("biased", [False, True])
def test_head_logprobs(rows, vocab, d, pad, biased):
    from paper_2602_01274_b200 import binding as b
    h, w, tok, bias_ids = make(rows, vocab, d, pad)
    bias_ids = bias_ids if biased else None
    got = b.pacer_head_logprobs(h, w, tok, bias_ids, 8.0)
    z = h.double() @ w.double().T
    if biased:
        ok = (bias_ids >= 0) & (bias_ids < vocab)
        z.scatter_add_(1, torch.where(ok, bias_ids, 0).long()[:, None], torch.where(ok, 8.0, 0.0).double()[:, None])
    want = ref.logprobs(z, tok)
    dz = (d / 16 + 1) * 2 * ref.F32 * h.double().norm(dim=1) * w.double().norm(dim=1).max()
    bound = 2 * dz + 240 * ref.F32 + 4 * ref.F32 * (z.abs().amax(1) + want[2].abs())
    for x, y, f, name in zip(got, want, (1, 40, 1), ("logp", "entropy", "lse")):
        over = ((x.double() - y).abs() - f * bound).max()
        assert torch.isfinite(x).all() and over <= 0, (name, float(over))
    assert (got[0][(tok < 0) | (tok >= vocab)] == 0).all()
    again = b.pacer_head_logprobs(h, w, tok, bias_ids, 8.0)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_scratch_between_calls_graphs_and_streams():
    """Scratch full of garbage, calls on two streams, and a captured call on new inputs."""
    from paper_2602_01274_b200 import binding as b
    from tests.common import filled_workspaces
    sets = [make(40, 32003, 256), make(300, 5000, 512)]
    want = [b.pacer_head_logprobs(h, w, t, i, 8.0) for h, w, t, i in sets]
    with filled_workspaces(0xFF) as sizes:
        got = [b.pacer_head_logprobs(h, w, t, i, 8.0) for h, w, t, i in sets]
    assert len(sizes) == 2 and all(torch.equal(x, y) for g, v in zip(got, want) for x, y in zip(g, v))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            for _ in range(4):
                got[k] = b.pacer_head_logprobs(*sets[k], 8.0)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g, v in zip(got, want) for x, y in zip(g, v))
    h, w, t, i = sets[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.pacer_head_logprobs(h, w, t, i, 8.0)
    h.copy_(h.flip(0))
    t.copy_(t.flip(0))
    i.copy_(i.flip(0))
    graph.replay()
    assert all(torch.equal(x, y.flip(0)) for x, y in zip(out, want[0]))


def test_head_agrees_with_the_logits_operator():
    """The same rows through written logits: pacer_linear's sums, then pacer_logprobs."""
    from paper_2602_01274_b200 import binding as b
    h, w, tok, _ = make(17, 32000, 768)
    fused = b.pacer_head_logprobs(h, w, tok)
    two = b.pacer_logprobs(b.pacer_linear(h, w), tok)
    for x, y in zip(fused, two):
        assert (x - y).abs().max() < 1e-4


def test_one_row_whatever_its_stride():
    from paper_2602_01274_b200 import binding as b
    h, w, t, _ = make(1, 300, 64)
    odd = torch.as_strided(h, (1, 64), (67, 1))              # (no second row: the stride says nothing)
    assert all(torch.equal(x, y) for x, y in zip(b.pacer_head_logprobs(odd, w, t), b.pacer_head_logprobs(h, w, t)))


def test_no_rows():
    from paper_2602_01274_b200 import binding as b
    h, w, _, _ = make(1, 100, 64)
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    assert [tuple(x.shape) for x in b.pacer_head_logprobs(h[:0], w, e)] == [(0,)] * 3


@pytest.mark.parametrize("rows,vocab,d", [(1025, 4099, 72), (1100, 32003, 136), (1152, 257, 1024), (1300, 33, 8), (1664, 5003, 256)])
@pytest.mark.parametrize("biased", [False, True])
def test_pairs_of_blocks_over_an_odd_number_of_row_tiles(rows, vocab, d, biased):
    """From nine tiles of 128 rows on pairs of blocks work on odd numbers of them too: the second block's last tile has no rows."""
    assert -(-rows // 128) % 2 == 1
    test_head_logprobs(rows, vocab, d, 0, biased)
