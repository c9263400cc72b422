"""A planted bias that takes a token out of a row (-infinity, f32's lowest value): the row's other tokens go as they would with a bias of -1e6, whose
exponential is 0 as well (equal bits), and that one as the 64-bit form does."""
import math

import pytest
import torch

from tests import logit_refs as ref
from tests.test_gpu_head_grads import BF16, DEV, F32, check, logits, slack, weights
from tests.test_gpu_head_logprobs import make

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min


def calls(h, w, tok, ids, bias, gs):
    from paper_2602_01274_b200 import binding as b
    logp, ent, lse = b.pacer_head_logprobs(h, w, tok, ids, bias)
    out = dict(logp=logp, entropy=ent, lse=lse)
    out["loss"], out["nll_dh"], out["nll_dw"] = b.pacer_head_nll_grad(h, w, tok, gs[0], ids, bias)
    for name, (gl, gh, gl2) in dict(one=(gs[0], None, None), all=gs).items():
        out[name + "_dh"], out[name + "_dw"] = b.pacer_head_logprobs_backward(h, w, tok, logp, lse, ent, gl, gh, gl2, ids, bias)
    return out


@pytest.mark.parametrize("rows,vocab,d", [(1, 300, 64), (40, 4099, 128), (200, 1003, 72), (300, 33, 64)])
def test_a_token_taken_out(rows, vocab, d):
    h, w, tok, ids = make(rows, vocab, d)
    ids = ids.clamp(0, vocab - 1)                                           # (every third row's token is its biased one)
    gs = weights(rows)
    want = calls(h, w, tok, ids, -1e6, gs)
    out = (tok == ids)
    for bias in (-math.inf, LOWEST, -3e38, -1e30):
        got = calls(h, w, tok, ids, bias, gs)
        for name, x in want.items():
            if name in ("logp", "loss"):
                assert torch.equal(got[name][~out], x[~out]), (bias, name)
            else:
                assert torch.equal(got[name], x), (bias, name)
        assert (got["logp"][out] <= max(bias, LOWEST) * 0.999).all() and torch.equal(got["loss"][out], -got["logp"][out])
    assert torch.isfinite(want["entropy"]).all()
    # the common result against 64 bits
    z = logits(h, w, ids, -1e6)
    lp, lse = ref.softmax_parts(z)
    sz, _ = slack(h, w, z.clamp(min=-100), 0)
    named = (tok >= 0) & (tok < vocab)
    at, g = torch.where(named, tok, 0).long()[:, None], torch.where(named, gs[0], 0.0).double()[:, None]
    dz, size = (lp.exp() * g).scatter_add(1, at, -g), (lp.exp() * g.abs()).scatter_add(1, at, g.abs())
    check(want["nll_dh"], dz, size, w.double(), True, sz + BF16 / 8, (vocab / 16 + 1) * 2 * F32, "dhidden")
    check(want["nll_dw"], dz, size, h.double(), False, sz + BF16 / 8, (rows / 16 + 1) * 2 * F32, "dhead")


def test_in_pieces_of_the_vocabulary():
    from paper_2602_01274_b200 import binding as b
    h, w, tok, ids = make(75000, 16001, 72)
    weight = weights(75000)[0]
    want, got = (b.pacer_head_nll_grad(h, w, tok, weight, ids, bias) for bias in (-1e6, -math.inf))
    out = (tok == ids) & (tok >= 0) & (tok < 16001)
    assert torch.equal(got[0][~out], want[0][~out]) and (got[0][out] == math.inf).all()
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
