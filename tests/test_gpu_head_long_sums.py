"""Sums of the fused head's gradients over many rows, tokens and columns whose terms have one sign: the tensor cores truncate when they add, by at most 2^-23
of the sum at each 16 terms, and would make such sums too small; an accumulator takes 16 384 terms of a gradient and 8192 columns of a logit.

Tolerances of the mean relative error over N results: the truncations' bound, and 6 standard deviations of N independent roundings to bf16 (at
most 2^-8 each)."""
import math

import pytest
import torch

from tests.test_gpu_head_grads import BF16, DEV, F32

pytestmark = pytest.mark.gpu
TRUNCATED = 16384 / 16 * 2 * F32


def gen():
    return torch.Generator(device=DEV).manual_seed(1)


@pytest.mark.parametrize("rows", [20000, 300000])
def test_dhead_over_many_rows(rows):
    from paper_2602_01274_b200 import binding as b
    g = gen()
    h = (1 + 0.3 * torch.randn(rows, 64, generator=g, device=DEV)).to(torch.bfloat16)
    w = (0.1 * torch.randn(512, 64, generator=g, device=DEV)).to(torch.bfloat16)
    _, _, dw = b.pacer_head_nll_grad(h, w, torch.zeros(rows, dtype=torch.int32, device=DEV), torch.ones(rows, device=DEV))
    want = torch.zeros(512, 64, dtype=torch.float64, device=DEV)
    for x in h.split(65536):
        want += torch.softmax(x.double() @ w.double().T, 1).T @ x.double()
    off = (dw.double() / want)[1:] - 1                                      # (the tokens' own row aside)
    assert abs(float(off.mean())) < TRUNCATED + 6 * BF16 / math.sqrt(off.numel()) and off.abs().max() < 1.01 * BF16 + 2 * TRUNCATED


@pytest.mark.parametrize("rows,vocab", [(2, 151936), (300, 151936), (20000, 60000)])
def test_dhidden_over_many_tokens(rows, vocab):
    """(20 000 rows of 60 000 tokens: in pieces of the vocabulary.)"""
    from paper_2602_01274_b200 import binding as b
    g = gen()
    h = (0.1 * torch.randn(rows, 64, generator=g, device=DEV)).to(torch.bfloat16)
    w = (1 + 0.1 * torch.randn(vocab, 64, generator=g, device=DEV)).to(torch.bfloat16)
    lse = b.pacer_head_logprobs(h, w, torch.zeros(rows, dtype=torch.int32, device=DEV))[2]
    dh, _ = b.pacer_head_logprobs_backward(h, w, None, None, lse, None, None, None, torch.ones(rows, device=DEV), grads=(True, False))
    off = torch.cat([dh[i:i + 100].double() / (torch.softmax(h[i:i + 100].double() @ w.double().T, 1) @ w.double()) - 1 for i in range(0, min(rows, 2000), 100)])
    assert abs(float(off.mean())) < TRUNCATED + 6 * BF16 / math.sqrt(off.numel()) and off.abs().max() < 1.01 * BF16 + 2 * TRUNCATED


@pytest.mark.parametrize("rows", [1, 140])
@pytest.mark.parametrize("d", [8256, 65536])
def test_logits_over_many_columns(rows, d):
    """p = exp(z - lse) with z of some 20 out of products above 0: too small a z would make every p too small."""
    from paper_2602_01274_b200 import binding as b
    g = gen()
    h = (1 + 0.2 * torch.rand(rows, d, generator=g, device=DEV)).to(torch.bfloat16)
    w = ((20 + torch.randn(300, 1, generator=g, device=DEV)) / d * (0.8 + 0.4 * torch.rand(300, d, generator=g, device=DEV))).to(torch.bfloat16)
    lse = b.pacer_head_logprobs(h, w, torch.zeros(rows, dtype=torch.int32, device=DEV))[2]
    _, dw = b.pacer_head_logprobs_backward(h, w, None, None, lse, None, None, None, torch.ones(rows, device=DEV), grads=(False, True))
    z = h.double() @ w.double().T
    p = torch.softmax(z, 1)
    off = dw.double() / (p.T @ h.double()) - 1
    # (p is off by the error of z and of lse)
    near = float(z.max()) * (8192 / 16 * 2 * F32 + 8 * F32)
    assert float(z.min()) > 10 and abs(float(off.mean())) < near + 6 * BF16 / math.sqrt(300 * min(rows, 16))
    assert off.abs().max() < 1.01 * (near + BF16 * (1 if rows <= 128 else 2))
