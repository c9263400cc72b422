"""The differentiable forms of the fused head, and a training step as it would be run: cross entropy and its gradients, their global norm, AdamW."""
import numpy as np
import pytest
import torch

from tests import logit_refs as ref
from tests.test_gpu_head_grads import BF16, F32, check, logits, slack, weights
from tests.test_gpu_head_logprobs import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def exact_dz(h, w, tok, bias_ids, weight):
    z = logits(h, w, bias_ids)
    lp, _ = ref.softmax_parts(z)
    named = (tok >= 0) & (tok < w.shape[0])
    at, g = torch.where(named, tok, 0).long()[:, None], torch.where(named, weight, 0.0).double()[:, None]
    loss = torch.where(named, -lp.gather(1, at)[:, 0], 0.0)
    return z, loss, (lp.exp() * g).scatter_add(1, at, -g), (lp.exp() * g.abs()).scatter_add(1, at, g.abs())


@pytest.mark.parametrize("trained", [(True, True), (True, False), (False, True), (False, False)])
def test_head_nll_is_differentiable(trained):
    from paper_2602_01274_b200 import losses
    h, w, tok, bias_ids = make(60, 1003, 128)
    weight = weights(60)[0] / 60
    h3 = h.clone().view(4, 15, 128).requires_grad_(trained[0])
    head = w.clone().requires_grad_(trained[1])
    wt = weight.clone().view(4, 15).requires_grad_(True)
    total = losses.head_nll(h3, head, tok.view(4, 15), wt, bias_ids.view(4, 15), 8.0)
    z, loss, dz, size = exact_dz(h, w, tok, bias_ids, weight)
    sz, _ = slack(h, w, z, 0)
    assert abs(float(total.detach()) - float((loss * weight.double()).sum())) <= 1e-5 * float((loss * weight.double()).abs().sum())
    (total * 0.5).backward()
    if trained[0]:
        check(h3.grad.view(60, 128), 0.5 * dz, 0.5 * size, w.double(), True, sz, (1003 / 16 + 1) * 2 * F32, "hidden")
    if trained[1]:
        check(head.grad, 0.5 * dz, 0.5 * size, h.double(), False, sz, (60 / 16 + 1) * 2 * F32, "head")
    assert (h3.grad is None) == (not trained[0]) and (head.grad is None) == (not trained[1])
    assert torch.allclose(wt.grad.view(-1).double(), 0.5 * loss, rtol=1e-5, atol=1e-5)
    # without gradients: the same sum, and none are computed
    from paper_2602_01274_b200 import binding
    asked, call = [], binding.pacer_head_nll_grad
    binding.pacer_head_nll_grad = lambda *a, **kw: asked.append(kw["grads"]) or call(*a, **kw)
    try:
        with torch.no_grad():
            again = losses.head_nll(h3, head, tok.view(4, 15), wt, bias_ids.view(4, 15), 8.0)
    finally:
        binding.pacer_head_nll_grad = call
    assert asked == [(False, False)] and torch.allclose(again, total.detach(), rtol=1e-5)


def test_head_logprobs_is_differentiable():
    from paper_2602_01274_b200 import losses
    h, w, tok, _ = make(48, 2003, 192)
    hidden, head = h.clone().view(6, 8, 192).requires_grad_(True), w.clone().requires_grad_(True)
    gs = weights(48)
    logp, ent, lse = losses.head_logprobs(hidden, head, tok.view(6, 8))
    sum((x.view(-1) * g).sum() for x, g in zip((logp, ent, lse), gs)).backward()
    z = logits(h, w, None)
    dz, size = ref.logprobs_grad(z, tok, lse.detach().view(-1), ent.detach().view(-1), *gs)
    sz, _ = slack(h, w, z, 0)
    check(hidden.grad.view(48, 192), dz, size, w.double(), True, sz, (2003 / 16 + 1) * 2 * F32, "hidden")
    check(head.grad, dz, size, h.double(), False, sz, (48 / 16 + 1) * 2 * F32, "head")
    # one output, a broadcast gradient; nothing that needs one
    hidden.grad = None
    losses.head_logprobs(hidden, w, tok.view(6, 8))[1].mean().backward()
    dz, size = ref.logprobs_grad(z, None, lse.detach().view(-1), ent.detach().view(-1), None, torch.full((48,), 1 / 48, device=DEV), None)
    check(hidden.grad.view(48, 192), dz, size, w.double(), True, sz, (2003 / 16 + 1) * 2 * F32, "hidden of the entropy")
    assert not losses.head_logprobs(h, w, tok)[0].requires_grad


@pytest.mark.parametrize("rows,bits", [(40, 32), (200, 32), (200, 8)])
def test_a_step_of_training(rows, bits):
    """Cross entropy, its gradients, their norm and AdamW together against the same in 64 bits; then captured and replayed."""
    from paper_2602_01274_b200 import binding as b
    h, w, tok, bias_ids = make(rows, 3001, 256)
    weight = torch.full((rows,), 1.0 / rows, device=DEV)
    dtype = torch.float32 if bits == 32 else torch.uint8
    m, v = torch.zeros(w.numel(), dtype=dtype, device=DEV), torch.zeros(w.numel(), dtype=dtype, device=DEV)
    scales = None if bits == 32 else [torch.zeros(-(-w.numel() // 256), 2, device=DEV)]
    head, master = w.clone(), w.float()
    tensors = b.AdamwTensors([master], [m], [v], scales, [head])
    step, lr, limit = torch.zeros((), dtype=torch.int32, device=DEV), 1e-3, 0.05

    def train():
        _, _, dhead = b.pacer_head_nll_grad(h, head, tok, weight, bias_ids, 8.0, grads=(False, True))
        norm = b.pacer_grad_norm([dhead])
        step.add_(1)
        b.pacer_adamw(tensors, [dhead], step, lr, weight_decay=0.1, norm=norm, max_norm=limit, seed=5)
        return dhead, norm

    dhead, norm = train()
    z, _, dz, size = exact_dz(h, w, tok, bias_ids, weight)
    sz, _ = slack(h, w, z, 0)
    check(dhead, dz, size, h.double(), False, sz, (rows / 16 + 1) * 2 * F32, "dhead")
    g = dhead.double().flatten()
    total = float(g.norm())
    assert abs(float(norm) - total) <= 2 * F32 * total and total > limit
    # the first step from states of 0 moves by lr g / (|g| + eps), whatever the states' bits
    g = g * limit / (total + 1e-6)
    want = w.double().flatten() * (1 - lr * 0.1) - lr * (0.1 * g / 0.1) / ((0.001 * g * g / 0.001).sqrt() + 1e-8)
    assert ((master.double().flatten() - want).abs() <= 40 * F32 * lr + 4 * F32 * w.double().flatten().abs()).all()
    assert torch.equal(head, master.to(torch.bfloat16))
    # the same from the start, captured: two replays are two steps, bit for bit
    train()
    after = [x.clone() for x in (head, master, m, v)]
    head.copy_(w)
    master.copy_(w)
    for x in (m, v, step, *(scales or [])):
        x.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train()
    graph.replay()
    graph.replay()
    assert int(step) == 2 and all(torch.equal(x, y) for x, y in zip(after, (head, master, m, v)))


@pytest.mark.parametrize("objective,optimizer", [("nll", "f32"), ("nll", "8bit"), ("kl", "f32"), ("kl", "8bit")])
def test_draft_training_runs(objective, optimizer):
    from paper_2602_01274_b200 import synth, train_draft
    cfg = synth.CONFIGS["tiny"]
    pair = synth.make_pair(cfg, seed=0, device=DEV, which=("target", "draft"))
    tensors, report = train_draft.train(cfg, pair, DEV, n_prompts=8, n_prompt_tokens=16, n_resp=8, epochs=1, top=16, batch_prompts=4, log=lambda *_: None,
                                        objective=objective, optimizer=optimizer)
    assert tensors["head"].shape == pair["draft"]["head"].shape and tensors["head"].dtype == torch.bfloat16
    assert not torch.equal(tensors["head"], pair["draft"]["head"])
    assert all(np.isfinite(report[k]) for k in ("held_out_nll_before", "held_out_nll_after", "held_out_kl"))
    assert report["objective"] == objective and report["optimizer"] == optimizer
    # the gradient that the objective takes
    prompts = synth.make_prompts(cfg.target.vocab, 4, 16, seed=9).to(DEV).long()
    d = train_draft.make_examples(cfg, pair, prompts, 12, 16)
    head = pair["draft"]["head"].clone().requires_grad_(True)
    train_draft.draft_nll(head, d, cfg.succ_bias).backward()
    z, _, dz, size = exact_dz(d["hidden"], pair["draft"]["head"], d["next"], d["planted"], torch.full((48,), 1 / 48, device=DEV))
    sz, _ = slack(d["hidden"], pair["draft"]["head"], z, 0)
    check(head.grad, dz, size, d["hidden"].double(), False, sz, (48 / 16 + 1) * 2 * F32, "head")


def test_preverify_training_runs():
    from paper_2602_01274_b200 import synth, train_preverify
    cfg = synth.CONFIGS["tiny"]
    pair = synth.make_pair(cfg, seed=0, device=DEV, which=("target", "draft"))
    for optimizer in ("f32", "8bit"):
        tensors, report = train_preverify.train(cfg, pair, DEV, n_prompts=8, n_prompt_tokens=16, n_resp=16, epochs=2, batch_prompts=4,
                                                log=lambda *_: None, optimizer=optimizer)
        assert all(torch.isfinite(t).all() for t in tensors.values()) and np.isfinite(report["held_out_loss"])
    for bad in (dict(optimizer="4bit"),):
        with pytest.raises(ValueError):
            train_preverify.train(cfg, pair, DEV, **bad)


def test_draft_training_refusals():
    from paper_2602_01274_b200 import synth, train_draft
    for bad in (dict(objective="ce"), dict(optimizer="sgd"), dict(objective="nll")):
        with pytest.raises(ValueError):
            train_draft.train(synth.CONFIGS["tiny"], {}, **bad)
