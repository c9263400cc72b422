"""The differentiable forms of the operators on rows of logits, the verify forward's log probabilities, and the operators run
together as the draft's training uses them."""
import numpy as np
import pytest
import torch

from tests import logit_refs as ref
from tests.test_gpu_logits import DEV, EPS, close, gen, make_logits, make_teacher, make_tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprobs_is_differentiable(dtype):
    from paper_2602_01274_b200 import losses
    z = make_logits(24, 1001, dtype, seed=40).view(4, 6, 1001).requires_grad_(True)
    tokens = make_tokens(24, 1001).view(4, 6)
    w = [torch.randn(4, 6, generator=gen(41 + i), device=DEV) for i in range(3)]
    logp, ent, lse, ids, tlp = losses.token_logprobs(z, tokens, 4)
    assert ids.shape == tlp.shape == (4, 6, 4) and not ids.requires_grad and not tlp.requires_grad
    (logp * w[0] + ent * w[1] + lse * w[2]).sum().backward()
    flat = z.detach().view(24, 1001)
    want, size = ref.logprobs_grad(flat, tokens.view(-1), lse.detach().view(-1), ent.detach().view(-1), *(x.view(-1) for x in w))
    half, least = ref.rounding(z.dtype)
    assert z.grad.dtype == z.dtype
    close(z.grad.view(24, 1001), want, half * 1.01 * want.abs() + 180 * ref.F32 * size + least, "grad")
    # one output alone, a broadcast incoming gradient, a scalar loss
    z.grad = None
    losses.token_logprobs(z, tokens)[1].mean().backward()
    want, size = ref.logprobs_grad(flat, None, lse.detach().view(-1), ent.detach().view(-1), None, torch.full((24,), 1 / 24, device=DEV), None)
    close(z.grad.view(24, 1001), want, half * 1.01 * want.abs() + 180 * ref.F32 * size + least, "entropy's grad")


def test_log_probabilities_may_be_changed_in_place():
    from paper_2602_01274_b200 import losses
    z = make_logits(12, 333, "f32", seed=45).requires_grad_(True)
    tokens = make_tokens(12, 333)
    mask = (torch.arange(12, device=DEV) % 2).float()
    logp, ent, _, _, tlp = losses.token_logprobs(z, tokens, 3)
    logp.mul_(mask)
    tlp.zero_()
    (logp.sum() + ent.sum()).backward()
    got, z.grad = z.grad, None
    _, ent, _, _, _ = losses.token_logprobs(z, tokens)
    ent += 1.0                                          # (the backward pass needs it as it was: torch says so)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        ent.sum().backward()
    logp, ent, _, _, _ = losses.token_logprobs(z, tokens)
    ((logp * mask).sum() + ent.sum()).backward()
    assert torch.equal(got, z.grad)
    # a second stream, and a leaf that a view of it went through
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    leaf = z.detach().clone().requires_grad_(True)
    with torch.cuda.stream(s):
        logp, ent, _, _, _ = losses.token_logprobs(leaf.view(3, 4, 333), tokens.view(3, 4))
        ((logp.view(-1) * mask).sum() + ent.sum()).backward()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(leaf.grad, z.grad)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_loss_is_differentiable(tail):
    from paper_2602_01274_b200 import losses
    z = make_logits(24, 1001, "bf16", seed=42).view(4, 6, 1001).requires_grad_(True)
    ids, t, tl = make_teacher(24, 1001, 9, tail, 2.0)
    w = torch.randn(24, generator=gen(43), device=DEV)
    loss = losses.distill_loss(z, ids.view(4, 6, 9), t.view(4, 6, 9).requires_grad_(True), 2.0, None if tl is None else tl.view(4, 6))
    want = ref.distill(z.detach().view(24, 1001), ids, t.detach(), 2.0, tl, w)
    close(loss.detach().view(-1), want[0], 60 * EPS, "loss")
    (loss.view(-1) * w).sum().backward()
    half, least = ref.rounding(z.dtype)
    close(z.grad.view(24, 1001), want[3], half * 1.01 * want[3].abs() + 8 * EPS * want[4] + least, "grad")
    assert t.grad is None


def test_two_backward_passes_and_a_captured_one():
    """retain_graph: the second pass gives the same; functions called directly are captured while an autograd graph lives."""
    from paper_2602_01274_b200 import binding as b, losses
    z = make_logits(40, 4099, "bf16", seed=44).requires_grad_(True)
    ids, t, tl = make_teacher(40, 4099, 20, True, 1.0)
    loss = losses.distill_loss(z, ids, t, 1.0, tl).sum()
    loss.backward(retain_graph=True)
    first, z.grad = z.grad, None
    graph = torch.cuda.CUDAGraph()
    one = torch.ones(40, device=DEV)
    with torch.cuda.graph(graph):
        _, d = b.pacer_distill_grad(z.detach(), ids, t, one, 1.0, tl)
    graph.replay()
    loss.backward()
    assert torch.equal(z.grad, first)
    half, least = ref.rounding(torch.bfloat16)
    close(d, first, 2 * half * first.double().abs() + 2 * least, "captured")      # (two roundings of values EPS apart)


@pytest.mark.parametrize("batch", [1, 3])
def test_verify_logprobs(batch):
    from paper_2602_01274_b200 import binding as b, synth
    cfg = synth.CONFIGS["tiny"]
    V, per = cfg.target.vocab, cfg.gamma_cap + 1
    pair = synth.make_pair(cfg, seed=0, device=DEV)
    ctx = b.Context(b.make_cfg(cfg.target, cfg.draft, batch, 64 + 32 + cfg.gamma_cap + 2, cfg.gamma_cap, cfg.block_b, cfg.rho, 0, cfg.succ_bias))
    b.load_pair(ctx, pair)
    with pytest.raises(b.PacerError, match="out of order"):
        ctx.pacer_verify_logprobs()
    ctx.pacer_prefill(synth.make_prompts(V, batch, 64, seed=3).numpy(), 32, cfg.gamma_cap, 0.5)
    for step in range(2):
        with pytest.raises(b.PacerError, match="not directly after pacer_verify"):
            ctx.pacer_verify_logprobs()
        for _ in range(cfg.gamma_cap // cfg.block_b):
            for _ in range(cfg.block_b):
                ctx.pacer_draft_step()
            ctx.pacer_preverify()
        ctx.pacer_verify()
        with pytest.raises(b.PacerError, match="top out of range"):
            ctx.pacer_verify_logprobs(top=129)
        logp, ent, ids, tlp = ctx.pacer_verify_logprobs(top=7)
        state = ctx.pacer_read_state(batch)
        z = torch.from_numpy(ctx.pacer_read_buffer(b.BUF_VERIFY_LOGITS, np.float32, batch * per * V).copy()).view(batch, per, V)
        drafts = ctx.pacer_read_buffer(b.BUF_DRAFTS, np.int32, batch * cfg.gamma_cap).reshape(batch, -1)
        for q in range(batch):
            n = state[q]["gamma"] + 1
            tokens = torch.tensor([*drafts[q, :n - 1], -1], dtype=torch.int32)
            want = b.pacer_logprobs(z[q, :n].to(DEV), tokens.to(DEV), 7)
            assert torch.allclose(logp[q, :n], want[0], atol=2 * EPS) and torch.allclose(ent[q, :n], want[1], atol=80 * EPS)
            assert torch.equal(ids[q, :n], want[3]) and torch.allclose(tlp[q, :n], want[4], atol=2 * EPS)
            close(want[0].cpu(), ref.logprobs(z[q, :n], tokens)[0], EPS + 4 * ref.F32 * 60, "logp")
            assert torch.isnan(logp[q, n:]).all() and torch.isnan(tlp[q, n:]).all() and (ids[q, n:] == -1).all()
        ctx.pacer_accept_rollback()
    ctx.pacer_generate(synth.make_prompts(V, batch, 64, seed=3).numpy(), 8, cfg.gamma_cap, 0.5)
    with pytest.raises(b.PacerError, match="not directly after pacer_verify"):
        ctx.pacer_verify_logprobs()
    ctx.close()


def test_draft_training_runs_and_its_gradient_is_right():
    from paper_2602_01274_b200 import binding as b, synth, train_draft
    cfg = synth.CONFIGS["tiny"]
    pair = synth.make_pair(cfg, seed=0, device=DEV)
    prompts = synth.make_prompts(cfg.target.vocab, 4, 16, seed=9).to(DEV).long()
    d = train_draft.make_examples(cfg, pair, prompts, 12, 16)
    assert d["hidden"].shape == (48, cfg.draft.d_model) and d["ids"].shape == d["teacher"].shape == (48, 16)
    assert torch.equal(d["ids"][:, 0], d["next"])                 # greedy: the target's token is its best
    # the gradient of the head against the formula in 64 bits on the same bf16 operands
    head = pair["draft"]["head"].float().requires_grad_(True)
    train_draft.draft_loss(head, d, cfg.succ_bias).backward()
    h, w = d["hidden"].double(), pair["draft"]["head"].double()
    z = h @ w.T
    z.scatter_add_(1, d["planted"].long()[:, None], torch.full((48, 1), float(cfg.succ_bias), dtype=torch.float64, device=DEV))
    dz = ref.distill(z, d["ids"], d["teacher"], 1.0, torch.zeros(48, device=DEV), torch.full((48,), 1 / 48, device=DEV))[3]
    want = dz.T @ h
    # torch's product gives bf16 logits (off by 2^-8 of at most 8 each, relative to p), takes bf16 gradients in (2^-8 each), and
    # rounds its own result to bf16
    slack = (8 * 2.0 ** -8 + 3 * 2.0 ** -8) * (dz.abs().T @ h.abs())
    assert ((head.grad.double() - want).abs() <= slack + 2.0 ** -8 * want.abs() + 1e-7).all()
    tensors, report = train_draft.train(cfg, pair, DEV, n_prompts=8, n_prompt_tokens=16, n_resp=8, epochs=1, top=16, batch_prompts=4, log=lambda *_: None)
    assert tensors["head"].shape == pair["draft"]["head"].shape and tensors["head"].dtype == torch.bfloat16
    assert all(np.isfinite(report[k]) for k in ("held_out_nll_before", "held_out_nll_after", "held_out_kl"))
    # a pair with that head decodes what the target alone decodes
    ctx = b.Context(b.make_cfg(cfg.target, cfg.draft, 1, 128, cfg.gamma_cap, cfg.block_b, cfg.rho, 0, cfg.succ_bias))
    ctx.pacer_load_weights(b.PACER_TARGET, pair["target"], pair["succ_T"])
    ctx.pacer_load_weights(b.PACER_DRAFT, {**pair["draft"], **tensors}, pair["succ_D"])
    ctx.pacer_load_weights(b.PACER_PREVERIFY, pair["preverify"])
    prompt = synth.make_prompts(cfg.target.vocab, 1, 32, seed=4).numpy()
    assert (ctx.pacer_generate(prompt, 24, cfg.gamma_cap, -1.0)[0] == ctx.pacer_generate_ar(prompt, 24)[0]).all()
    ctx.close()


def test_autograd_sees_what_calls_write():
    """Outputs of the caller count as changed in place: a backward pass that saved them raises, as with torch's own functions."""
    from paper_2602_01274_b200 import binding as b, losses
    tokens = make_tokens(12, 333)
    ids, t, _ = make_teacher(12, 333, 5, False, 1.0)
    w = torch.ones(12, device=DEV)
    leaf = make_logits(12, 333, "f32", seed=46).requires_grad_(True)

    def saved():
        z = leaf * 1.0
        logp, _, lse, _, _ = losses.token_logprobs(z, tokens)
        return z.detach(), logp, lse.detach()

    z, logp, lse = saved()
    ent = b.pacer_logprobs(z, tokens)[1]
    saved_loss, saved_lse, _ = b.pacer_distill(z, ids, t)
    writes = [lambda z: b.pacer_distill_grad(z, ids, t, w, out=z), lambda z: b.pacer_logprobs_backward(z, tokens, lse, ent, w, out=z),
              lambda z: b.pacer_distill_backward(z, ids, t, saved_lse, None, w, out=z),
              lambda z: b.pacer_distill_grad(z.clone(), ids, t, w, out=z), lambda z: b.pacer_logprobs_backward(z[:5], tokens[:5], lse[:5], ent[:5], w[:5], out=z[:5])]
    for write in writes:
        z, logp, _ = saved()
        write(z)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            logp.sum().backward()
    out = [torch.empty(12, device=DEV) for _ in range(3)] + [torch.empty(12, 2, dtype=torch.int32, device=DEV), torch.empty(12, 2, device=DEV)]
    x = torch.ones(12, device=DEV, requires_grad=True)
    y = x * out[0]                                      # (saves out[0])
    b.pacer_logprobs(z, tokens, 2, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    # outputs that the call makes, and calls that write nothing of the caller's, disturb nothing
    z, logp, lse = saved()
    b.pacer_distill_grad(z, ids, t, w)
    b.pacer_logprobs_backward(z, tokens, lse, ent, w)
    logp.sum().backward()
    assert torch.isfinite(leaf.grad).all()
    with torch.inference_mode():
        z = make_logits(12, 333, "f32", seed=46)
        b.pacer_distill_grad(z, ids, t, w, out=z)
