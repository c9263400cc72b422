"""Distils the draft model's LM head from the target on the target's own responses.

A draft is accepted where the two models agree, so a speculative-decoding pair profits from a draft that was trained
towards its target.  The target generates greedy responses to seeded random prompts; at every position its best
logits (``pacer_logprobs``) are the teacher's list, with all other tokens as one further class; the draft's LM head is
trained on KL(target || draft) over the frozen draft's hidden states (``losses.distill_loss``, AdamW).  The held-out
negative log-likelihood of the target's tokens under the draft is taken before and after, straight from hidden states
and head (``pacer_head_logprobs``).  With ``--objective nll`` the head is trained on that likelihood itself, loss and
gradient straight from hidden states and head (``losses.head_nll``), as a bf16 tensor with an f32 master; ``--optimizer f32`` or ``8bit``
takes the library's AdamW (``optim.AdamW``), which the objective needs.

Like ``train_preverify`` this is a small PyTorch job outside the decoding path; it needs a GPU (the operators have no
CPU form).  It produces a bf16 ``head`` for ``pacer_load_weights(PACER_DRAFT, ...)``.

    python -m paper_2602_01274_b200.train_draft --config tiny --out draft_head.pt
"""
from __future__ import annotations

import argparse
import time

import torch

from . import binding, losses, optim, synth
from .train_preverify import Decoder


@torch.no_grad()
def make_examples(cfg: synth.PairConfig, pair, prompts, n_resp, top, dtype=torch.bfloat16):
    """For prompts [B][n_p]: the target's greedy response (n_resp tokens) and, for the rows that lead to a response token, flat
    over sequences: hidden bf16 [N][d] (the draft's), ids int32 [N][top] and teacher f32 [N][top] (the target's best tokens and
    their log probabilities), next int32 [N] (the target's token), planted int32 [N] (the draft's biased token)."""
    B, n_p = prompts.shape
    T = n_p + n_resp
    target = Decoder(cfg.target, pair["target"], pair["succ_T"], cfg.succ_bias, T + 1, dtype)
    target.reset(B, T)
    _, logits = target.forward(prompts)
    seq, lists = [prompts], []
    for _ in range(n_resp):
        rows = logits[:, -1].contiguous()
        token = rows.argmax(-1, keepdim=True)
        _, _, _, ids, top_logp = binding.pacer_logprobs(rows, token[:, 0].to(torch.int32), top)
        lists.append((ids, top_logp))
        seq.append(token)
        if len(seq) <= n_resp:
            _, logits = target.forward(token)
    full = torch.cat(seq, dim=1)                                    # [B][T]
    draft = Decoder(cfg.draft, pair["draft"], None, 0.0, T + 1, dtype)
    draft.reset(B, T)
    hidden, _ = draft.forward(full[:, :-1])
    flat = lambda t: t.transpose(0, 1).flatten(0, 1)                # [n_resp][B] -> [B * n_resp]
    return dict(hidden=hidden[:, n_p - 1:].flatten(0, 1).to(torch.bfloat16),
                ids=flat(torch.stack([i for i, _ in lists])).contiguous(), teacher=flat(torch.stack([t for _, t in lists])).contiguous(),
                next=full[:, n_p:].flatten().to(torch.int32), planted=pair["succ_D"][full[:, n_p - 1:-1].flatten().long()].to(torch.int32))


def draft_loss(head, d, bias, temperature=1.0):
    """Mean KL from the target's lists to the draft's head [V][d] over the rows of a batch `d` of make_examples."""
    logits = (d["hidden"] @ head.to(torch.bfloat16).T).float()
    logits = logits.scatter_add(1, d["planted"].long()[:, None], torch.full_like(logits[:, :1], bias))
    # (the teacher's values are log probabilities: their log-sum-exp over the whole row is 0 at temperature 1; at others the list
    # is renormalised)
    whole = torch.zeros_like(d["teacher"][:, 0]) if temperature == 1.0 else None
    return losses.distill_loss(logits, d["ids"], d["teacher"], temperature, whole).mean()


def draft_nll(head, d, bias):
    """Mean negative log-likelihood of the target's tokens under the draft's head, bf16 [V][d], differentiable in it."""
    return losses.head_nll(d["hidden"], head, d["next"], torch.full_like(d["teacher"][:, 0], 1.0 / len(d["next"])), d["planted"], bias)


def held_out_nll(head, d, bias):
    """Mean negative log-likelihood of the target's tokens under the draft."""
    logp, _, _ = binding.pacer_head_logprobs(d["hidden"], head.to(torch.bfloat16), d["next"], d["planted"], bias)
    return float(-logp.mean())


def train(cfg: synth.PairConfig, pair, device="cuda:0", n_prompts=64, n_prompt_tokens=32, n_resp=64, epochs=4, lr=1e-3, top=32,
          batch_prompts=8, temperature=1.0, seed=0, log=print, prompt_seed=5000, objective="kl", optimizer="torch"):
    """Returns ({"head": bf16 [V][d]}, report dict).  `pair` holds the target and draft tensors on `device`.  objective: "kl" or "nll";
    optimizer: "torch", "f32" or "8bit" (the library's AdamW with such states)."""
    if objective not in ("kl", "nll") or optimizer not in ("torch", "f32", "8bit"):
        raise ValueError("objective: 'kl' or 'nll'; optimizer: 'torch', 'f32' or '8bit'")
    if objective == "nll" and optimizer == "torch":
        raise ValueError("objective 'nll' trains a bf16 head with an f32 master: optimizer 'f32' or '8bit'")
    t0 = time.time()
    data = [make_examples(cfg, pair, synth.make_prompts(cfg.target.vocab, batch_prompts, n_prompt_tokens, seed=prompt_seed + i).to(device).long(),
                          n_resp, top) for i in range(0, n_prompts + batch_prompts, batch_prompts)]
    held = data.pop()                                               # the last batch is held out
    head = pair["draft"]["head"].detach().to(torch.float32 if objective == "kl" else torch.bfloat16, copy=True).requires_grad_(True)
    rep = {"held_out_nll_before": held_out_nll(head.detach(), held, cfg.succ_bias)}
    if optimizer == "torch":
        opt = torch.optim.AdamW([head], lr=lr, betas=(0.9, 0.999), weight_decay=0.0)
    else:
        opt = optim.AdamW([head], lr=lr, betas=(0.9, 0.999), weight_decay=0.0, states=optimizer, seed=seed if optimizer == "8bit" else None)
    for ep in range(epochs):
        total = 0.0
        for i in torch.randperm(len(data), generator=torch.Generator().manual_seed(seed + ep)).tolist():
            loss = draft_loss(head, data[i], cfg.succ_bias, temperature) if objective == "kl" else draft_nll(head, data[i], cfg.succ_bias)
            opt.zero_grad(set_to_none=True)
            loss.backward()
            opt.step()
            total += float(loss.detach())
        log(f"[train_draft] epoch {ep + 1}/{epochs}: {objective.upper()} {total / len(data):.4f}")
    with torch.no_grad():
        rep.update(held_out_nll_after=held_out_nll(head, held, cfg.succ_bias), held_out_kl=float(draft_loss(head, held, cfg.succ_bias)),
                   prompts=n_prompts, response_tokens=n_resp, epochs=epochs, lr=lr, top=top, objective=objective, optimizer=optimizer,
                   seconds=time.time() - t0)
    log(f"[train_draft] held-out NLL {rep['held_out_nll_before']:.3f} -> {rep['held_out_nll_after']:.3f}")
    return {"head": head.detach().to(torch.bfloat16).contiguous()}, rep


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="tiny")
    ap.add_argument("--out", required=True)
    ap.add_argument("--device", default="cuda:0")
    ap.add_argument("--prompts", type=int, default=64)
    ap.add_argument("--prompt-tokens", type=int, default=32)
    ap.add_argument("--response-tokens", type=int, default=64)
    ap.add_argument("--epochs", type=int, default=4)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--top", type=int, default=32)
    ap.add_argument("--batch-prompts", type=int, default=8)
    ap.add_argument("--objective", choices=("kl", "nll"), default="kl")
    ap.add_argument("--optimizer", choices=("torch", "f32", "8bit"), default=None, help="default: torch, with --objective nll f32")
    args = ap.parse_args()
    cfg = synth.CONFIGS[args.config]
    pair = synth.make_pair(cfg, seed=0, device=args.device, which=("target", "draft"))
    w, rep = train(cfg, pair, args.device, args.prompts, args.prompt_tokens, args.response_tokens, args.epochs, args.lr, args.top,
                   args.batch_prompts, objective=args.objective, optimizer=args.optimizer or ("torch" if args.objective == "kl" else "f32"))
    torch.save({"tensors": {k: v.cpu() for k, v in w.items()}, "report": rep, "config": args.config}, args.out)
    print(rep)


if __name__ == "__main__":
    main()
