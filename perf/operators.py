"""The operators on rows of logits, as a user's program calls them, with their plain forms.

  logprobs       log probabilities of given tokens, entropy and the best alternatives of rows of logits
  logprobs_back  the gradient of those log probabilities, entropies and log-sum-exps with respect to the logits
  distill_step   a training step's loss and gradient: KL from a teacher's top logits to the student's whole row
  distill_pair   the same loss and gradient as a forward call and a backward call
  head           log probabilities and entropy of given tokens straight from hidden rows and the LM head

Logits are noise of the width that an LM head gives, with one planted favourite a row (a confident model). Sizes: the
vocabularies and widths of ``synth.CONFIGS``, the rows of a verify window, of a batch of windows, of prompts and of a
training batch.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_BYTES = 650e6              # a drawn case's logits
MOST_FLOPS = 2.0 * 2048 * 4096 * 32000


def _logits(op, name, rows, vocab, dtype, **more):
    return dict(name=name, op=op, rows=rows, vocab=vocab, dtype=dtype, **more)


def _head(name, rows, vocab, d, bias):
    return dict(name=name, op="head", rows=rows, vocab=vocab, d=d, bias=bias)


def listed():
    return [
        # one token of a served sequence, the largest vocabulary, the alternatives that a client asks for
        _logits("logprobs", "logprobs_token", 1, 151936, "f32", top=20, pad=0, masked=0.0),
        # the verify window of a chat turn: last accepted token and 16 drafts
        _logits("logprobs", "logprobs_window", 17, 32000, "f32", top=5, pad=0, masked=0.0),
        # eight sequences' windows under a grammar that leaves a part of the vocabulary
        _logits("logprobs", "logprobs_batch", 136, 32256, "bf16", top=20, pad=0, masked=0.9),
        # a teacher's top logits for every position of a training batch; rows padded to a multiple of 64 columns
        _logits("logprobs", "logprobs_teacher", 2048, 32003, "bf16", top=64, pad=61, masked=0.0),
        # policy gradient or cross entropy over a batch of responses
        _logits("logprobs_back", "back_bf16", 2048, 32000, "bf16", pad=0, entropy=False),
        # ... with an entropy bonus and a penalty on the log-sum-exp, odd sizes
        _logits("logprobs_back", "back_entropy_f32", 1021, 32003, "f32", pad=0, entropy=True),
        # a draft model's training step on the target's 64 best logits
        _logits("distill_step", "distill_step_bf16", 2048, 32000, "bf16", pad=0, k=64, temperature=1.0, tail=False),
        # ... the largest vocabulary, the mass outside the teacher's list as one class
        _logits("distill_step", "distill_step_tail", 997, 151936, "f32", pad=0, k=20, temperature=2.0, tail=True),
        # two calls, few rows: the loss of one short sequence and its gradient
        _logits("distill_pair", "distill_pair_small", 33, 32003, "f16", pad=0, k=8, temperature=2.0, tail=True),
        # the draft model's head over one token
        _head("head_token", 1, 32000, 768, True),
        # scoring a full window under the widest target
        _head("head_window", 25, 32256, 7168, False),
        # scoring a whole prompt
        _head("head_prompt", 2048, 32000, 4096, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_back", "distill_step", "distill_pair", "head", "head"])
    vocab = rng.choice([4096, 32000, 32256, 151936, _log_int(rng, 500, 160000), _log_int(rng, 500, 160000)])
    if op == "head":
        d = rng.choice([128, 256, 768, 1536, 2048, 4096, 5120, 7168])
        return dict(op=op, rows=_log_int(rng, 1, min(2048, MOST_FLOPS / (2.0 * d * vocab))), vocab=vocab, d=d, bias=rng.random() < 0.5)
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    rows = _log_int(rng, 1, min(4096, MOST_BYTES / (vocab * TYPES[dtype].itemsize)))
    case = dict(op=op, rows=rows, vocab=vocab, dtype=dtype, pad=rng.choice([0, 0, 0, -vocab % 64, 3]))
    if op == "logprobs":
        return dict(case, top=rng.choice([0, 1, 5, 20, 64]), masked=rng.choice([0.0, 0.0, 0.5, 0.9]))
    if op == "logprobs_back":
        return dict(case, entropy=rng.random() < 0.5)
    return dict(case, k=_log_int(rng, 1, 128), temperature=rng.choice([1.0, 1.0, 2.0, 0.7]), tail=rng.random() < 0.5)


# ----------------------------------------------------------------------------- inputs


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(g, hi, *shape):
    return torch.randint(0, hi, shape, generator=g, device=DEVICE, dtype=torch.int32)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def prepare(case, seed):
    g, rows, vocab = _gen(seed), case["rows"], case["vocab"]
    s = dict(case=case)
    if case["op"] == "head":
        s["hidden"] = _normal(g, rows, case["d"]).to(torch.bfloat16)
        s["head"] = torch.empty(vocab, case["d"], device=DEVICE, dtype=torch.bfloat16)
        s["head"].normal_(0.0, 0.02, generator=g)
        s["tokens"] = _ints(g, vocab, rows)
        s["bias_ids"] = _ints(g, vocab, rows) if case["bias"] else None
        s["tokens"][::7] = -1 if rows > 7 else s["tokens"][::7]         # positions without a token to score
        return s
    dt = TYPES[case["dtype"]]
    z = _normal(g, rows, vocab + case["pad"])
    z.mul_(1.5)
    z.scatter_add_(1, _ints(g, vocab, rows, 1).long(), torch.full((rows, 1), 8.0, device=DEVICE))
    if case.get("masked"):
        keep = torch.rand(1, vocab + case["pad"], generator=g, device=DEVICE) >= case["masked"]
        keep[:, :128] = True
        z.masked_fill_(~keep, -math.inf)
    s["logits"] = z.to(dt)[:, :vocab]
    del z
    s["tokens"] = _ints(g, min(vocab, 128) if case.get("masked") else vocab, rows)
    if rows > 7:
        s["tokens"][::7] = -1                                           # padded positions
    if case["op"] == "logprobs_back":
        s["grad_logp"] = _normal(g, rows)
        s["grad_entropy"] = 0.01 * _normal(g, rows) if case["entropy"] else None
        s["grad_lse"] = 1e-3 * _normal(g, rows) if case["entropy"] else None
        # what the forward call left: the rows' log-sum-exp and entropy
        x = s["logits"].double() if rows * vocab < 3e7 else s["logits"].float()
        lse = torch.logsumexp(x, 1)
        x = x - lse[:, None]
        s["lse"], s["entropy"] = lse.float(), -(x * x.exp()).sum(1).float()
    if case["op"].startswith("distill"):
        k = min(case["k"], vocab)
        s["ids"] = torch.rand(rows, vocab, generator=g, device=DEVICE).topk(k, 1).indices.to(torch.int32) if rows * vocab < 1e7 else \
            ((_ints(g, vocab, rows, 1).long() + torch.arange(k, device=DEVICE) * (vocab // k)) % vocab).to(torch.int32)
        s["teacher"] = (1.5 * _normal(g, rows, k)).sort(1, descending=True).values + 6.0
        s["teacher_lse"] = None
        if case["tail"]:                                                # a tenth to a half of the teacher's mass lies outside
            outside = 0.1 + 0.4 * torch.rand(rows, generator=g, device=DEVICE)
            s["teacher_lse"] = torch.logsumexp(s["teacher"] / case["temperature"], 1) - torch.log1p(-outside)
        # a mean over the rows; in f16, whose small gradients vanish, with a loss scale of as many
        s["weight"] = torch.rand(rows, generator=g, device=DEVICE) / (1 if dt == torch.float16 else rows)
    return s


# ----------------------------------------------------------------------------- the passes


def _shift(z):
    """Rows minus their largest value, and that value: a row of -inf stays what it is."""
    m = z.max(1, keepdim=True).values
    return z - torch.where(torch.isinf(m), torch.zeros_like(m), m), m[:, 0]


def _log_softmax(z):
    x, m = _shift(z)
    total = x.exp().sum(1).log()
    return x - total[:, None], torch.where(torch.isinf(m), m, m + total)


def _picked(lp, tokens):
    at = tokens.clamp(min=0).long()[:, None]
    return torch.where(tokens >= 0, lp.gather(1, at)[:, 0], torch.zeros_like(lp[:, 0]))


def _entropy(lp):
    return -torch.where(torch.isinf(lp), torch.zeros_like(lp), lp * lp.exp()).sum(1)


def _plain_logprobs(logits, tokens, top):
    z = logits.float()
    lp, lse = _log_softmax(z)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top] if top else tokens.new_empty(len(tokens), 0).long()
    return dict(logp=_picked(lp, tokens), entropy=_entropy(lp), lse=lse, top_ids=order.to(torch.int32), top_logp=lp.gather(1, order))


def _plain_back(s):
    lp = s["logits"].float() - s["lse"][:, None]
    p = lp.exp()
    a = torch.where(s["tokens"] >= 0, -s["grad_logp"], torch.zeros_like(s["grad_logp"]))
    if s["grad_lse"] is not None:
        dz = p * (a + s["grad_lse"])[:, None] - p * s["grad_entropy"][:, None] * (lp + s["entropy"][:, None])
    else:
        dz = p * a[:, None]
    dz.scatter_add_(1, s["tokens"].clamp(min=0).long()[:, None], -a[:, None])
    return dz.to(s["logits"].dtype)


def _plain_distill(s):
    t, ids = s["case"]["temperature"], s["ids"].long()
    lp, _ = _log_softmax(s["logits"].float() / t)
    lq = s["teacher"] / t
    lq = _log_softmax(lq)[0] if s["teacher_lse"] is None else lq - s["teacher_lse"][:, None]
    q, lpk = lq.exp(), lp.gather(1, ids)
    loss, p = (q * (lq - lpk)).sum(1), lp.exp()
    if s["teacher_lse"] is None:
        dz = p * q.sum(1, keepdim=True)
    else:
        rest = lp.scatter(1, ids, -math.inf)
        log_pt = _log_softmax(rest)[1]
        qt = 1.0 - q.sum(1)
        loss = loss + qt * (qt.log() - log_pt)
        dz = p - (rest - log_pt[:, None]).exp() * qt[:, None]
    dz = dz.scatter_add(1, ids, -q) * (s["weight"] / t)[:, None]
    return dict(loss=loss, dlogits=dz.to(s["logits"].dtype))


def _plain_head(s):
    z = s["hidden"].float() @ s["head"].float().T
    if s["bias_ids"] is not None:
        z.scatter_add_(1, s["bias_ids"].long()[:, None], torch.full((len(z), 1), 8.0, device=z.device))
    lp, lse = _log_softmax(z)
    return dict(logp=_picked(lp, s["tokens"]), entropy=_entropy(lp), lse=lse)


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        from paper_2602_01274_b200 import binding as b
        if op == "logprobs":
            return dict(zip(("logp", "entropy", "lse", "top_ids", "top_logp"), b.pacer_logprobs(s["logits"], s["tokens"], case["top"])))
        if op == "logprobs_back":
            return b.pacer_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["entropy"], s["grad_logp"], s["grad_entropy"], s["grad_lse"])
        if op == "distill_step":
            loss, dlogits = b.pacer_distill_grad(s["logits"], s["ids"], s["teacher"], s["weight"], case["temperature"], s["teacher_lse"])
            return dict(loss=loss, dlogits=dlogits)
        if op == "distill_pair":
            loss, lse, tail_lse = b.pacer_distill(s["logits"], s["ids"], s["teacher"], case["temperature"], s["teacher_lse"])
            return dict(loss=loss, dlogits=b.pacer_distill_backward(s["logits"], s["ids"], s["teacher"], lse, tail_lse, s["weight"],
                                                                    case["temperature"], s["teacher_lse"]))
        return dict(zip(("logp", "entropy", "lse"), b.pacer_head_logprobs(s["hidden"], s["head"], s["tokens"], s["bias_ids"], 8.0)))
    if op == "logprobs":
        return _plain_logprobs(s["logits"], s["tokens"], case["top"])
    if op == "logprobs_back":
        return _plain_back(s)
    if op == "head":
        return _plain_head(s)
    return _plain_distill(s)


def work(case):
    rows, vocab = case["rows"], case["vocab"]
    if case["op"] == "head":
        d = case["d"]
        return dict(bytes=2.0 * vocab * d + 2.0 * rows * d + 20.0 * rows, flops=2.0 * rows * vocab * d + 4.0 * rows * vocab)
    n = float(rows) * vocab
    once = n * TYPES[case["dtype"]].itemsize
    if case["op"] == "logprobs":
        return dict(bytes=once + rows * (16.0 + 8.0 * case["top"]), flops=5.0 * n)
    if case["op"] == "logprobs_back":
        return dict(bytes=2 * once + 16.0 * rows, flops=(7.0 if case["entropy"] else 3.0) * n)
    return dict(bytes=2 * once + rows * (12.0 + 8.0 * case["k"]), flops=7.0 * n)


# ----------------------------------------------------------------------------- in 64 bits, from the definitions


def _exact_rows(case, s, lo, hi):
    """The outputs for rows lo..hi-1."""
    inf = math.inf
    if case["op"] == "head":
        z = torch.mm(s["hidden"][lo:hi].double(), s["head"].double().t())
        if s["bias_ids"] is not None:
            z[torch.arange(hi - lo, device=z.device), s["bias_ids"][lo:hi].long()] += 8.0
    else:
        z = s["logits"][lo:hi].double()
    r = torch.arange(hi - lo, device=z.device)
    if case["op"] in ("head", "logprobs"):
        lse = torch.logsumexp(z, dim=1)
        tok = s["tokens"][lo:hi].long()
        logp = torch.where(tok < 0, 0.0, z[r, tok.clamp(min=0)] - lse)
        p = torch.softmax(z, dim=1)
        out = dict(logp=logp, entropy=lse - torch.nan_to_num(p * z, nan=0.0).sum(1), lse=lse)
        if case["op"] == "logprobs":
            out["top_ids"] = None
            out["top_logp"] = z.topk(case["top"], dim=1).values - lse[:, None]
        return out
    if case["op"] == "logprobs_back":
        lse, ent, tok, g = s["lse"][lo:hi].double(), s["entropy"][lo:hi].double(), s["tokens"][lo:hi].long(), s["grad_logp"][lo:hi].double()
        g = g * (tok >= 0)
        p = torch.exp(z - lse[:, None])
        dz = -g[:, None] * p
        dz[r, tok.clamp(min=0)] += g
        if s["grad_lse"] is not None:
            dz += s["grad_lse"][lo:hi].double()[:, None] * p
            dz -= s["grad_entropy"][lo:hi].double()[:, None] * p * (z - lse[:, None] + ent[:, None])
        return dz
    t, ids = case["temperature"], s["ids"][lo:hi].long()
    z = z / t
    teach = s["teacher"][lo:hi].double() / t
    q = torch.softmax(teach, 1) if s["teacher_lse"] is None else torch.exp(teach - s["teacher_lse"][lo:hi].double()[:, None])
    p = torch.softmax(z, 1)
    pk = p.gather(1, ids)
    loss = (q * (q / pk).log()).sum(1)
    dz = p * q.sum(1, keepdim=True)
    if s["teacher_lse"] is not None:
        pt = p.scatter(1, ids, 0.0).sum(1)
        qt = 1.0 - q.sum(1)
        loss = loss + qt * (qt / pt).log()
        dz = p.scatter(1, ids, 0.0) * (1.0 - qt / pt)[:, None]
        dz.scatter_(1, ids, pk)
    dz[r[:, None], ids] -= q
    return dict(loss=loss, dlogits=dz * (s["weight"][lo:hi].double() / t)[:, None])


def exact(case, seed):
    s = prepare(case, seed)
    rows = case["rows"]
    step = max(1, int(4e7 // case["vocab"]))
    parts = [_exact_rows(case, s, lo, min(rows, lo + step)) for lo in range(0, rows, step)]
    if torch.is_tensor(parts[0]):
        return torch.cat(parts)
    return {k: None if v is None else torch.cat([p[k] for p in parts]) for k, v in parts[0].items()}
