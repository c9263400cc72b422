"""The operators of a head's training step, as a user's program calls them, with their plain forms.

  nll      negative log-likelihood of given tokens straight from hidden rows and the LM head, with the gradients of both
  back     the gradients of hidden rows and head from those of the log probabilities, entropies and log-sum-exps that an earlier
           call (``pacer_head_logprobs``) returned
  adamw    an AdamW step over a list of tensors, states in 32 or in 8 bits, with or without clipping by the global norm

Sizes: the vocabularies and widths of ``synth.CONFIGS``, the rows of a short response up to those of a training batch, the tensors
of the pre-verification layers, of a draft model, of heads, and odd ones.

States in 8 bits: blocks of 256 elements with two f32 scales.  The first moment is held as sign, 4 exponent and 3 mantissa bits of
its share of the block's largest (codes up to 480 steps of 1), the second as the root of its value, 4 exponent and 4 mantissa bits
(up to 496); no code stands for infinities or NaN.  With a seed, states and 16-bit parameters are rounded up or down at random with
16 random bits, a hash of (seed, step, tensor, element), the mean being the value; without one to nearest, halves up.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_FLOPS = 6.0 * 4093 * 151936 * 1536
MOST_ELEMENTS = 6e8
BETAS, EPS, DECAY, LR, STEP, SEED, MAX_NORM = (0.9, 0.999), 1e-8, 0.01, 1e-4, 37, 1234, 1.0
BLOCK, TOP_M, TOP_R = 256, 480.0, 496.0


def _head(op, name, rows, vocab, d, **more):
    return dict(dict(name=name, op=op, rows=rows, vocab=vocab, d=d, bias=False, grads="both", entropy=False), **more)


def _model(name, d, kv, ffn, layers, **more):
    """Tensors of decoder layers, stacked over layers."""
    return dict(dict(name=name, op="adamw", d=d, kv=kv, ffn=ffn, layers=layers, vocab=0, param="f32", grad="f32", master=False, bits=32,
                     seeded=False, clip=False), **more)


def _list(name, count, most, **more):
    """Tensors of odd sizes up to `most`."""
    return dict(dict(name=name, op="adamw", count=count, most=most, param="f32", grad="f32", master=False, bits=32, seeded=False, clip=False), **more)


def listed():
    return [
        # one short response under the draft's head
        _head("nll", "nll_short", 33, 32000, 768, bias=True),
        # the draft's head on a batch of eight responses of 64 tokens, the hidden states frozen
        _head("nll", "nll_draft", 512, 32000, 768, bias=True, grads="head"),
        # a batch under a 7B model's head
        _head("nll", "nll_wide", 2048, 32000, 4096),
        # the largest vocabulary, an odd number of rows
        _head("nll", "nll_vocab", 4093, 151936, 1536),
        # a policy gradient with an entropy bonus and a penalty on the log-sum-exp, odd sizes
        _head("back", "back_policy", 1021, 32003, 2048, entropy=True),
        # log probabilities of long responses
        _head("back", "back_long", 8192, 32256, 2048),
        # the pre-verification layer of the smallest pair: a launch and little else
        _model("adamw_tiny", 128, 128, 512, 1, clip=True),
        # the pre-verification layer of a 1.3B draft
        _model("adamw_preverify", 2048, 2048, 5504, 1, clip=True),
        # a 7B model's head in bf16 with an f32 master
        _model("adamw_head", 4096, 0, 0, 0, vocab=32000, param="bf16", grad="bf16", master=True),
        # many tensors of odd sizes
        _list("adamw_odd", 200, 400003, grad="f16", clip=True),
        # the largest head in bf16 without a master, states in 8 bits
        _model("adamw8_head", 1536, 0, 0, 0, vocab=151936, param="bf16", grad="bf16", bits=8, seeded=True),
        # twelve layers of a 1.3B draft
        _model("adamw8_layers", 2048, 2048, 5504, 12, grad="bf16", bits=8, clip=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["nll", "nll", "back", "adamw", "adamw", "adamw"])
    if op != "adamw":
        vocab = rng.choice([4096, 32000, 32256, 151936, _log_int(rng, 500, 160000), _log_int(rng, 500, 160000)])
        d = rng.choice([128, 256, 768, 1536, 2048, 4096, 5120, 7168, 8 * _log_int(rng, 16, 512)])
        rows = _log_int(rng, 1, min(8192, MOST_FLOPS / (6.0 * d * vocab)))
        c = _head(op, "", rows, vocab, d, bias=rng.random() < 0.4, grads=rng.choice(["both", "both", "both", "head", "hidden"]),
                  entropy=op == "back" and rng.random() < 0.5)
    else:
        kind = dict(param=rng.choice(["f32", "bf16"]), grad=rng.choice(["f32", "bf16", "bf16", "f16"]), bits=rng.choice([32, 8]),
                    seeded=rng.random() < 0.5, clip=rng.random() < 0.5)
        kind["master"] = kind["param"] == "bf16" and rng.random() < 0.5
        if rng.random() < 0.4:
            count = _log_int(rng, 1, 300)
            c = _list("", count, _log_int(rng, 50, MOST_ELEMENTS / 4 / count), **kind)
        else:
            d = rng.choice([128, 256, 768, 1536, 2048])
            ffn, kv = rng.choice([5 * d // 2, 8 * (d // 3)]), rng.choice([d, d // 4])
            layers = _log_int(rng, 1, min(28, MOST_ELEMENTS / (3 * d * ffn + 2 * d * d + 2 * d * kv)))
            c = _model("", d, kv, ffn, layers, **kind)
    del c["name"]
    return c


# ----------------------------------------------------------------------------- inputs


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(g, hi, *shape):
    return torch.randint(0, hi, shape, generator=g, device=DEVICE, dtype=torch.int32)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _shapes(case):
    if "count" in case:
        # sizes over the range, the first the largest, from a multiplicative sequence
        return [(max(1, int(case["most"] * (i * 0.6180339887 % 1.0) ** 2)) if i else case["most"],) for i in range(case["count"])]
    d, kv, f, n = case["d"], case["kv"], case["ffn"], case["layers"]
    layers = [(n, d + 2 * kv, d), (n, d, d), (n, f, d), (n, f, d), (n, d, f), (n, d), (n, d), (d,), (2, d)] if n else []
    return layers + ([(case["vocab"], d)] if case["vocab"] else [])


def _flat(shapes, dtype):
    """Tensors of the given shapes side by side in one buffer, each from a multiple of 64 elements on."""
    sizes = [math.prod(s) for s in shapes]
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + -(-n // 64) * 64)
    flat = torch.zeros(starts[-1], dtype=dtype, device=DEVICE)
    return flat, [flat[a:a + n].view(s) for a, n, s in zip(starts, sizes, shapes)]


def _prepare_adamw(case, g):
    shapes = _shapes(case)
    s = dict(case=case)
    pt = torch.float32 if case["master"] else TYPES[case["param"]]
    s["flat"], s["params"] = _flat(shapes, pt)
    s["flat"].normal_(0.0, 0.02, generator=g)
    s["flat_copy"], s["copies"] = _flat(shapes, torch.bfloat16) if case["master"] else (None, None)
    flat_grad, s["grads"] = _flat(shapes, TYPES[case["grad"]])
    flat_grad.normal_(0.0, 1e-2, generator=g)
    if case["bits"] == 32:
        s["flat_m"], s["exp_avg"] = _flat(shapes, torch.float32)
        s["flat_m"].normal_(0.0, 3e-3, generator=g)
        s["flat_v"], s["exp_avg_sq"] = _flat(shapes, torch.float32)
        s["flat_v"].normal_(0.0, 8e-3, generator=g).square_()
        s["scales"] = None
        return s
    # codes as earlier steps would have left them, and the blocks' scales
    s["flat_m"], s["exp_avg"] = _flat(shapes, torch.uint8)
    s["flat_v"], s["exp_avg_sq"] = _flat(shapes, torch.uint8)
    s["flat_m"].random_(0, 256, generator=g)
    s["flat_v"].random_(150, 256, generator=g)
    s["scales"] = []
    for t in s["params"]:
        k = -(-t.numel() // BLOCK)
        s["scales"].append((0.5 + torch.rand(k, 2, generator=g, device=DEVICE)) * torch.tensor([1e-2 / TOP_M, 2e-2 / TOP_R], device=DEVICE))
    return s


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, g)
    rows, vocab, d = case["rows"], case["vocab"], case["d"]
    s = dict(case=case)
    s["hidden"] = _normal(g, rows, d).to(torch.bfloat16)
    s["head"] = torch.empty(vocab, d, device=DEVICE, dtype=torch.bfloat16)
    s["head"].normal_(0.0, 1.5 / math.sqrt(d), generator=g)
    s["tokens"] = _ints(g, vocab, rows)
    s["bias_ids"] = _ints(g, vocab, rows) if case["bias"] else None
    if case["bias"]:
        s["tokens"][::2] = s["bias_ids"][::2]
    if rows > 7:
        s["tokens"][::7] = -1                                           # padded positions
    if case["op"] == "nll":
        s["weight"] = torch.rand(rows, generator=g, device=DEVICE) / rows
        return s
    s["grad_logp"] = _normal(g, rows) / rows
    s["grad_entropy"] = 0.1 * _normal(g, rows) / rows if case["entropy"] else None
    s["grad_lse"] = 0.01 * torch.rand(rows, generator=g, device=DEVICE) / rows if case["entropy"] else None
    s["logp"], s["entropy"], s["lse"] = _forward(s)[:3]                 # what the forward call left
    return s


# ----------------------------------------------------------------------------- the passes


def _logits(s):
    z = s["hidden"].float() @ s["head"].float().T
    if s["bias_ids"] is not None:
        z.scatter_add_(1, s["bias_ids"].long()[:, None], torch.full((len(z), 1), 8.0, device=z.device))
    return z


def _forward(s):
    """(log p of the tokens, entropy, log-sum-exp, log p)"""
    z = _logits(s)
    m = z.max(1, keepdim=True).values
    lse = (z - m).exp().sum(1, keepdim=True).log() + m
    lp = z - lse
    picked = torch.where(s["tokens"] >= 0, lp.gather(1, s["tokens"].clamp(min=0).long()[:, None])[:, 0], 0.0)
    return picked, -(lp * lp.exp()).sum(1), lse[:, 0], lp


def _products(s, dz):
    """The gradients of hidden rows and head from those of the logits."""
    g, out = s["case"]["grads"], {}
    if g != "head":
        out["dhidden"] = (dz @ s["head"].float()).to(torch.bfloat16)
    if g != "hidden":
        out["dhead"] = (dz.T @ s["hidden"].float()).to(torch.bfloat16)
    return out


def _at_tokens(s, dz, value):
    """dz with `value` added where the tokens are."""
    at = s["tokens"].clamp(min=0).long()[:, None]
    return dz.scatter_add_(1, at, torch.where(s["tokens"] >= 0, value, 0.0)[:, None])


def _plain_nll(s):
    logp, _, _, lp = _forward(s)
    w = torch.where(s["tokens"] >= 0, s["weight"], 0.0)
    dz = _at_tokens(s, lp.exp_().mul_(w[:, None]), -w)
    return dict(loss=-logp, **_products(s, dz))


def _plain_back(s):
    lp = _logits(s).sub_(s["lse"][:, None])
    p = lp.exp()
    gl = torch.where(s["tokens"] >= 0, s["grad_logp"], 0.0)
    c = -gl if s["grad_lse"] is None else s["grad_lse"] - gl
    dz = p * c[:, None]
    if s["grad_entropy"] is not None:
        dz -= p * (lp + s["entropy"][:, None]) * s["grad_entropy"][:, None]
    return _products(s, _at_tokens(s, dz, gl))


def _mix(x):
    """A hash of 32-bit numbers (held in int64)."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(n, tensor):
    """Two 16-bit numbers and a third for every element of a tensor."""
    key = _mix(SEED ^ _mix(STEP ^ _mix(tensor)))
    h = _mix(torch.arange(n, device=DEVICE) ^ key)
    return h & 0xFFFF, h >> 16, ((h * 0x9E3779B1) & 0xFFFFFFFF) >> 16


def _table(shift):
    return (torch.arange(256, dtype=torch.int32, device=DEVICE) << shift).view(torch.float32) * 2.0 ** 120


def _values(codes, scales, signed):
    """What 8-bit codes of one tensor stand for: first moments, or roots of second ones."""
    c = codes.reshape(-1).long()
    v = torch.where(c >= 128, -1.0, 1.0) * _table(20)[c & 127] if signed else _table(19)[c]
    return v * scales[:, 0 if signed else 1].repeat_interleave(BLOCK)[:len(v)]


def _codes(x, dither, top, shift, most):
    """(codes of |x|, scales) of one tensor."""
    n, a = len(x), x.abs()
    blocks = torch.nn.functional.pad(a, (0, -n % BLOCK)).view(-1, BLOCK)
    peak = blocks.max(1).values
    inverse = torch.where(peak > 1e-30, torch.full_like(peak, top) / peak, 0.0)
    scale = torch.where(peak > 1e-30, peak * (1.0 / top), 0.0)
    bits = (a * inverse.repeat_interleave(BLOCK)[:n] * 2.0 ** -120).view(torch.int32).long()
    code = (bits + (dither << (shift - 16) if dither is not None else 1 << (shift - 1))) >> shift
    return code.clamp(max=most), scale


def _clip(s):
    """The factor that takes the gradients' global norm to at most MAX_NORM, and the norm."""
    norm = sum(g.double().square().sum() for g in s["grads"]).sqrt().float()
    return (MAX_NORM / (norm + 1e-6)).clamp(max=1.0), norm


def _plain_adamw(s):
    case, out = s["case"], {}
    a, s2 = LR / (1 - BETAS[0] ** STEP), 1 / math.sqrt(1 - BETAS[1] ** STEP)
    if case["clip"]:
        factor, out["norm"] = _clip(s)
    for i, p in enumerate(s["params"]):
        g, m, v = s["grads"][i].float(), s["exp_avg"][i], s["exp_avg_sq"][i]
        if case["clip"]:
            g = g * factor
        g = g.reshape(-1)
        if case["bits"] == 32:
            m, r2 = m.view(-1), v.view(-1)
        else:
            m, r = _values(m, s["scales"][i], True), _values(v, s["scales"][i], False)
            r2 = r * r
        m = m * BETAS[0] + g * (1 - BETAS[0])
        v = r2 * BETAS[1] + (g * g) * (1 - BETAS[1])
        r = v.sqrt()
        x = p.reshape(-1).float() * (1 - LR * DECAY) - (m / (r * s2 + EPS)) * a
        rm, rr, rp = _random(len(x), i) if case["seeded"] else (None, None, None)
        if case["bits"] == 32:
            s["exp_avg"][i].view(-1).copy_(m)
            s["exp_avg_sq"][i].view(-1).copy_(v)
        else:
            code, s["scales"][i][:, 0] = _codes(m, rm, TOP_M, 20, 127)
            s["exp_avg"][i].view(-1).copy_(torch.where(m < 0, code + 128, code))
            code, s["scales"][i][:, 1] = _codes(r, rr, TOP_R, 19, 255)
            s["exp_avg_sq"][i].view(-1).copy_(torch.where(r > 0, code.clamp(min=1), code))
        if p.dtype == torch.bfloat16 and case["seeded"]:
            x = ((x.view(torch.int32).long() + rp) >> 16 << 16).to(torch.int32).view(torch.float32)
        p.view(-1).copy_(x)
        if case["master"]:
            s["copies"][i].view(-1).copy_(x)
    return out


def _states(s):
    """The updated parameters and states; what is held in 8 bits as the values it stands for."""
    case = s["case"]
    if case["bits"] == 32:
        m, v = s["flat_m"], s["flat_v"]
    elif own:
        from paper_2602_01274_b200 import binding as b
        sizes = [t.numel() for t in s["params"]]
        m, v = torch.empty(2, sum(sizes), device=DEVICE).unbind()
        b.pacer_adamw_states(s["exp_avg"], s["exp_avg_sq"], s["scales"], out=(m.split(sizes), v.split(sizes)))
    else:
        m = torch.cat([_values(c, k, True) for c, k in zip(s["exp_avg"], s["scales"])])
        v = torch.cat([_values(c, k, False).square() for c, k in zip(s["exp_avg_sq"], s["scales"])])
    return dict(params=s["flat"], exp_avg=m, exp_avg_sq=v, copies=s["flat_copy"])


def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2602_01274_b200 import binding as b
        want = (case.get("grads") != "head", case.get("grads") != "hidden")
        if case["op"] == "nll":
            loss, dhidden, dhead = b.pacer_head_nll_grad(s["hidden"], s["head"], s["tokens"], s["weight"], s["bias_ids"], 8.0, grads=want)
            return dict(loss=loss, dhidden=dhidden, dhead=dhead)
        if case["op"] == "back":
            dhidden, dhead = b.pacer_head_logprobs_backward(s["hidden"], s["head"], s["tokens"], s["logp"], s["lse"], s["entropy"], s["grad_logp"],
                                                            s["grad_entropy"], s["grad_lse"], s["bias_ids"], 8.0, grads=want)
            return dict(dhidden=dhidden, dhead=dhead)
        norm = b.pacer_grad_norm(s["grads"]) if case["clip"] else None
        b.pacer_adamw(s["params"], s["grads"], s["exp_avg"], s["exp_avg_sq"], STEP, LR, BETAS, EPS, DECAY, scales=s["scales"], copies=s["copies"],
                      seed=SEED if case["seeded"] else None, norm=norm, max_norm=MAX_NORM)
        return dict(_states(s), norm=norm)
    if case["op"] == "nll":
        return _plain_nll(s)
    if case["op"] == "back":
        return _plain_back(s)
    return dict(_plain_adamw(s), **_states(s))


def work(case):
    if case["op"] == "adamw":
        n = float(sum(math.prod(s) for s in _shapes(case)))
        p = 10.0 if case["master"] else 2.0 * TYPES[case["param"]].itemsize
        g = float(TYPES[case["grad"]].itemsize) * (2 if case["clip"] else 1)      # the norm needs all of them before the first step
        # read and written; in 8 bits the states' values go out beside the codes
        states = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK + 8.0
        return dict(bytes=n * (p + g + states), flops=15.0 * n)
    rows, vocab, d = case["rows"], case["vocab"], case["d"]
    both = 2 if case["grads"] == "both" else 1
    once = (vocab + rows) * d * 2.0
    out = {"both": (vocab + rows) * d * 2.0, "head": vocab * d * 2.0, "hidden": rows * d * 2.0}[case["grads"]]
    return dict(bytes=once + out + 24.0 * rows, flops=2.0 * (1 + both) * rows * vocab * d)


# ----------------------------------------------------------------------------- in 64 bits, from the definitions


def _exact_head(case, s):
    rows, vocab, d = case["rows"], case["vocab"], case["d"]
    head = s["head"].double()
    dhidden = torch.empty(rows, d, dtype=torch.float64, device=DEVICE) if case["grads"] != "head" else None
    dhead = torch.zeros(vocab, d, dtype=torch.float64, device=DEVICE) if case["grads"] != "hidden" else None
    loss = torch.empty(rows, dtype=torch.float64, device=DEVICE)
    step = max(1, int(1e8 // vocab))
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        h, tok, r = s["hidden"][lo:hi].double(), s["tokens"][lo:hi].long(), torch.arange(hi - lo, device=DEVICE)
        z = torch.mm(h, head.t())
        if s["bias_ids"] is not None:
            z[r, s["bias_ids"][lo:hi].long()] += 8.0
        named = (tok >= 0).double()
        tok = tok.clamp(min=0)
        if case["op"] == "nll":
            p = torch.softmax(z, 1)
            loss[lo:hi] = named * (torch.logsumexp(z, 1) - z[r, tok])
            w = s["weight"][lo:hi].double() * named
            dz = p * w[:, None]
            dz[r, tok] -= w
        else:
            lse, ent, g = s["lse"][lo:hi].double(), s["entropy"][lo:hi].double(), s["grad_logp"][lo:hi].double() * named
            p = torch.exp(z - lse[:, None])
            dz = -p * g[:, None]
            dz[r, tok] += g
            if case["entropy"]:
                dz += p * s["grad_lse"][lo:hi].double()[:, None]
                dz -= p * (z - lse[:, None] + ent[:, None]) * s["grad_entropy"][lo:hi].double()[:, None]
        if dhidden is not None:
            dhidden[lo:hi] = torch.mm(dz, head)
        if dhead is not None:
            dhead.addmm_(dz.t(), h)
    out = dict(loss=loss) if case["op"] == "nll" else {}
    return dict(out, **{k: v for k, v in (("dhidden", dhidden), ("dhead", dhead)) if v is not None})


def _exact_adamw(case, s):
    total = math.sqrt(sum(float(g.double().square().sum()) for g in s["grads"]))
    f = min(1.0, MAX_NORM / (total + 1e-6)) if case["clip"] else 1.0
    params = s["flat"].double()
    at, ms, vs = 0, [], []
    for i, p in enumerate(s["params"]):
        n = p.numel()
        g = s["grads"][i].double().reshape(-1) * f
        if case["bits"] == 8:
            k = torch.arange(n, device=DEVICE) // BLOCK
            c = s["exp_avg"][i].reshape(-1).long()
            e, x = (c >> 3) & 15, (c & 7).double()
            m = torch.where(e == 0, x / 8 * 2.0 ** -6, (1 + x / 8) * torch.exp2(e.double() - 7)) * (1 - 2 * (c >> 7)) * s["scales"][i][k, 0].double()
            c = s["exp_avg_sq"][i].reshape(-1).long()
            e, x = c >> 4, (c & 15).double()
            v = (torch.where(e == 0, x / 16 * 2.0 ** -6, (1 + x / 16) * torch.exp2(e.double() - 7)) * s["scales"][i][k, 1].double()) ** 2
        else:
            m, v = s["exp_avg"][i].double().reshape(-1), s["exp_avg_sq"][i].double().reshape(-1)
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
        step = m / (1 - BETAS[0] ** STEP) / ((v / (1 - BETAS[1] ** STEP)).sqrt() + EPS)
        x = p.reshape(-1).double() * (1 - LR * DECAY) - LR * step
        params[at:at + n] = x
        pad = -n % 64
        at += n + pad
        ms.append(torch.nn.functional.pad(m, (0, pad)))
        vs.append(torch.nn.functional.pad(v, (0, pad)))
    if case["bits"] == 8:
        # which of two codes a value gets goes by its last f32 bit: 64-bit arithmetic takes the other one for a few in a million, a
        # sixteenth of their value off
        ms = vs = None
    else:                                                               # (what lies between the tensors stays as it is)
        ms, vs = torch.cat(ms), torch.cat(vs)
        tail = [torch.ones(p.numel() + -p.numel() % 64, dtype=torch.bool, device=DEVICE) for p in s["params"]]
        for p, t in zip(s["params"], tail):
            t[p.numel():] = False
        tail = torch.cat(tail)
        ms, vs = torch.where(tail, ms, s["flat_m"].double()), torch.where(tail, vs, s["flat_v"].double())
    out = dict(params=params, exp_avg=ms, exp_avg_sq=vs, copies=None)
    if case["master"]:
        out["copies"] = _flat([p.shape for p in s["params"]], torch.float64)[0]
        inside = torch.zeros_like(out["copies"], dtype=torch.bool)
        at = 0
        for p in s["params"]:
            inside[at:at + p.numel()] = True
            at += p.numel() + -p.numel() % 64
        out["copies"] = torch.where(inside, params, out["copies"])
    if case["clip"]:
        out["norm"] = torch.tensor(total, dtype=torch.float64)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(case, s) if case["op"] == "adamw" else _exact_head(case, s)
