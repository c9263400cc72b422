"""Plain 64-bit forms of the operators on rows of logits, from their definitions, and the bounds that fp32 arithmetic allows."""
import math

import torch

F32 = 2.0 ** -24                                   # half a step of fp32, relative


def rounding(dtype):
    """Half a step of a type relative to the value, and half its smallest step."""
    info = torch.finfo(dtype)
    return info.eps / 2, info.smallest_normal * info.eps / 2


def order(z, top):
    """Ids of the `top` best of one row: larger first, of equal ones the lower id, NaN last (-0 equals 0)."""
    row = z.tolist()
    return sorted(range(len(row)), key=lambda i: (math.isnan(row[i]), 0.0 if math.isnan(row[i]) else -row[i], i))[:top]


def order_rows(z, top):
    """The same for rows without NaN, by a stable sort."""
    return torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :top]


def softmax_parts(z):
    """(log p, lse) of 64-bit rows; a row of -inf keeps log p = -inf, lse = -inf."""
    m = z.max(1, keepdim=True).values
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    s = (z - m).exp().sum(1, keepdim=True)
    return torch.where(s == 0, torch.full_like(z, -math.inf), z - m - s.log()), (m + s.log())[:, 0]


def xlogx(lp):
    return torch.where(lp == -math.inf, torch.zeros_like(lp), lp * lp.exp())


def logprobs(z, tokens):
    z = z.double()
    lp, lse = softmax_parts(z)
    named = (tokens >= 0) & (tokens < z.shape[1])
    at = torch.where(named, tokens, torch.zeros_like(tokens)).long()
    return torch.where(named, lp.gather(1, at[:, None])[:, 0], torch.zeros_like(lse)), -xlogx(lp).sum(1), lse, lp


def logprobs_grad(z, tokens, lse, entropy, gl, gh, gs):
    """From the given (f32) lse and entropy, with the size of the terms that the result is a sum of."""
    z = z.double()
    l = z - lse.double()[:, None]
    dead = (lse == -math.inf)[:, None]
    p = torch.where(dead, torch.zeros_like(l), l.exp())
    zero = torch.zeros(z.shape[0], dtype=torch.float64, device=z.device)
    named = (tokens >= 0) & (tokens < z.shape[1]) if tokens is not None else zero > 0
    gl = torch.where(named, zero if gl is None else gl.double(), zero)
    gh = zero if gh is None else gh.double()
    gs = zero if gs is None else gs.double()
    ent = torch.zeros_like(p) if entropy is None else torch.where(p == 0, torch.zeros_like(p), p * (l + entropy.double()[:, None]))
    d = p * (gs - gl)[:, None] - gh[:, None] * ent
    size = p * (gs.abs() + gl.abs())[:, None] + gh.abs()[:, None] * (ent.abs() + p)
    if tokens is not None:
        at = torch.where(named, tokens, torch.zeros_like(tokens)).long()[:, None]
        add = torch.where(dead[:, 0], zero, gl)[:, None]
        d, size = d.scatter_add(1, at, add), size.scatter_add(1, at, add.abs())
    return d, size


def distill(z, ids, teacher, temperature, teacher_lse, weight):
    """(loss, lse, tail_lse, weight * gradient, size of its terms), entry by entry over the list."""
    z, t = z.double(), teacher.double() / temperature
    R, V = z.shape
    top = z.max(1, keepdim=True).values
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    z = (z - top) / temperature                    # (a row of huge values keeps its differences)
    ok = (ids >= 0) & (ids < V)
    t = torch.where(ok, t, torch.full_like(t, -math.inf))
    at = torch.where(ok, ids, torch.zeros_like(ids)).long()
    lq = softmax_parts(t)[0] if teacher_lse is None else t - teacher_lse.double()[:, None]
    q = lq.exp()
    lp, lse = softmax_parts(z)
    lpk = lp.gather(1, at)
    loss = torch.where(q > 0, q * (lq - lpk), torch.zeros_like(q)).sum(1)
    Q = q.sum(1)
    p = lp.exp()
    tail = None
    if teacher_lse is None:
        d = p * Q[:, None]
    else:
        inside = torch.zeros(R, V, dtype=torch.bool, device=z.device)
        for k in range(ids.shape[1]):
            inside[torch.arange(R, device=z.device)[ok[:, k]], at[ok[:, k], k]] = True
        rest = torch.where(inside, torch.full_like(z, -math.inf), z)
        w, tail = softmax_parts(rest)
        qt = (1 - Q).clamp(min=0)
        lpt = torch.where(tail == -math.inf, tail, tail - lse)
        loss = loss + torch.where(qt > 0, qt * (qt.log() - lpt), torch.zeros_like(qt))
        Q = Q + qt
        w = w.exp()
        d = torch.where(inside, p * Q[:, None], p * Q[:, None] - w * qt[:, None])
    size = d.abs() + p * Q[:, None]
    d, size = d.scatter_add(1, at, -q), size.scatter_add(1, at, q)
    if teacher_lse is not None:
        size = size + torch.where(inside, torch.zeros_like(w), w * qt[:, None])
    dead = ~ok.any(1) | (lse == -math.inf)
    loss = torch.where(dead, torch.zeros_like(loss), loss)
    d = torch.where(dead[:, None], torch.zeros_like(d), d)
    g = (weight.double() / temperature)[:, None]
    top = top[:, 0] / temperature
    return loss, lse + top, None if tail is None else tail + top, d * g, size * g.abs()
