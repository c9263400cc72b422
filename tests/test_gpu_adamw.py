"""AdamW over many tensors against its formulas in 64 bits, 8-bit states against a 32-bit evaluation of the same formulas (equal bits: which of
two codes a value gets goes by its last one) and against the codes' definition, the gradients' norm, and the optimiser on top.

Tolerance of a step in f32: m and v are sums of two rounded products (three half steps of their terms), the update has six roundings and two
approximate functions of 2 units (16 half steps), the parameter three."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = [1, 0, 255, 256, 257, 4096, 4097, 31, 8 * 1024 + 5, 100003]


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def make(sizes, ptype, gtype, bits, seed=0, master=False, shift=0):
    """Tensors that begin `shift` elements into their storage."""
    g = gen(seed)

    def new(n, dtype, scale):
        x = torch.randn(n + shift, generator=g, device=DEV) * scale
        return (x.to(torch.uint8) if dtype is torch.uint8 else x.to(dtype))[shift:]

    p = [new(n, torch.float32 if master else TYPES[ptype], 0.02) for n in sizes]
    gr = [new(n, TYPES[gtype], 1e-2) for n in sizes]
    copies = [new(n, torch.bfloat16, 0.0) for n in sizes] if master else None
    if bits == 32:
        return p, gr, [new(n, torch.float32, 3e-3) for n in sizes], [new(n, torch.float32, 8e-3).square() for n in sizes], None, copies
    m = [torch.randint(0, 256, (n + shift,), generator=g, device=DEV, dtype=torch.uint8)[shift:] for n in sizes]
    v = [torch.randint(0, 256, (n + shift,), generator=g, device=DEV, dtype=torch.uint8)[shift:] for n in sizes]
    s = [torch.rand(-(-n // 256), 2, generator=g, device=DEV) * torch.tensor([2e-5, 6e-9], device=DEV) for n in sizes]
    return p, gr, m, v, s, copies


def mix(x):
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_bits(n, seed, step, tensor):
    key = mix((seed & 0xFFFFFFFF) ^ mix(seed >> 32) ^ mix(step ^ mix(tensor)))
    h = mix(torch.arange(n, device=DEV) ^ key)
    return h & 0xFFFF, h >> 16, ((h * 0x9E3779B1) & 0xFFFFFFFF) >> 16


def value(codes, scale, mantissa, exponent_bits, lowest):
    """A code's value from its definition: sign (with 4 exponent bits), exponent, mantissa; in 64 bits."""
    c = codes.long()
    sign = torch.where(c >= 128, -1.0, 1.0).double() if exponent_bits == 4 else 1.0
    c = c & 127 if exponent_bits == 4 else c
    e, x = c >> mantissa, (c & 7).double() / 8
    return sign * torch.where(e == 0, x * 2.0 ** lowest, (1 + x) * torch.exp2(e.double() + lowest - 1)) * scale.double()


def values(m, v, s):
    k = torch.arange(len(m), device=DEV) // 256
    return value(m, s[k, 0], 3, 4, -6), value(v, s[k, 1], 3, 5, -15)


def encode(x, dither, signed):
    """Codes and scales of f32 values, by f32 operations rounded one by one: the grid's floor after the dither."""
    n, top, low = len(x), (480.0 if signed else 61440.0), (-6 if signed else -15)
    if not n:
        return x.to(torch.uint8), torch.zeros(0, device=DEV)
    peak = torch.nn.functional.pad(x.abs(), (0, -n % 256)).view(-1, 256).max(1).values
    some = peak > 1e-30
    inv = torch.where(some, torch.full_like(peak, top) / peak, 0.0)
    scale = torch.where(some, peak * (1.0 / top), 0.0)
    u = (x.abs() * inv.repeat_interleave(256)[:n]).double()
    # (what is smaller than 2^-23 of the smallest step has no f32 bits behind it)
    least = 2.0 ** (low - 23)
    u = torch.where(u < 2.0 ** low, torch.round(u / least) * least, u)
    step = torch.exp2(torch.floor(torch.log2(u.clamp(min=2.0 ** low))) - 3)
    q = torch.floor(u / step + (0.5 if dither is None else dither.double() / 65536)) * step
    q = q.clamp(max=top)
    e = torch.floor(torch.log2(q.clamp(min=2.0 ** low)))
    code = torch.where(q < 2.0 ** low, q / 2.0 ** (low - 3), (e - low + 1) * 8 + (q / torch.exp2(e) - 1) * 8).round().long()
    code = torch.where(x < 0, code + 128, code) if signed else torch.where(x > 0, code.clamp(min=1), code)
    return code.to(torch.uint8), scale


def step64(p, g, m, v, lr, betas, eps, wd, t):
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    up = lr / (1 - betas[0] ** t) * m / ((v / (1 - betas[1] ** t)).sqrt() + eps)
    return p * (1 - lr * wd) - up, m, v, up


HYPER = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)


@pytest.mark.parametrize("ptype,master", [("f32", False), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("gtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("clip", [False, True])
def test_step(ptype, master, gtype, shift, clip):
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, _, copies = make(SIZES, ptype, gtype, 32, 1, master, shift)
    old = [[x.double() for x in y] for y in (p, g, m, v)]
    norm = b.pacer_grad_norm(g)
    total = math.sqrt(sum(float(x.square().sum()) for x in old[1]))
    assert abs(float(norm) - total) <= 2 * F32 * total
    b.pacer_adamw(b.AdamwTensors(p, m, v, copies=copies), g, 5, norm=norm if clip else None, max_norm=0.3 if clip else 0.0, **HYPER)
    f = min(1.0, 0.3 / (total + 1e-6)) if clip else 1.0
    assert not clip or f < 0.5
    for i in range(len(SIZES)):
        want, wm, wv, up = step64(old[0][i], old[1][i] * f, old[2][i], old[3][i], HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], 5)
        terms = 0.9 * old[2][i].abs() + 0.1 * (old[1][i] * f).abs()
        assert ((m[i].double() - wm).abs() <= 6 * F32 * terms).all()
        assert ((v[i].double() - wv).abs() <= 8 * F32 * wv + 1e-38).all()
        # (a first moment that is the difference of its terms is off by more than its size says)
        off = 16 * F32 * up.abs() + 8 * F32 * terms * torch.where(wm != 0, up / wm, 0.0).abs() + 4 * F32 * old[0][i].abs()
        half = 0.0 if p[i].dtype == torch.float32 else 2.0 ** -8
        assert ((p[i].double() - want).abs() <= off + half * 1.01 * want.abs() + 1e-38).all()
        if master:
            assert torch.equal(copies[i], p[i].to(torch.bfloat16))


@pytest.mark.parametrize("ptype,gtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("seed", [None, 77, (5 << 32) + 3])
def test_step_with_8_bit_states(ptype, gtype, shift, seed):
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, s, _ = make(SIZES, ptype, gtype, 8, 2, False, shift)
    tensors = b.AdamwTensors(p, m, v, s)
    got_m, got_v = b.pacer_adamw_states(tensors)
    for i in range(len(SIZES)):
        wm, wv = values(m[i], v[i], s[i])
        assert torch.equal(got_m[i], wm.float()) and torch.equal(got_v[i], wv.float())
    old_p, before = [x.clone() for x in p], [(a.clone(), c.clone()) for a, c in zip(got_m, got_v)]
    b.pacer_adamw(tensors, g, 9, seed=seed, **HYPER)
    for i, n in enumerate(SIZES):
        x = g[i].float()
        nm = before[i][0] * 0.9 + x * (1 - 0.9)
        nv = before[i][1] * 0.999 + (x * x) * (1 - 0.999)
        rm, rv, rp = random_bits(n, seed, 9, i) if seed is not None else (None, None, None)
        for new, codes, col, dither in ((nm, m[i], 0, rm), (nv, v[i], 1, rv)):
            want, scale = encode(new, dither, col == 0)
            assert torch.equal(codes, want) and torch.equal(s[i][:, col], scale), (i, n, col)
        want, wm, wv, up = step64(old_p[i].double(), x.double(), before[i][0].double(), before[i][1].double(), *[HYPER[k] for k in ("lr", "betas", "eps", "weight_decay")], 9)
        off = 16 * F32 * up.abs() + 8 * F32 * (before[i][0].abs() + x.abs()).double() * torch.where(wm != 0, up / wm, 0.0).abs() + 4 * F32 * old_p[i].double().abs()
        half = 0.0 if ptype == "f32" else 2.0 ** -8 if seed is None else 2.0 ** -7
        assert ((p[i].double() - want).abs() <= off + half * 1.01 * want.abs() + 1e-38).all()


def test_types_mixed_in_a_list():
    """Every pair of types in one call, tensors on and off the 16-byte grid: the random numbers go by the place in the list."""
    from paper_2602_01274_b200 import binding as b
    kinds = [(pt, gt, shift) for pt in ("f32", "bf16") for gt in ("f32", "bf16", "f16") for shift in (0, 1)]
    made = [make([n], pt, gt, 8, 20 + i, False, shift) for i, ((pt, gt, shift), n) in enumerate(zip(kinds, [700, 3000, 1, 9000, 512, 255, 4097, 31, 256, 8192, 100, 2047]))]
    p, g, m, v, s = ([x[k][0] for x in made] for k in range(5))
    old_m, old_v = b.pacer_adamw_states(b.AdamwTensors(p, m, v, s))
    b.pacer_adamw(b.AdamwTensors(p, m, v, s), g, 6, seed=1234567890123, **HYPER)
    for i in range(len(p)):
        x = g[i].float()
        rm, rv, _ = random_bits(len(x), 1234567890123, 6, i)
        for new, codes, col, dither in ((old_m[i] * 0.9 + x * (1 - 0.9), m[i], 0, rm), (old_v[i] * 0.999 + (x * x) * (1 - 0.999), v[i], 1, rv)):
            want, scale = encode(new, dither, col == 0)
            assert torch.equal(codes, want) and torch.equal(s[i][:, col], scale), (i, kinds[i])


def test_16_bit_parameters_rounded_at_random_move_as_they_should():
    """Updates far below a parameter's last bit: nearest never moves, at random the mean does."""
    from paper_2602_01274_b200 import binding as b
    n, lr, steps = 1 << 16, 1e-4, 40
    for seed in (None, 3):
        p = [torch.ones(n, device=DEV, dtype=torch.bfloat16)]
        t = b.AdamwTensors(p, [torch.zeros(n, device=DEV)], [torch.zeros(n, device=DEV)])
        g = [torch.ones(n, device=DEV, dtype=torch.bfloat16)]
        for k in range(steps):
            b.pacer_adamw(t, g, k + 1, lr, weight_decay=0.0, seed=seed)
        moved = 1.0 - float(p[0].double().mean())
        # (each step moves by lr; a step of 2^-8 below 1 is taken with chance lr / 2^-8: the mean of n * steps of them)
        sigma = 2.0 ** -8 * math.sqrt(lr * 2.0 ** 8 * steps / n)
        assert moved == 0.0 if seed is None else abs(moved - lr * steps) < 6 * sigma + 1e-3 * lr * steps


def test_8_bit_second_moments_follow():
    """A second moment whose gradients change size: rounded at random it follows the 32-bit one, an eighth of a step apart at most on average."""
    from paper_2602_01274_b200 import binding as b
    n = 1 << 14
    state = [(b.AdamwTensors([torch.zeros(n, device=DEV)], [torch.zeros(n, device=DEV)], [torch.zeros(n, device=DEV)])),
             (b.AdamwTensors([torch.zeros(n, device=DEV)], [torch.zeros(n, dtype=torch.uint8, device=DEV)], [torch.zeros(n, dtype=torch.uint8, device=DEV)],
                             [torch.zeros(n // 256, 2, device=DEV)]))]
    g = gen(4)
    for k in range(600):
        x = [torch.randn(n, generator=g, device=DEV) * (1.0 if k < 200 else 0.25)]
        for t in state:
            b.pacer_adamw(t, x, k + 1, 1e-4, seed=11)
    v32, v8 = state[0].tensors[3][0].double(), b.pacer_adamw_states(state[1])[1][0].double()
    # each step rounds v by at most an eighth of it, independently and without bias; with b2 = 0.999 some 500 roundings are alive, and n
    # elements are averaged: the mean's deviation is below (1 / 8) sqrt(500 / n) / 2 of it
    assert abs(float(v8.mean() / v32.mean()) - 1) < 6 * math.sqrt(500 / n) / 16
    assert float((v8 - v32).abs().mean() / v32.mean()) < 1.0


def test_not_finite_and_zero():
    from paper_2602_01274_b200 import binding as b
    for bits in (32, 8):
        p, g, m, v, s, _ = make([1000, 5000], "f32", "f32", bits, 3)
        g[1][77] = math.inf
        keep = [x.clone() for y in (p, m, v) for x in y]
        norm = b.pacer_grad_norm(g)
        assert not torch.isfinite(norm)
        b.pacer_adamw(b.AdamwTensors(p, m, v, s), g, 1, 1e-3, norm=norm, max_norm=1.0)
        b.pacer_adamw(b.AdamwTensors(p, m, v, s), g, 1, 1e-3, norm=norm)
        assert all(torch.equal(x, y) for x, y in zip(keep, [x for y in (p, m, v) for x in y]))
        # without the norm the element (in 8 bits its block) is spoiled, and nothing else
        t = b.AdamwTensors(p, m, v, s)
        b.pacer_adamw(t, g, 1, 1e-3)
        assert torch.isfinite(p[0]).all() and not torch.isfinite(p[1][77]) and int((~torch.isfinite(p[1])).sum()) == 1
        x = (m, v) if bits == 32 else b.pacer_adamw_states(t)
        assert torch.isfinite(x[0][0]).all() and not torch.isfinite(x[0][1][77])
        bad = ~torch.isfinite(x[0][1])
        assert int(bad.sum()) == 1 if bits == 32 else not bad[256:].any()
    # all zeros: no update but the decay, states stay 0
    z = torch.zeros(600, device=DEV)
    p, s = torch.ones(600, device=DEV), torch.zeros(3, 2, device=DEV)
    c = [torch.zeros(600, dtype=torch.uint8, device=DEV) for _ in range(2)]
    t = b.AdamwTensors([p], [c[0]], [c[1]], [s])
    b.pacer_adamw(t, [z], 1, 0.5, weight_decay=0.5, seed=1)
    assert (p == 0.75).all() and (s == 0).all() and (c[1] == 0).all()


def test_many_tensors_streams_and_graphs():
    """More tensors than one launch takes; a captured step whose count and rate are on the device."""
    from paper_2602_01274_b200 import binding as b
    sizes = [(i * 37) % 700 for i in range(1100)]
    p, g, m, v, _, _ = make(sizes, "f32", "bf16", 32, 6)
    norm = b.pacer_grad_norm(g)
    assert abs(float(norm) - math.sqrt(sum(float(x.double().square().sum()) for x in g))) <= 2 * F32 * float(norm)
    want = [[x.clone() for x in y] for y in (p, m, v)]
    one = [b.AdamwTensors([want[0][i]], [want[1][i]], [want[2][i]]) for i in range(len(sizes))]
    for i in range(0, len(sizes), 50):
        b.pacer_adamw(one[i], [g[i]], 3, 1e-3)
    b.pacer_adamw(b.AdamwTensors(p, m, v), g, 3, 1e-3)
    for i in range(0, len(sizes), 50):
        assert torch.equal(p[i], want[0][i]) and torch.equal(m[i], want[1][i]) and torch.equal(v[i], want[2][i])
    # captured: three replays are three steps
    p, g, m, v, s, _ = make([5000, 300], "bf16", "bf16", 8, 7)
    q = [[x.clone() for x in y] for y in (p, m, v, s)]
    t, u = b.AdamwTensors(p, m, v, s), b.AdamwTensors(*q)
    step, lr = torch.zeros((), dtype=torch.int32, device=DEV), torch.full((), 1e-3, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step += 1
        b.pacer_adamw(t, g, step, lr, seed=9, norm=b.pacer_grad_norm(g), max_norm=0.5)
    for k in range(3):
        lr.fill_(1e-3 * (k + 1))
        graph.replay()
        b.pacer_adamw(u, g, k + 1, float(lr), seed=9, norm=b.pacer_grad_norm(g), max_norm=0.5)
    assert int(step) == 3 and all(torch.equal(x, y) for a, c in zip((p, m, v, s), q) for x, y in zip(a, c))


def test_elements_beyond_32_bits():
    """A tensor whose last elements have numbers above 2^32 (27 GB): they go as they would by themselves."""
    from paper_2602_01274_b200 import binding as b
    n, last = (1 << 32) + 300, 556                                       # (the last blocks of 256 begin at 2^32 - 256)
    p, g = (torch.zeros(n, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    m, v = (torch.zeros(n, device=DEV, dtype=torch.uint8) for _ in range(2))
    s = torch.zeros(-(-n // 256), 2, device=DEV)
    q, h, c, d, e = make([last], "bf16", "bf16", 8, 10)[:5]
    for big, small in zip((p, g, m, v), (q, h, c, d)):
        big[-last:] = small[0]
    s[-3:] = e[0]
    norm = b.pacer_grad_norm([g])
    assert torch.equal(norm, b.pacer_grad_norm(h))
    b.pacer_adamw(b.AdamwTensors([p], [m], [v], [s]), [g], 4, 1e-3)
    b.pacer_adamw(b.AdamwTensors(q, c, d, e), h, 4, 1e-3)
    for big, small in zip((p, m, v), (q, c, d)):
        assert torch.equal(big[-last:], small[0]) and not big[-last - 300:-last].any()
    assert torch.equal(s[-3:], e[0])


def test_refusals():
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, _, _ = make([100, 50], "f32", "f32", 32, 8)
    for bad in (lambda: b.AdamwTensors(p, m[:1], v), lambda: b.AdamwTensors(p, m, [v[0], v[1][:-1]]), lambda: b.AdamwTensors(p, m, [x.double() for x in v]),
                lambda: b.AdamwTensors([x.half() for x in p], m, v), lambda: b.AdamwTensors([x.cpu() for x in p], m, v),
                lambda: b.AdamwTensors([torch.zeros(200, device=DEV)[::2], p[1]], m, v), lambda: b.AdamwTensors(p, m, v, copies=p),
                lambda: b.AdamwTensors(p, [x.to(torch.uint8) for x in m], [x.to(torch.uint8) for x in v], [torch.zeros(2, 2, device=DEV)] * 2),
                lambda: b.pacer_adamw(b.AdamwTensors(p, m, v), g[:1], 1, 1e-3), lambda: b.pacer_adamw(b.AdamwTensors(p, m, v), [g[0], g[1][:-1]], 1, 1e-3),
                lambda: b.pacer_adamw(b.AdamwTensors(p, m, v), g, torch.ones((), device=DEV), 1e-3), lambda: b.pacer_grad_norm([])):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(b.PacerError, match="two params overlap"):
        b.pacer_adamw(b.AdamwTensors([p[0], p[0]], [m[0], m[0].clone()], [v[0], v[0].clone()]), [g[0], g[0]], 1, 1e-3)
    with pytest.raises(b.PacerError, match="step out of range"):
        b.pacer_adamw(b.AdamwTensors(p, m, v), g, 0, 1e-3)
    b.pacer_adamw(b.AdamwTensors([], [], []), [], 1, 1e-3)
    versions = [x._version for x in (*p, *m, *v)]
    b.pacer_adamw(b.AdamwTensors(p, m, v), g, 1, 1e-3)
    assert all(x._version > y for x, y in zip((*p, *m, *v), versions))


# ----------------------------------------------------------------------------- the optimiser


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_optimiser_against_torch(dtype):
    """Twelve steps beside torch.optim.AdamW in 64 bits on the same gradients."""
    from paper_2602_01274_b200 import optim
    g = gen(12)
    start = [torch.randn(s, generator=g, device=DEV).to(dtype) for s in ((33, 65), (7,), (128, 64), ())]
    mine = [torch.nn.Parameter(x.clone()) for x in start]
    theirs = [torch.nn.Parameter(x.double()) for x in start]
    groups = lambda ps: [dict(params=ps[:2], lr=1e-2), dict(params=ps[2:], weight_decay=0.3)]
    a = optim.AdamW(groups(mine), lr=3e-3, betas=(0.8, 0.95), max_norm=2.0)
    c = torch.optim.AdamW(groups(theirs), lr=3e-3, betas=(0.8, 0.95))
    for k in range(12):
        for x, y in zip(mine, theirs):
            grad = torch.randn(x.shape, generator=g, device=DEV).to(dtype)
            x.grad, y.grad = grad, grad.double()
        if k == 5:                                                         # one parameter left out of a step
            mine[1].grad = theirs[1].grad = None
        torch.nn.utils.clip_grad_norm_([y for y in theirs if y.grad is not None], 2.0)
        a.step()
        c.step()
    for x, y, s in zip(mine, theirs, start):
        # 12 steps of at most lr * a few; each f32 step is off by 20 half steps of its update and 4 of the parameter
        bound = 12 * (40 * F32 * 1e-2 * 5 + 4 * F32 * (y.abs() + s.double().abs() + 0.1)) + (0 if dtype == torch.float32 else 2.0 ** -8 * y.abs())
        assert ((x.double() - y).abs() <= bound).all()
    assert a.state[mine[1]]["step"] == 11 and ("master" in a.state[mine[0]]) == (dtype == torch.bfloat16)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_optimiser_saved_loaded_and_captured(states):
    from paper_2602_01274_b200 import optim
    new = lambda: [torch.nn.Parameter(torch.randn(n, generator=gen(n), device=DEV).to(torch.bfloat16)) for n in (5000, 300, 70000)]
    grads = [[torch.randn(p.shape, generator=gen(30 + k), device=DEV).to(torch.bfloat16) for p in new()] for k in range(6)]

    def run(opt, ps, ks):
        for k in ks:
            for p, x in zip(ps, grads[k]):
                p.grad = x.clone() if p.grad is None else p.grad.copy_(x)
            opt.step()

    a = new()
    oa = optim.AdamW(a, lr=1e-3, states=states, seed=4)
    run(oa, a, range(6))
    if states == "8bit":
        assert oa.state[a[0]]["exp_avg"].dtype == torch.uint8 and oa.state[a[1]]["exp_avg"].dtype == torch.float32
    b = new()
    ob = optim.AdamW(b, lr=1e-3, states=states, seed=4)
    run(ob, b, range(3))
    c = [torch.nn.Parameter(p.detach().clone()) for p in b]
    oc = optim.AdamW(c, lr=1e-3, states=states, seed=4)
    oc.load_state_dict(ob.state_dict())
    run(oc, c, range(3, 6))
    assert all(torch.equal(x, y) for x, y in zip(a, c))
    d = new()
    od = optim.AdamW(d, lr=torch.full((), 1e-3, device=DEV), states=states, seed=4, capturable=True)
    run(od, d, range(1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        od.step()
    for k in range(1, 6):
        for p, x in zip(d, grads[k]):
            p.grad.copy_(x)
        graph.replay()
    assert all(torch.equal(x, y) for x, y in zip(a, d))


def test_optimiser_refusals():
    from paper_2602_01274_b200 import optim
    p = torch.nn.Parameter(torch.zeros(8, device=DEV))
    for bad in (dict(states="4bit"), dict(betas=(1.0, 0.9)), dict(lr=-1.0), dict(lr=torch.ones((), device=DEV)), dict(max_norm=-1.0)):
        with pytest.raises(ValueError):
            optim.AdamW([p], **bad)
    for q in (torch.zeros(8), torch.zeros(8, device=DEV, dtype=torch.float16), torch.zeros(8, 8, device=DEV).T[:4]):
        with pytest.raises(ValueError):
            optim.AdamW([torch.nn.Parameter(q)])


def test_optimiser_whose_parameters_take_turns():
    """Parameters without a gradient in some steps have counts of their own, on the host and on the device alike; copies of an optimiser, groups
    that are added."""
    import copy
    from paper_2602_01274_b200 import optim
    new = lambda: [torch.nn.Parameter(torch.randn(n, generator=gen(n), device=DEV)) for n in (500, 300, 70)]
    sides = [new(), new()]
    opts = [optim.AdamW(ps[:2], lr=1e-2, capturable=c) for ps, c in zip(sides, (False, True))]
    for o, ps in zip(opts, sides):
        o.add_param_group(dict(params=ps[2:], lr=1e-3))
    turns = [(0, 1, 2), (0,), (0, 2), (1, 2), (0, 1, 2), (2,)]
    for k, turn in enumerate(turns):
        for o, ps in zip(opts, sides):
            for i, p in enumerate(ps):
                p.grad = torch.randn(p.shape, generator=gen(50 + k * 3 + i), device=DEV) if i in turn else None
            o.step()
    assert all(torch.equal(x, y) for x, y in zip(*sides))
    want = [sum(i in t for t in turns) for i in range(3)]
    for o, ps in zip(opts, sides):
        assert [int(o.state[p]["step"]) for p in ps] == want
    twin = copy.deepcopy(opts[0])
    assert twin.states == "f32" and len(twin.param_groups) == 2
    for p, g in zip([p for gr in twin.param_groups for p in gr["params"]], sides[0]):
        p.grad = g.grad = torch.ones_like(p)
    twin.step()
    opts[0].step()
    assert all(torch.equal(p, q) for p, q in zip([p for gr in twin.param_groups for p in gr["params"]], sides[0]))
    with pytest.raises(ValueError):
        opts[0].add_param_group(dict(params=[torch.nn.Parameter(torch.zeros(4))]))
    assert len(opts[0].param_groups) == 2


def test_tensors_whose_storage_is_exchanged():
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, _, _ = make([1000, 40], "f32", "f32", 32, 9)
    t = b.AdamwTensors(p, m, v)
    b.pacer_adamw(t, g, 1, 1e-3)
    q = [x.clone() for x in (p[0], m[0], v[0])]
    b.pacer_adamw(b.AdamwTensors(q[:1], q[1:2], q[2:]), g[:1], 2, 1e-3)
    kept = p[0].clone()
    p[0].data = kept.clone()
    b.pacer_adamw(t, g, 2, 1e-3)
    assert torch.equal(p[0], q[0]) and torch.equal(m[0], q[1])
    p[0].data = torch.zeros(999, device=DEV)
    with pytest.raises(AssertionError, match="another size"):
        b.pacer_adamw(t, g, 3, 1e-3)
