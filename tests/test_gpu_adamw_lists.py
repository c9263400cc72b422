"""AdamW called with lists of tensors, and second moments in 8 bits by their roots: codes against a 32-bit evaluation of the formulas rounded operation by
operation (equal bits), values against the codes' definition, parameters against the formulas in 64 bits.

Tolerance of a parameter: as in test_gpu_adamw (16 half steps of the update, 4 of the parameter); a second moment out of its root has one more
rounding, half a step of v, a quarter of one of the update."""
import pytest
import torch

from tests.test_gpu_adamw import DEV, F32, HYPER, SIZES, gen, make, random_bits, step64

pytestmark = pytest.mark.gpu


def values(m, v, s):
    """What codes stand for, from their definition, in 64 bits: m, and the root of v."""
    k = torch.arange(len(m), device=DEV) // 256
    c = m.long()
    e, x = (c >> 3) & 15, (c & 7).double() / 8
    vm = torch.where(e == 0, x * 2.0 ** -6, (1 + x) * torch.exp2(e.double() - 7)) * (1 - 2 * (c >> 7)) * s[k, 0].double()
    c = v.long()
    e, x = c >> 4, (c & 15).double() / 16
    return vm, torch.where(e == 0, x * 2.0 ** -6, (1 + x) * torch.exp2(e.double() - 7)) * s[k, 1].double()


def encode(x, dither, mantissa, top):
    """Codes of |x| and scales by f32 operations rounded one by one: the grid's floor after the dither."""
    n, low = len(x), -6
    if not n:
        return x.to(torch.uint8), torch.zeros(0, device=DEV)
    peak = torch.nn.functional.pad(x.abs(), (0, -n % 256)).view(-1, 256).max(1).values
    some = peak > 1e-30
    inv = torch.where(some, torch.full_like(peak, top) / peak, 0.0)
    scale = torch.where(some, peak * (1.0 / top), 0.0)
    u = (x.abs() * inv.repeat_interleave(256)[:n]).double()
    least = 2.0 ** (low - 23)                                               # (what is smaller has no f32 bits behind it)
    u = torch.where(u < 2.0 ** low, torch.round(u / least) * least, u)
    step = torch.exp2(torch.floor(torch.log2(u.clamp(min=2.0 ** low))) - mantissa)
    q = (torch.floor(u / step + (0.5 if dither is None else dither.double() / 65536)) * step).clamp(max=top)
    e, f = torch.floor(torch.log2(q.clamp(min=2.0 ** low))), 2 ** mantissa
    code = torch.where(q < 2.0 ** low, q / 2.0 ** (low - mantissa), (e - low + 1) * f + (q / torch.exp2(e) - 1) * f).round().long()
    return code, scale


@pytest.mark.parametrize("ptype,gtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("seed", [None, (5 << 32) + 3])
@pytest.mark.parametrize("lists", [True, False])
def test_roots(ptype, gtype, shift, seed, lists):
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, s, _ = make(SIZES, ptype, gtype, 8, 2, False, shift)
    for x in s:
        x *= torch.tensor([1.0, 1e4], device=DEV)                           # (roots of what the second moments' scales were)
    kept = b.AdamwTensors(p, m, v, s, roots=True)
    got_m, got_v = b.pacer_adamw_states(m, v, s) if lists else b.pacer_adamw_states(kept)
    for i in range(len(SIZES)):
        wm, wr = values(m[i], v[i], s[i])
        assert torch.equal(got_m[i], wm.float()) and torch.equal(got_v[i], wr.float() * wr.float())
    old_p, before = [x.clone() for x in p], [(a.clone(), c.clone()) for a, c in zip(got_m, got_v)]
    if lists:
        b.pacer_adamw(p, g, m, v, 9, scales=s, seed=seed, **HYPER)
    else:
        b.pacer_adamw(kept, g, 9, seed=seed, **HYPER)
    for i, n in enumerate(SIZES):
        x = g[i].float()
        nm = before[i][0] * 0.9 + x * (1 - 0.9)
        nr = (before[i][1] * 0.999 + (x * x) * (1 - 0.999)).sqrt()
        rm, rv, _ = random_bits(n, seed, 9, i) if seed is not None else (None, None, None)
        code, scale = encode(nm, rm, 3, 480.0)
        assert torch.equal(m[i], torch.where(nm < 0, code + 128, code).to(torch.uint8)) and torch.equal(s[i][:, 0], scale), (i, n)
        code, scale = encode(nr, rv, 4, 496.0)
        assert torch.equal(v[i], torch.where(nr > 0, code.clamp(min=1), code).to(torch.uint8)) and torch.equal(s[i][:, 1], scale), (i, n)
        want, wm, wv, up = step64(old_p[i].double(), x.double(), before[i][0].double(), before[i][1].double(), *[HYPER[k] for k in ("lr", "betas", "eps", "weight_decay")], 9)
        off = 16 * F32 * up.abs() + 8 * F32 * (before[i][0].abs() + x.abs()).double() * torch.where(wm != 0, up / wm, 0.0).abs() + 4 * F32 * old_p[i].double().abs()
        half = 0.0 if ptype == "f32" else 2.0 ** -8 if seed is None else 2.0 ** -7
        assert ((p[i].double() - want).abs() <= off + half * 1.01 * want.abs() + 1e-38).all()


def test_roots_of_zero_tiny_and_not_finite_moments():
    from paper_2602_01274_b200 import binding as b
    p, g = torch.ones(1024, device=DEV), torch.zeros(1024, device=DEV)
    g[256], g[300], g[512], g[600] = 1.0, 1e-7, 1e-29, float("nan")
    m, v, s = torch.zeros(1024, dtype=torch.uint8, device=DEV), torch.zeros(1024, dtype=torch.uint8, device=DEV), torch.zeros(4, 2, device=DEV)
    b.pacer_adamw([p], [g], [m], [v], 1, 1e-3, weight_decay=0.0, scales=[s], seed=1)
    r = b.pacer_adamw_states([m], [v], [s])[1][0]
    assert (r[:256] == 0).all() and (p[:256] == 1).all()                   # no gradient: nothing is held, nothing moves
    assert v[256] == 255 and v[300] == 1 and (v[257:300] == 0).all()       # the largest gets the largest code, what is above 0 stays so
    bad = ~torch.isfinite(r)
    assert bad[600] and not bad[:512].any() and not bad[768:].any() and int((~torch.isfinite(p)).sum()) == 1


@pytest.mark.parametrize("ptype,master", [("f32", False), ("bf16", False), ("bf16", True)])
def test_lists_are_the_same_step(ptype, master):
    """With 32-bit states, with copies, clipped, codes of the moments themselves: the bits that AdamwTensors give."""
    from paper_2602_01274_b200 import binding as b
    for bits, clip in ((32, True), (32, False), (8, True)):
        one, two = (make(SIZES, ptype, "bf16", bits, 3, master) for _ in range(2))
        norm = b.pacer_grad_norm(one[1]) if clip else None
        p, g, m, v, s, c = one
        b.pacer_adamw(b.AdamwTensors(p, m, v, s, c), g, 4, 1e-3, (0.8, 0.99), 1e-8, 0.01, 5, norm, 0.3 if clip else 0.0)
        p, g, m, v, s, c = two
        versions = [x._version for x in (*p, *m, *v, *(s or []), *(c or []))]
        # (no norm: max_norm has nothing to scale by)
        b.pacer_adamw(p, iter(g), m, v, 4, 1e-3, (0.8, 0.99), 1e-8, 0.01, scales=s, copies=c, seed=5, norm=norm, max_norm=0.3, roots=False)
        assert all(x._version > y for x, y in zip((*p, *m, *v, *(s or []), *(c or [])), versions))
        assert all(torch.equal(x, y) for a, d in zip(one, two) if a is not None for x, y in zip(a, d))


def test_codes_mixed_in_a_table():
    """Rows of one table that differ in the code of exp_avg_sq, and their values read back in one call."""
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, s, _ = make([700, 4096, 31], "f32", "f32", 8, 4)
    q = [[x.clone() for x in y] for y in (p, m, v, s)]
    t = b.AdamwTensors(p, m, v, s)
    t.with_grads(g)
    t.table[1, 7] |= 1 << 48
    cfg = b.AdamwCfg(lr=1e-3, beta_one=0.9, beta_two=0.999, eps=1e-8, weight_decay=0.01, step=2, state_bits=8, seeded=0)
    b._call(b._lib.pacer_adamw, t, t._address, 3, b.C.byref(cfg))
    for i, roots in enumerate((False, True, False)):
        a, c, d, e = ([x[i]] for x in q)
        b.pacer_adamw(a, [g[i]], c, d, 2, 1e-3, scales=e, roots=roots)
        assert torch.equal(a[0], p[i]) and torch.equal(c[0], m[i]) and torch.equal(d[0], v[i]) and torch.equal(e[0], s[i])
    got = b.pacer_adamw_states(t)
    for i, roots in enumerate((False, True, False)):
        want = b.pacer_adamw_states([m[i]], [v[i]], [s[i]], roots=roots)
        assert torch.equal(got[0][i], want[0][0]) and torch.equal(got[1][i], want[1][0])


def test_refusals():
    from paper_2602_01274_b200 import binding as b
    p, g, m, v, s, _ = make([300, 50], "f32", "f32", 8, 8)
    f = [torch.zeros_like(x) for x in p]
    for bad in (lambda: b.pacer_adamw(p, g, m, v, 1, 1e-3), lambda: b.pacer_adamw(p, g, m, v[:1], 1, 1e-3, scales=s), lambda: b.pacer_adamw(p, g, f, f, 1, 1e-3, scales=s),
                lambda: b.pacer_adamw(p, g, m, v, 1, 1e-3, scales=[x[:1] for x in s]), lambda: b.pacer_adamw(p, g[:1], m, v, 1, 1e-3, scales=s),
                lambda: b.pacer_adamw([x.cpu() for x in p], g, m, v, 1, 1e-3, scales=s), lambda: b.pacer_adamw(p, g, m, [x.cpu() for x in v], 1, 1e-3, scales=s),
                lambda: b.pacer_adamw(p, g, f, [torch.zeros(600, device=DEV)[::2], f[1]], 1, 1e-3), lambda: b.pacer_adamw(p, g, f, f, 1, 1e-3, copies=f),
                lambda: b.pacer_adamw_states(m, v[:1], s), lambda: b.pacer_adamw_states(m, f, s), lambda: b.pacer_adamw_states(m, v, f),
                lambda: b.pacer_adamw_states([x.cpu() for x in m], [x.cpu() for x in v], [x.cpu() for x in s]),
                lambda: b.pacer_adamw_states(m, v, s, out=(f, f[:1]))):
        with pytest.raises(AssertionError):
            bad()
    b.pacer_adamw([], [], [], [], 1, 1e-3)
    assert b.pacer_adamw_states([], [], []) == ([], [])
