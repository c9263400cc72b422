"""The optimiser when a program changes its state, loads one, or captures its first step."""
from collections import defaultdict

import pytest
import torch

from tests.test_gpu_adamw import DEV, gen

pytestmark = pytest.mark.gpu
SIZES = (5000, 300, 70000)


def params(dtype=torch.bfloat16):
    return [torch.nn.Parameter(torch.randn(n, generator=gen(n), device=DEV).to(dtype)) for n in SIZES]


def run(opt, ps, ks):
    for k in ks:
        for i, p in enumerate(ps):
            x = torch.randn(p.shape, generator=gen(100 + 10 * k + i), device=DEV).to(p.dtype)
            p.grad = x if p.grad is None else p.grad.copy_(x)
        opt.step()


def clones(ps):
    return [torch.nn.Parameter(p.detach().clone()) for p in ps]


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("capturable", [False, True])
@pytest.mark.parametrize("how", ["clear", "new dict", "pop"])
def test_state_started_anew(states, capturable, how):
    """An optimiser whose state was dropped goes on as a new one does."""
    from paper_2602_01274_b200 import optim
    a = params()
    oa = optim.AdamW(a, lr=1e-3, states=states, seed=4, capturable=capturable)
    run(oa, a, range(3))
    with torch.no_grad():
        for p in a:                                                         # (weights of another place, no longer the masters')
            p.mul_(0.5)
    b = clones(a)
    if how == "clear":
        oa.state.clear()
    elif how == "new dict":
        oa.state = defaultdict(dict)
    else:
        for p in a:
            oa.state.pop(p)
    ob = optim.AdamW(b, lr=1e-3, states=states, seed=4, capturable=capturable)
    run(oa, a, range(3, 6))
    run(ob, b, range(3, 6))
    for p, q in zip(a, b):
        assert torch.equal(p, q)
        assert oa.state[p].keys() == ob.state[q].keys()
        for name in oa.state[p]:
            x, y = oa.state[p][name], ob.state[q][name]
            assert torch.equal(x, y) if torch.is_tensor(x) else x == y, name


@pytest.mark.parametrize("name", ["exp_avg", "exp_avg_sq", "scales", "master"])
def test_entry_of_the_state_exchanged(name):
    """A tensor put into the state is the one that the next steps read and write."""
    from paper_2602_01274_b200 import optim
    a = params()
    oa = optim.AdamW(a, lr=1e-3, states="8bit" if name == "scales" else "f32", seed=4)
    run(oa, a, range(2))
    b = clones(a)
    ob = optim.AdamW(b, lr=1e-3, states="8bit" if name == "scales" else "f32", seed=4)
    ob.load_state_dict(oa.state_dict())
    old = oa.state[a[0]][name]
    for o, ps in ((oa, a), (ob, b)):
        o.state[ps[0]][name] = o.state[ps[0]][name] * 0.5                   # the one after steps, the other before its first
    new, kept, before = oa.state[a[0]][name], old.clone(), oa.state[a[0]][name].clone()
    run(oa, a, range(2, 4))
    run(ob, b, range(2, 4))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert oa.state[a[0]][name] is new and not torch.equal(new, before) and torch.equal(old, kept)
    assert all(torch.equal(oa.state[a[0]][k], ob.state[b[0]][k]) for k in ("exp_avg", "exp_avg_sq", "master"))


def test_first_step_is_not_captured():
    """Its zeroed moments and counts would be part of the graph: every replay would be a first step.  Nor is one whose count is on the host."""
    from paper_2602_01274_b200 import optim
    a = params(torch.float32)
    o = optim.AdamW(a, lr=1e-3, capturable=True)
    for p in a:
        p.grad = torch.ones_like(p)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="after a first one"):
            o.step()
    a[1].grad = None
    o.step()
    assert not o.state.get(a[1]) and int(o.state[a[0]]["step"]) == 1
    a[1].grad = torch.ones_like(a[1])
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="after a first one"):
            o.step()
    o.step()                                                                # and goes on as if nothing had been
    assert [int(o.state[p]["step"]) for p in a] == [2, 1, 2]
    b = params(torch.float32)
    h = optim.AdamW(b, lr=1e-3)
    run(h, b, range(1))
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="capturable"):
            h.step()
    assert h.state[b[0]]["step"] == 1


def test_hooks_of_loading():
    """What a pre-hook returns is what is loaded; a post-hook sees states of their own types."""
    from paper_2602_01274_b200 import optim
    a = params()
    oa = optim.AdamW(a, lr=1e-3, states="8bit", seed=4)
    run(oa, a, range(2))
    saved = oa.state_dict()
    b = clones(a)
    ob = optim.AdamW(b, lr=1e-3, states="8bit", seed=4)
    seen = []

    def nested(_, d):                                                       # (a checkpoint with a level of its own, counts moved on)
        return {**d["optimizer"], "state": {k: {**s, "step": s["step"] + 5} for k, s in d["optimizer"]["state"].items()}}

    ob.register_load_state_dict_pre_hook(nested)
    ob.register_load_state_dict_post_hook(lambda o: seen.extend((o.state[p]["exp_avg"].dtype, o.state[p]["step"]) for p in b))
    ob.load_state_dict({"optimizer": saved, "param_groups": saved["param_groups"], "state": {}})
    assert seen == [(torch.uint8, 7), (torch.float32, 7), (torch.uint8, 7)]
    for p in a:
        oa.state[p]["step"] += 5
    run(oa, a, range(2, 4))
    run(ob, b, range(2, 4))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_states_without_masters():
    """Moments of an optimiser that had none: bf16 parameters go on from their value as masters."""
    from paper_2602_01274_b200 import optim
    a = params()
    theirs = torch.optim.AdamW([torch.nn.Parameter(p.detach().float()) for p in a], lr=1e-3)
    for p, q in zip(a, theirs.param_groups[0]["params"]):
        q.grad = torch.ones_like(q)
    theirs.step()
    o = optim.AdamW(a, lr=1e-6)
    o.load_state_dict(theirs.state_dict())
    for g in o.param_groups:
        g.update(lr=1e-6, weight_decay=0.0)
    start = [p.detach().clone() for p in a]
    for p in a:
        p.grad = torch.ones_like(p)
    for _ in range(3):
        o.step()
    for p, x in zip(a, start):
        m = o.state[p]["master"]
        assert m.dtype == torch.float32 and o.state[p]["step"] == 4
        # (three updates of 1e-6 each, far below a bf16 step: the master holds them)
        assert ((x.float() - m) - 3e-6).abs().max() < 2 * 2.0 ** -24 * float(m.abs().max()) * 3 + 1e-8 and torch.equal(p.detach(), m.to(torch.bfloat16))
    # without masters where none are asked for
    o = optim.AdamW(a, lr=1e-6, master=False)
    o.load_state_dict(theirs.state_dict())
    o.step()
    assert "master" not in o.state[a[0]]


def test_rounding_at_random_unless_nearest_is_asked_for():
    """Second moments in 8 bits whose gradients become smaller: their mean follows that of f32 states (the bound of
    test_gpu_adamw.test_8_bit_second_moments_follow), to nearest it does not."""
    from paper_2602_01274_b200 import binding, optim
    n, means = 1 << 14, {}
    for name, more in (("f32", {}), ("8bit", dict(states="8bit")), ("nearest", dict(states="8bit", seed=None))):
        p = torch.nn.Parameter(torch.zeros(n, device=DEV))
        o = optim.AdamW([p], lr=1e-4, **more)
        g = gen(4)
        for k in range(600):
            p.grad = torch.randn(n, generator=g, device=DEV) * (1.0 if k < 200 else 0.25)
            o.step()
        s = o.state[p]
        v = s["exp_avg_sq"] if name == "f32" else binding.pacer_adamw_states([s["exp_avg"]], [s["exp_avg_sq"]], [s["scales"]], roots=False)[1][0]
        means[name] = float(v.double().mean())
    bound = 6 * (500 / n) ** 0.5 / 16
    assert abs(means["8bit"] / means["f32"] - 1) < bound < abs(means["nearest"] / means["f32"] - 1)


def test_other_strides_in_place():
    """A parameter that was transposed where it lies keeps address and size: its elements are no longer in the order of its moments."""
    from paper_2602_01274_b200 import optim
    p = torch.nn.Parameter(torch.randn(64, 64, generator=gen(1), device=DEV))
    o = optim.AdamW([p], lr=1e-3)
    p.grad = torch.ones_like(p)
    o.step()
    kept = p.detach().clone()
    p.grad = None
    p.data = p.data.t()
    p.grad = torch.ones(64, 64, device=DEV)
    with pytest.raises(RuntimeError, match="contiguous"):
        o.step()
    assert torch.equal(p.detach().t(), kept) and o.state[p]["step"] == 1


def test_a_refused_step_is_not_counted():
    """A state that does not fit stops the step before any parameter of any group has moved or been counted."""
    from paper_2602_01274_b200 import optim
    a = params(torch.float32)
    o = optim.AdamW([dict(params=a[:1]), dict(params=a[1:], lr=1e-4)], lr=1e-3)
    run(o, a, range(2))
    kept, m = [p.detach().clone() for p in a], o.state[a[2]]["exp_avg"]
    o.state[a[2]]["exp_avg"] = m.double()
    with pytest.raises(AssertionError, match="exp_avg"):
        o.step()
    assert [o.state[p]["step"] for p in a] == [2, 2, 2] and all(torch.equal(p.detach(), x) for p, x in zip(a, kept))
    o.state[a[2]]["exp_avg"] = m
    o.step()
    assert [o.state[p]["step"] for p in a] == [3, 3, 3] and not any(torch.equal(p.detach(), x) for p, x in zip(a, kept))
