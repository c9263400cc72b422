"""What AdamW over many tensors and the gradients' norm refuse, before any kernel is launched (no GPU is needed: the addresses are not read)."""
import ctypes as C

import numpy as np
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2602_01274_b200 import build
    build.build_lib()
    from paper_2602_01274_b200 import binding
    return binding


def table(**change):
    """One row of pacer_adamw_tensor: param, copy, grad, exp_avg, exp_avg_sq, scales, numel, types."""
    a = dict(param=0x10000, copy=0, grad=0x20000, m=0x30000, v=0x40000, scales=0x50000, numel=100, types=0)
    a.update(change)
    return list(a.values())


def call(b, rows, **cfg):
    a = dict(lr=1e-3, beta_one=0.9, beta_two=0.999, eps=1e-8, weight_decay=0.1, step=1, state_bits=32)
    a.update(cfg)
    t = np.array(rows, dtype=np.int64).reshape(-1, 8)
    rc = b._lib.pacer_adamw(t.ctypes.data, len(t), C.byref(b.AdamwCfg(**a)), None)
    return rc, b._lib.pacer_last_error(None).decode()


@pytest.mark.parametrize("change,text", [
    (dict(numel=-1), "numel out of range"), (dict(numel=1 << 40), "numel out of range"), (dict(types=2), "unknown type of param"),
    (dict(types=7), "unknown type of param"), (dict(types=3 << 32), "unknown type of grad"), (dict(param=0), "is null"), (dict(grad=0), "is null"),
    (dict(m=0), "is null"), (dict(v=0), "is null"), (dict(types=1, copy=0x60000), "a copy of a 16-bit param"), (dict(param=0x10002), "misaligned param"),
    (dict(grad=0x20001, types=1 << 32), "misaligned param, copy or grad"), (dict(copy=0x60001), "misaligned"), (dict(m=0x30002), "misaligned states"),
])
def test_tensors(b, change, text):
    rc, said = call(b, [table(**change)])
    assert rc == -1 and text in said
    # among others
    rc, said = call(b, [table(param=0x90000), table(**change)])
    assert rc == -1 and text in said


@pytest.mark.parametrize("change,text", [(dict(scales=0), "a state is null"), (dict(scales=0x50004), "misaligned scales")])
def test_scales(b, change, text):
    rc, said = call(b, [table(**change)], state_bits=8)
    assert rc == -1 and text in said
    t = np.array([table(**change)], dtype=np.int64)
    assert b._lib.pacer_adamw_states(t.ctypes.data, 1, None, None, None) == -1 and text in b._lib.pacer_last_error(None).decode()


@pytest.mark.parametrize("cfg,text", [
    (dict(state_bits=16), "state_bits"), (dict(beta_one=1.0), "a beta outside"), (dict(beta_two=-0.1), "a beta outside"), (dict(beta_one=float("nan")), "a beta outside"),
    (dict(eps=-1.0), "eps, weight_decay or lr"), (dict(eps=float("nan")), "eps"), (dict(lr=float("inf")), "lr"), (dict(weight_decay=float("nan")), "weight_decay"),
    (dict(step=0), "step out of range"), (dict(step=1 << 31), "step out of range"), (dict(max_norm=1.0), "max_norm without norm"),
    (dict(max_norm=float("nan")), "max_norm without norm"),
])
def test_settings(b, cfg, text):
    rc, said = call(b, [table()], **cfg)
    assert rc == -1 and text in said


def test_lists(b):
    assert call(b, [table(), table(m=0x70000, v=0x80000)]) [0] == -1 and "two params overlap" in b._lib.pacer_last_error(None).decode()
    assert call(b, [table(), table(param=0x10000 + 396)])[0] == -1 and "two params overlap" in b._lib.pacer_last_error(None).decode()
    assert b._lib.pacer_adamw(None, 1, C.byref(b.AdamwCfg(state_bits=32, step=1)), None) == -1
    assert b._lib.pacer_adamw(None, 0, None, None) == -1
    assert b._lib.pacer_adamw(None, -1, C.byref(b.AdamwCfg(state_bits=32, step=1)), None) == -1
    # nothing to do
    assert b._lib.pacer_adamw(None, 0, C.byref(b.AdamwCfg(state_bits=32, step=1)), None) == 0
    assert call(b, [table(numel=0, param=0, types=9)])[0] == 0


@pytest.mark.parametrize("row,text", [
    ((0x10000, -1, 0), "numel out of range"), ((0x10000, 5, 3), "unknown type"), ((0, 5, 0), "grad is null"), ((0x10002, 5, 0), "misaligned"), ((0x10001, 5, 1), "misaligned"),
])
def test_norm(b, row, text):
    t = np.array([row], dtype=np.int64)
    need = b._lib.pacer_grad_norm_scratch_bytes(1)
    assert b._lib.pacer_grad_norm(t.ctypes.data, 1, 0x20000, 0x30000, need, None) == -1 and text in b._lib.pacer_last_error(None).decode()


def test_norm_places(b):
    t = np.array([(0x10000, 5, 0)], dtype=np.int64)
    need = b._lib.pacer_grad_norm_scratch_bytes(1)
    assert need > 0 and b._lib.pacer_grad_norm_scratch_bytes(-1) == 0
    f = b._lib.pacer_grad_norm
    assert f(t.ctypes.data, 1, None, 0x30000, need, None) == f(t.ctypes.data, 1, 0x20000, None, need, None) == f(t.ctypes.data, 1, 0x20000, 0x30004, need, None) == -1
    assert f(t.ctypes.data, 1, 0x20000, 0x30000, need - 1, None) == -2
    assert f(None, 1, 0x20000, 0x30000, need, None) == -1


def test_structures_match_the_header(b):
    """Sizes of the structures that the binding fills, from the header's fields."""
    assert C.sizeof(b.AdamwCfg) == 6 * 8 + 2 * 8 + 3 * 8 + 2 * 4
    assert np.zeros((1, 8), dtype=np.int64).nbytes == 6 * 8 + 8 + 2 * 4          # pacer_adamw_tensor
