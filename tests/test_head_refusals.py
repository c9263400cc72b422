"""What the gradients of the fused head refuse, before any kernel is launched (no GPU is needed: the addresses are not read)."""
import pytest

A, B, X, S = 0x10000, 0x90000000, 0x20000, 0x70000000    # made-up addresses
DH, DW = 0xA0000000, 0xB0000000


@pytest.fixture(scope="module")
def lib():
    from paper_2602_01274_b200 import build
    build.build_lib()
    from paper_2602_01274_b200 import binding
    return binding._lib


COMMON = [
    (dict(rows=-1), "rows out of range", -1), (dict(rows=(1 << 20) + 1), "rows out of range", -1), (dict(vocab=0), "vocab out of range", -1),
    (dict(vocab=(1 << 21) + 1), "vocab out of range", -1), (dict(d=0), "d out of range", -1), (dict(d=12), "d out of range", -1),
    (dict(d=1 << 17), "d out of range", -1), (dict(lh=56), "bad row stride", -1), (dict(lw=68), "bad row stride", -1),
    (dict(h=None), "is null", -1), (dict(w=None), "is null", -1), (dict(s=None), "scratch is null", -1), (dict(h=A + 2), "misaligned", -1),
    (dict(w=B + 8), "misaligned", -1), (dict(s=S + 16), "misaligned", -1), (dict(dh=DH + 8), "misaligned gradient", -1),
    (dict(dw=DW + 2), "misaligned gradient", -1), (dict(ldh=56), "bad row stride of a gradient", -1), (dict(ldw=68), "bad row stride of a gradient", -1),
    (dict(dh=A + 16), "overlaps", -1), (dict(dw=B), "overlaps", -1), (dict(dh=DW + 128), "overlaps", -1), (dict(dw=A + 128), "overlaps", -1),
    (dict(short=1), "scratch too small", -2),
]


def args(change):
    a = dict(h=A, lh=64, w=B, lw=64, rows=4, vocab=100, d=64, tok=X, logp=X, lse=X, ent=X, gl=X, gh=None, gs=None, dh=DH, ldh=64, dw=DW, ldw=64,
             s=S, short=0)
    a.update(change)
    return a


@pytest.mark.parametrize("change,text,code", COMMON + [
    (dict(lse=None), "lse is null", -1), (dict(gl=None), "no gradient comes in", -1), (dict(tok=None), "g_logp without tokens", -1),
    (dict(logp=None), "g_logp without tokens or logp", -1), (dict(gh=X, ent=None), "g_entropy without entropy", -1),
    (dict(dh=None, dw=None), "no gradient is asked for", -1),
])
def test_backward(lib, change, text, code):
    a = args(change)
    need = lib.pacer_head_logprobs_backward_scratch_bytes(4, 100, 64)
    assert need > 0
    rc = lib.pacer_head_logprobs_backward(a["h"], a["lh"], a["w"], a["lw"], a["rows"], a["vocab"], a["d"], a["tok"], None, 0.0, a["logp"], a["lse"],
                                          a["ent"], a["gl"], a["gh"], a["gs"], a["dh"], a["ldh"], a["dw"], a["ldw"], a["s"], need - a["short"], None)
    assert rc == code and text in lib.pacer_last_error(None).decode()


@pytest.mark.parametrize("change,text,code", COMMON + [
    (dict(tok=None), "tokens is null", -1), (dict(gl=None), "a gradient without weight", -1),
])
def test_nll(lib, change, text, code):
    a = args(change)
    need = lib.pacer_head_nll_grad_scratch_bytes(4, 100, 64)
    assert need > 0
    rc = lib.pacer_head_nll_grad(a["h"], a["lh"], a["w"], a["lw"], a["rows"], a["vocab"], a["d"], a["tok"], None, 0.0, a["gl"], X, a["dh"], a["ldh"],
                                 a["dw"], a["ldw"], a["s"], need - a["short"], None)
    assert rc == code and text in lib.pacer_last_error(None).decode()


def test_scratch(lib):
    for n in (lib.pacer_head_logprobs_backward_scratch_bytes, lib.pacer_head_nll_grad_scratch_bytes):
        assert n(0, 100, 64) == n(1, 0, 64) == n((1 << 20) + 1, 100, 64) == n(1, (1 << 21) + 1, 64) == n(1, 100, 12) == n(1, 100, 1 << 17) == 0
        for rows, vocab, d in ((1, 1, 8), (1, 32000, 768), (2048, 32003, 4096), (100000, 151936, 1536), (1 << 20, 1 << 21, 64)):
            # dz of a piece of the vocabulary, sums of dhidden in fp32 for at most a few shares
            assert rows * 2 <= n(rows, vocab, d) <= (2 << 30) + (1 << 20) + rows * 512 + 130 * (rows + 256) * d * 4 + rows * 2 * (vocab / 16 + 2) * 16
    assert lib.pacer_head_nll_grad(None, 64, None, 64, 0, 100, 64, None, None, 0.0, None, None, None, 0, None, 0, None, 0, None) == 0
