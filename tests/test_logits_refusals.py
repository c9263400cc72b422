"""What the operators on rows of logits refuse, before any kernel is launched (no GPU is needed: the addresses are not read)."""
import pytest

A, B, X = 0x10000, 0x90000000, 0x20000                  # made-up addresses


@pytest.fixture(scope="module")
def lib():
    from paper_2602_01274_b200 import build
    build.build_lib()
    from paper_2602_01274_b200 import binding
    return binding._lib


def refused(lib, rc, text):
    assert rc == -1 and text in lib.pacer_last_error(None).decode(), (rc, lib.pacer_last_error(None))


LOGITS = [  # changes of (logits, dtype, ld, rows, vocab) and the reason
    (dict(z=None), "logits is null"), (dict(dtype=3), "unknown type"), (dict(dtype=-1), "unknown type"), (dict(ld=99), "ld is less"),
    (dict(ld=1 << 36), "ld out of range"),
    (dict(rows=-1), "rows out of range"), (dict(rows=(1 << 24) + 1), "rows out of range"), (dict(vocab=0), "vocab out of range"),
    (dict(vocab=393217, ld=1 << 22), "vocab out of range"), (dict(z=A + 2), "misaligned logits"),
    (dict(z=A + 1, dtype=1), "misaligned logits"),
]


def rows(z=A, dtype=0, ld=100, rows=4, vocab=100):
    return z, dtype, ld, rows, vocab


@pytest.mark.parametrize("change,text", LOGITS)
def test_rows(lib, change, text):
    r = rows(**change)
    refused(lib, lib.pacer_logprobs(*r, X, 0, X, X, X, None, None, None), text)
    ld = max(change.get("ld", 100), r[4])
    refused(lib, lib.pacer_logprobs_backward(*r, X, X, X, X, None, None, B, ld, None), text)
    refused(lib, lib.pacer_distill(*r, X, X, 0, 4, None, 1.0, X, X, None, None, None, 0, None), text)
    refused(lib, lib.pacer_distill_backward(*r, X, X, 0, 4, None, 1.0, X, None, X, B, ld, None), text)


@pytest.mark.parametrize("tokens,top,logp,text", [
    (X, -1, X, "top out of range"), (X, 101, X, "top out of range"), (X, 129, X, "top out of range"), (None, 0, X, "logp without tokens"),
])
def test_logprobs(lib, tokens, top, logp, text):
    refused(lib, lib.pacer_logprobs(*rows(), tokens, top, logp, X, X, X, X, None), text)
    refused(lib, lib.pacer_logprobs(*rows(ld=500, vocab=500), X, 129, X, X, X, X, X, None), "top out of range")


@pytest.mark.parametrize("change,text", [
    (dict(lse=None), "lse is null"), (dict(gl=None), "no gradient comes in"), (dict(tokens=None), "g_logp without tokens"),
    (dict(gh=X, entropy=None), "g_entropy without entropy"), (dict(dz=None), "dlogits is null"), (dict(ld_dz=99), "ld_dlogits is less"),
    (dict(ld_dz=1 << 36), "ld_dlogits out of range"),
    (dict(dz=B + 2), "misaligned dlogits"), (dict(dz=A + 4), "overlaps"), (dict(dz=A, ld_dz=101), "overlaps"), (dict(dz=A + 1200), "overlaps"),
])
def test_logprobs_backward(lib, change, text):
    a = dict(tokens=X, lse=X, entropy=X, gl=X, gh=None, gs=None, dz=B, ld_dz=100)
    a.update(change)
    refused(lib, lib.pacer_logprobs_backward(*rows(), *a.values(), None), text)


@pytest.mark.parametrize("change,text", [
    (dict(k=0), "k out of range"), (dict(k=257), "k out of range"), (dict(td=3), "unknown type of teacher"), (dict(T=0.0), "temperature"),
    (dict(T=-1.0), "temperature"), (dict(T=float("nan")), "temperature"), (dict(T=float("inf")), "temperature"), (dict(ids=None), "ids or teacher"),
    (dict(t=None), "ids or teacher"),
])
def test_teacher(lib, change, text):
    a = dict(ids=X, t=X, td=0, k=4, tl=None, T=1.0)
    a.update(change)
    refused(lib, lib.pacer_distill(*rows(), *a.values(), X, X, None, None, None, 0, None), text)
    refused(lib, lib.pacer_distill_backward(*rows(), *a.values(), X, None, X, B, 100, None), text)


def test_distill(lib):
    t = (X, X, 0, 4)
    refused(lib, lib.pacer_distill(*rows(), *t, None, 1.0, X, X, X, None, None, 0, None), "tail_lse without teacher_lse")
    refused(lib, lib.pacer_distill(*rows(), *t, None, 1.0, X, X, None, None, B, 100, None), "dlogits without weight")
    refused(lib, lib.pacer_distill(*rows(), *t, None, 1.0, X, X, None, X, B, 99, None), "ld_dlogits is less")
    refused(lib, lib.pacer_distill(*rows(), *t, None, 1.0, X, X, None, X, A + 400, 100, None), "overlaps")
    refused(lib, lib.pacer_distill_backward(*rows(), *t, None, 1.0, None, None, X, B, 100, None), "lse or g_loss is null")
    refused(lib, lib.pacer_distill_backward(*rows(), *t, None, 1.0, X, None, None, B, 100, None), "lse or g_loss is null")
    refused(lib, lib.pacer_distill_backward(*rows(), *t, X, 1.0, X, None, X, B, 100, None), "teacher_lse without tail_lse")


def test_no_rows_is_no_work(lib):
    assert lib.pacer_logprobs(*rows(z=None, rows=0), None, 5, None, None, None, None, None, None) == 0
    assert lib.pacer_logprobs_backward(*rows(z=None, rows=0), None, None, None, None, None, None, None, 100, None) == 0
    assert lib.pacer_distill(*rows(z=None, rows=0), None, None, 0, 4, None, 1.0, None, None, None, None, None, 0, None) == 0
    assert lib.pacer_distill_backward(*rows(z=None, rows=0), None, None, 0, 4, None, 1.0, None, None, None, None, 100, None) == 0


@pytest.mark.parametrize("change,text,code", [
    (dict(rows=-1), "rows out of range", -1), (dict(rows=(1 << 20) + 1), "rows out of range", -1), (dict(vocab=0), "vocab out of range", -1),
    (dict(vocab=(1 << 21) + 1), "vocab out of range", -1), (dict(d=0), "d out of range", -1), (dict(d=12), "d out of range", -1),
    (dict(d=1 << 17), "d out of range", -1), (dict(lh=56), "bad row stride", -1), (dict(lw=68), "bad row stride", -1),
    (dict(h=None), "is null", -1), (dict(w=None), "is null", -1), (dict(s=None), "is null", -1), (dict(h=A + 2), "misaligned", -1),
    (dict(w=A + 8), "misaligned", -1), (dict(s=X + 16), "misaligned", -1), (dict(tok=None), "logp without tokens", -1),
    (dict(short=1), "scratch too small", -2),
])
def test_head_logprobs(lib, change, text, code):
    a = dict(h=A, lh=64, w=B, lw=64, rows=4, vocab=100, d=64, tok=X, s=X, short=0)
    a.update(change)
    need = lib.pacer_head_logprobs_scratch_bytes(4, 100)
    assert need > 0
    rc = lib.pacer_head_logprobs(a["h"], a["lh"], a["w"], a["lw"], a["rows"], a["vocab"], a["d"], a["tok"], None, 0.0, X, X, X, a["s"],
                                 need - a["short"], None)
    assert rc == code and text in lib.pacer_last_error(None).decode()


def test_head_scratch(lib):
    n = lib.pacer_head_logprobs_scratch_bytes
    assert n(0, 100) == n(1, 0) == n((1 << 20) + 1, 100) == n(1, (1 << 21) + 1) == 0
    for rows, vocab in ((1, 1), (1, 32000), (25, 151936), (129, 32003), (2048, 32000)):
        assert n(rows, vocab) >= rows * 4 + rows * 2 * -(-vocab // 256) * 16      # two parts of 16 bytes per tile of at most 256 tokens
    assert lib.pacer_head_logprobs(None, 64, None, 64, 0, 100, 64, None, None, 0.0, None, None, None, None, 0, None) == 0
