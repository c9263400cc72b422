"""A bias that would leave a row of a vocabulary of one no token is refused (no GPU is needed: the addresses are not read)."""
import math

import pytest

from tests.test_head_refusals import A, B, DH, DW, S, X, lib  # noqa: F401  (lib: the fixture)


@pytest.mark.parametrize("bias", [-math.inf, -3.4028234e38, -1e30])
def test_no_token_left(lib, bias):  # noqa: F811
    big = 1 << 40
    said = lambda: lib.pacer_last_error(None).decode()
    assert lib.pacer_head_logprobs(A, 64, B, 64, 4, 1, 64, X, X, bias, X, X, X, S, big, None) == -1 and "no token" in said()
    assert lib.pacer_head_logprobs_backward(A, 64, B, 64, 4, 1, 64, X, X, bias, X, X, X, X, None, None, DH, 64, DW, 64, S, big, None) == -1 and "no token" in said()
    assert lib.pacer_head_nll_grad(A, 64, B, 64, 4, 1, 64, X, X, bias, X, X, DH, 64, DW, 64, S, big, None) == -1 and "no token" in said()
    # (with two tokens, without ids and with another bias the next thing is looked at: the scratch)
    for vocab, ids, other in ((2, X, bias), (1, None, bias), (1, X, 8.0)):
        assert lib.pacer_head_logprobs(A, 64, B, 64, 4, vocab, 64, X, ids, other, X, X, X, S, 0, None) == -2
        assert lib.pacer_head_nll_grad(A, 64, B, 64, 4, vocab, 64, X, ids, other, X, X, DH, 64, DW, 64, S, 0, None) == -2
