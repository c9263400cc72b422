"""Codes of second moments that do not exist are refused before any kernel is launched (no GPU is needed: the addresses are not read)."""
import pytest

from tests.test_adamw_refusals import b, call, table  # noqa: F401  (b: the fixture)


@pytest.mark.parametrize("code", [2, -1, 1 << 14])
def test_unknown_codes(b, code):  # noqa: F811
    import numpy as np
    row = table(types=(code & 0xFFFF) << 48 if code >= 0 else -(1 << 48))
    rc, said = call(b, [row], state_bits=8)
    assert rc == -1 and "unknown code of exp_avg_sq" in said
    t = np.array([row], dtype=np.int64)
    assert b._lib.pacer_adamw_states(t.ctypes.data, 1, None, None, None) == -1 and "unknown code" in b._lib.pacer_last_error(None).decode()
