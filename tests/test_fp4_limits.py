"""The sizes that include/nvfp4mm.h says the 4-bit calls take, and the workspace queries beyond them (no GPU needed)."""
import pytest

from paper_2606_07618_gb300 import binding as B

ROWS, COLS = 65535 * 128, 2 ** 30
RANGE = 4


def call(m, n, k, grad):
    """The status of a call whose pointers are all null: what is not refused for its size is for those."""
    if grad:
        return B.lib().fp4_matmul_backward(1, None, None, m, n, k, None, n, None, k, None, k, None, None, 0, None)
    return B.lib().fp4_matmul(1, None, None, m, n, k, None, 0, n, None, None)


def gated(t, f, d, grad):
    if grad:
        return B.lib().fp4_gated_ff_backward(1, 0, None, None, None, t, f, d, None, f, None, d, None, None, d, None, f, None, None,
                                             0, None)
    return B.lib().fp4_gated_ff(1, 0, None, None, None, t, f, d, None, f, None, None, None, None)


@pytest.mark.parametrize("fn", [call, gated])
def test_sizes(fn):
    for grad in (False, True):
        assert RANGE not in (fn(ROWS, 8, 64, grad), fn(4, ROWS, 64, grad), fn(4, 8, ROWS, grad))
        assert fn(ROWS + 1, 8, 64, grad) == RANGE and fn(4, ROWS + 1, 64, grad) == RANGE and fn(4, 8, COLS + 32, grad) == RANGE
    assert fn(4, 8, COLS, False) != RANGE and fn(4, 8, ROWS + 32, True) == RANGE


@pytest.mark.parametrize("query", ["fp4_matmul_backward_workspace", "fp4_gated_ff_backward_workspace"])
def test_no_workspace_for_sizes_that_are_refused(query):
    q = getattr(B, query)
    assert q(4, 8, ROWS) > 0 and q(ROWS, 8, 32) > 0 and q(4, ROWS, 32) > 0
    assert q(4, 8, ROWS + 32) == 0 and q(ROWS + 1, 8, 32) == 0 and q(4, ROWS + 1, 32) == 0
