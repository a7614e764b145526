"""How many rows one call of include/pda_lm.h takes, as its header says (no GPU needed: a NULL pointer ends the calls that are
within the limits)."""

import pytest

from paper_2605_20863_amd import _lib as L
from tests import test_lm_abi as A

ROWS = 1 << 22


def error(rc):
    assert rc == L.EINVAL
    return L.last_error()


@pytest.mark.parametrize("width", [8, 8192, 8200, 16384, 32768])
@pytest.mark.parametrize("out", [L.F32, L.BF16, L.FP8_E4M3])
def test_rows_of_a_norm(width, out):
    """A launch has below 2^32 threads, of which a row above a width of 8,192 takes 1,024."""
    most = ROWS - (width > 8192)
    more = dict(x=None, scales=A.P if out == L.FP8_E4M3 else None)
    assert error(A.forward(A.norm(num_tokens=most, width=width, out_dtype=out), **more)) == "x is NULL"
    assert "num_tokens" in error(A.forward(A.norm(num_tokens=most + 1, width=width, out_dtype=out), **more))
    assert error(A.backward(A.norm(num_tokens=ROWS, width=width), h=None)) == "h is NULL"
    assert "num_tokens" in error(A.backward(A.norm(num_tokens=ROWS + 1, width=width), h=None))


def test_rows_of_logits():
    assert error(A.top(A.logits(num_tokens=ROWS), z=None)) == "logits is NULL"
    assert error(A.top(A.logits(num_tokens=ROWS + 1), 8)) and "num_tokens" in L.last_error()
    assert error(A.distill(A.logits(num_tokens=ROWS // 4), A.options(), z=None)) == "logits is NULL"
    assert error(A.distill(A.logits(num_tokens=ROWS // 4 + 1), A.options())) and "num_tokens" in L.last_error()
