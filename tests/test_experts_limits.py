"""The largest sizes the experts' entry points take: what is beyond them is an argument error, before any device is asked for (no GPU here)."""
import ctypes

import pytest

from paper_2607_06202_b200 import binding as B
from paper_2607_06202_b200 import build as libbuild


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return B.load()


P = 1 << 20      # an address that is never followed
MOST = 1 << 20   # features


def _codes(lib, wide, narrow, ranks=1, cap=64, gated=True):
    """The codes of the four calls on a device that does not exist."""
    r = ctypes.byref(B.ubep_expert_rows_t(P, P, 8 * ranks, ranks, cap, 1 << 20, None))
    got = [lib.ubep_expert_linear(r, P, P, None, None, None, wide, narrow, 0, P, None, None),
           lib.ubep_expert_linear_backward(r, P, P, None, None, P, wide, narrow, 0, None, P, P, None, None, None, None)]
    if gated:
        got += [lib.ubep_expert_gated(r, P, None, P, wide, narrow, 1, P, None, None, None),
                lib.ubep_expert_gated_backward(r, P, None, P, P, P, wide, narrow, 1, P, P, P, None, None)]
    return set(got)


def test_an_expert_s_weights(lib):
    # (taken: the call goes on and finds no such device)
    assert _codes(lib, MOST, (1 << 18) - 8) == {B.UBEP_ERR_CUDA}
    assert _codes(lib, MOST, 1 << 18) == {B.UBEP_ERR_ARG, B.UBEP_ERR_CUDA}             # 2^40 bytes in two matrices, half of it in one
    assert _codes(lib, MOST, (1 << 19) - 8, gated=False) == {B.UBEP_ERR_CUDA}
    assert _codes(lib, MOST, 1 << 19) == {B.UBEP_ERR_ARG}
    assert _codes(lib, MOST, MOST) == {B.UBEP_ERR_ARG}
    assert _codes(lib, MOST + 8, 8) == _codes(lib, 8, MOST + 8) == {B.UBEP_ERR_ARG}


def test_all_rows_of_an_array(lib):
    assert _codes(lib, 1 << 19, 8, ranks=2, cap=1 << 18) == {B.UBEP_ERR_CUDA}
    assert _codes(lib, MOST, 8, ranks=2, cap=1 << 18) == {B.UBEP_ERR_ARG}
    assert _codes(lib, 8, 1 << 18, ranks=2, cap=1 << 19) == {B.UBEP_ERR_ARG, B.UBEP_ERR_CUDA}   # saved products of both matrices
    assert _codes(lib, 8, MOST, ranks=1, cap=1 << 20) == {B.UBEP_ERR_ARG}
