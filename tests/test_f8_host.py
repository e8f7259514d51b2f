"""Refusals of the 8-bit floating-point calls that need no GPU: they come before anything is launched."""
import ctypes

import pytest

from paper_1806_08342_b200 import build as qbuild

INVALID = -1


@pytest.fixture(scope="module")
def lib():
    qbuild.build()
    from paper_1806_08342_b200 import qtz
    return qtz.load_library()


def test_calls_without_a_handle_or_a_plan(lib):
    one = 4096                                                           # never read
    assert lib.qtz_f8_rmsnorm(None, one, 128, None, 0, one, 1e-6, 1, 128, 16, None, 0, None, 0, one, 128, one, 1, None) == INVALID
    assert lib.qtz_f8_quantize(None, one, 128, None, 0, 1, 128, 16, one, 128, one, 1, None) == INVALID
    assert lib.qtz_f8_quantize_weights(None, one, 128, 128, 128, 16, one, one, None) == INVALID
    plan = ctypes.c_void_p(7)
    assert lib.qtz_f8_linear_create(None, 128, 128, one, 128, one, None, 16, ctypes.byref(plan), None) == INVALID and not plan.value
    assert lib.qtz_f8_linear_create(None, 128, 128, one, 128, one, None, 16, None, None) == INVALID
    assert lib.qtz_f8_linear(None, one, 128, one, 1, 1, 1, one, 128, 16, None) == INVALID
    assert lib.qtz_f8_linear_destroy(None) == INVALID
