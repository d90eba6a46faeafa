"""Calls of the microscaled 4-bit operators without rows: an empty tensor's pointer is
null, and the call is nothing to do (CPU: no entry point reaches a device)."""
import ctypes as C

import pytest

from paper_2605_28803_amd import _lib

OK, SHAPE, ALIGN, ARG = 0, -2, -3, -7


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _activation(lib, M=0, F=64, ld=128, dtype=0, act=0, ldh=0):
    return lib.oq_gated_activation(None, M, F, ld, dtype, act, None, ldh, None, None, None)


@pytest.mark.parametrize("change,status", [
    (dict(), OK),                       # as the binding calls for codes: no H, no stride of it
    (dict(ldh=64), OK), (dict(ldh=3), OK), (dict(F=40, ld=80), OK),
    (dict(F=12, ld=24), SHAPE), (dict(ld=120), SHAPE), (dict(ld=132), ALIGN), (dict(dtype=2), ARG), (dict(act=2), ARG), (dict(M=-1), SHAPE)])
def test_activation(lib, change, status):
    assert _activation(lib, **change) == status


def test_the_others(lib):
    norm = _lib.oq_norm(1, 1e-6, 0.0, None, None)
    assert lib.oq_mx4_quantize(None, 0, 64, 64, 0, 1, None, None, None) == OK
    assert lib.oq_mx4_dequantize(None, None, 0, 64, None, 64, 0, None) == OK
    assert lib.oq_mx4_linear(None, None, 0, None, None, None, 16, 64, None, 16, 0, None) == OK
    assert lib.oq_residual_norm(None, 0, 0, None, 0, 0, 0, 64, None, C.byref(norm), 1.0, None, None, None, 0, 0, None, None, 0, None, 0,
                                None, None, None) == OK
