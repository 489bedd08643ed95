"""Calls of the operators of first-order training at the ends of their ranges, as far as the host decides them (no GPU
needed: what passes the checks here has no array to touch)."""
import ctypes
import os

import pytest

from paper_2609_37899_amd import soma


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(soma.LIB_PATH):
        from paper_2609_37899_amd import build
        build.build()
    return soma.load()


def passed(rc):
    """Past the checks: done, or nothing to run it on."""
    return rc in (soma.SOMA_OK, soma.SOMA_EDEVICE)


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_scan_of_no_rows_is_no_error(lib, dtype):
    """Arrays of no rows have no address."""
    c = soma.ScanConfig(0, 64, 3, dtype, 256)
    assert passed(lib.soma_scan_forward(ctypes.byref(c), None, None, None, None, None, None, None, 0, None))
    assert passed(lib.soma_scan_backward(ctypes.byref(c), None, None, None, None, None, None, None, None, None, 0, None))
