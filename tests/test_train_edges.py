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


@pytest.mark.parametrize("dtype", [0, 1])
def test_gradients_of_no_rows_are_no_error(lib, dtype):
    """df of no rows has no address; without dE nothing is left to do."""
    c = soma.CrossEntropyConfig(0, 100, 64, dtype, 64, 64)
    need, ws = ctypes.c_size_t(), ctypes.c_void_p(0x100000)
    assert lib.soma_ce_workspace_size(ctypes.byref(c), 1, ctypes.byref(need)) == soma.SOMA_OK
    assert lib.soma_ce_grad(ctypes.byref(c), None, ctypes.c_void_p(0x200000), None, None, None, None, None, ws, need.value,
                            None) == soma.SOMA_OK
