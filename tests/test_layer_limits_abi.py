"""Sizes of the gated scan at the end of what a launch takes (2^32 threads, 512 a tile, whole batch rows): refused beyond it,
before any HIP call is made."""
import ctypes

import pytest

from paper_2607_05583_amd import _lib as L

BASE = 0x7F0000000000  # addresses that are never read: every call here is refused
D = 1 << 21            # 32768 blocks of channels


def at(k):
    return ctypes.c_void_p(BASE + (k << 36))


def rows(k, T):
    return L.Rows(BASE + (k << 36), T * D, D)


def fwd(T):
    return L.lib().resonator_gated_scan_fwd(rows(1, T), rows(2, T), rows(3, T), L.RES_BF16, None, 1, T, D, at(5), None, None, at(6), None,
                                            at(7), 256, None)


def bwd(T):
    return L.lib().resonator_gated_scan_bwd(*(rows(k, T) for k in range(1, 5)), L.RES_BF16, *(rows(k, T) for k in range(5, 8)), 1, T, D,
                                            at(8), at(9), None, None, at(10), None, at(11), 256, None)


@pytest.mark.parametrize("call,steps", [(fwd, 256), (bwd, 128)])
def test_rows_beyond_a_launch(call, steps):
    """256 tiles of 32768 blocks of channels are 2^32 threads; 255 go on to the next check (the workspace is too small)."""
    assert call(255 * steps) == L.RES_ERR_WORKSPACE
    assert call(255 * steps + 1) == L.RES_ERR_UNSUPPORTED and "launch" in L.lib().resonator_last_error().decode()
