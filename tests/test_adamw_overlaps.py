"""What an AdamW step writes must not overlap what else it reads or writes (tensors are stepped side by side): each such call is
refused before any HIP call is made."""
import ctypes

import pytest

from paper_2607_05583_amd import _lib as L

BASE = 0x7F0000000000  # addresses that are never read: every call here is refused


def at(k, off=0):
    return BASE + (k << 32) + off


def step(tensors, state, out=None, bits=32, scale=None):
    table = (L.AdamWTensor * len(tensors))(*(L.AdamWTensor(*t) for t in tensors))
    a = L.AdamWState(bits, *state)
    b = a if out is None else L.AdamWState(bits, *out)
    return L.lib().resonator_adamw_step(table, len(tensors), L.RES_F32, L.RES_F32, ctypes.byref(a), ctypes.byref(b), 0.1, 0.9, 0.99,
                                        1e-8, 0.0, 1, None if scale is None else ctypes.c_void_p(scale), None)


N = 1000  # elements of a tensor: 4000 bytes, four blocks
ST = (at(10), at(11), None, None, None)
ST8 = (at(10), at(11), at(12), at(13), None)


@pytest.mark.parametrize("name,tensors,state,out,bits,scale", [
    ("a tensor twice", [(at(1), at(2), at(1), N, 0), (at(1), at(3), at(1), N, 1024)], ST, None, 32, None),
    ("the second from the middle of the first", [(at(1), at(2), at(1), N, 0), (at(1, 2000), at(3), at(1, 2000), N, 1024)], ST, None, 32, None),
    ("the first from the middle of the second", [(at(1, 3996), at(2), at(1, 3996), N, 0), (at(1), at(3), at(1), N, 1024)], ST, None, 32, None),
    ("new values twice", [(at(1), at(2), at(5), N, 0), (at(3), at(4), at(5), N, 1024)], ST, None, 32, None),
    ("over another tensor's gradient", [(at(1), at(2), at(1), N, 0), (at(3), at(1, 4), at(3), N, 1024)], ST, None, 32, None),
    ("over another tensor's old values", [(at(1), at(2), at(3), N, 0), (at(3), at(4), at(5), N, 1024)], ST, None, 32, None),
    ("the same state", [(at(1), at(2), at(1), N, 0), (at(3), at(4), at(3), N, 0)], ST, None, 32, None),
    ("states that meet", [(at(1), at(2), at(1), N, 768), (at(3), at(4), at(3), N, 0)], ST, None, 32, None),
    ("m is v", [(at(1), at(2), at(1), N, 0)], (at(10), at(10), None, None, None), None, 32, None),
    ("m meets v", [(at(1), at(2), at(1), N, 0)], (at(10), at(10, 3984), None, None, None), None, 32, None),
    ("new m over old v", [(at(1), at(2), at(1), N, 0)], ST, (at(11), at(14), None, None, None), 32, None),
    ("new m from the middle of old m", [(at(1), at(2), at(1), N, 0)], ST, (at(10, 16), at(14), None, None, None), 32, None),
    ("m over a parameter", [(at(1), at(2), at(1), N, 0)], (at(1, -16), at(11), None, None, None), None, 32, None),
    ("a gradient in v", [(at(1), at(11, 64), at(1), N, 0)], ST, None, 32, None),
    ("scales of one kind", [(at(1), at(2), at(1), N, 0)], (at(10), at(11), at(12), at(12), None), None, 8, None),
    ("a scale among the codes", [(at(1), at(2), at(1), N, 0)], (at(10), at(11), at(10, 996), at(13), None), None, 8, None),
    ("the gradients' factor in m", [(at(1), at(2), at(1), N, 0)], ST, None, 32, at(10, 4)),
    ("the gradients' factor in a parameter", [(at(1), at(2), at(1), N, 0)], ST8, None, 8, at(1, 3996)),
])
def test_overlaps(name, tensors, state, out, bits, scale):
    assert step(tensors, state, out, bits, scale) == L.RES_ERR_INVALID_ARG, name
    assert "overlap" in L.lib().resonator_last_error().decode()


def test_many_tensors_one_of_them_twice():
    """Found wherever it stands among the others."""
    for k in (0, 7, 98):
        t = [(at(1, 4000 * ((37 * j) % 100)), at(2), at(1, 4000 * ((37 * j) % 100)), N, 1024 * j) for j in range(100)]
        t[k + 1] = t[k][:4] + (1024 * (k + 1),)
        assert step(t, ST) == L.RES_ERR_INVALID_ARG


@pytest.mark.parametrize("m,v,scale_m,scale_v,code", [
    (at(1), at(2), at(1, 512), at(13), L.RES_ERR_INVALID_ARG), (at(1), at(2), at(12), at(1, 1020), L.RES_ERR_INVALID_ARG),
    (at(1), at(2), at(2, 4), at(13), L.RES_ERR_INVALID_ARG), (at(1), at(2), at(12), at(2), L.RES_ERR_INVALID_ARG),
    (at(10, 240), at(2), at(12), at(13), L.RES_ERR_INVALID_ARG), (at(1), at(11), at(12), at(13), L.RES_ERR_INVALID_ARG),
    (at(1), at(2), at(12, 2), at(13), L.RES_ERR_MISALIGNED), (at(1), at(2), at(12), at(13, 1), L.RES_ERR_MISALIGNED)])
def test_values_over_what_they_are_read_from(m, v, scale_m, scale_v, code):
    """The values of 256 codes, over the codes or one of their scales, and scales that are not aligned."""
    s = L.AdamWState(8, at(10), at(11), scale_m, scale_v, None)
    assert L.lib().resonator_adamw_values(ctypes.byref(s), 256, ctypes.c_void_p(m), ctypes.c_void_p(v), None) == code
