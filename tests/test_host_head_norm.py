"""Refusals of normalised and turned heads that need no device, and the angles' whole numbers."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2502_00021_amd import pxr


@pytest.mark.parametrize("change,code", [
    (dict(d_head=0), "INVALID_ARG"), (dict(d_rotary=5), "INVALID_ARG"), (dict(d_rotary=10), "INVALID_ARG"), (dict(d_head=257), "UNSUPPORTED"), (dict(frequencies=None), "INVALID_ARG"),
    (dict(f=[1.0, float("nan")]), "INVALID_ARG"), (dict(f=[float("inf"), 1.0]), "INVALID_ARG"), (dict(f=[1.0, 2.0 ** 21]), "INVALID_ARG"), (dict(eps=-1.0), "INVALID_ARG"),
    (dict(eps=float("nan")), "INVALID_ARG"), (dict(eps=float("inf")), "INVALID_ARG")])
def test_descriptions(change, code):
    f = np.float64(change.pop("f", [1.0, 0.5]))
    d = pxr.HeadNormDesc(8, 4, f.ctypes.data, 1e-6)
    for name, value in change.items():
        setattr(d, name, value)
    h = C.c_void_p()
    assert pxr.lib().pxr_head_norm_create(C.byref(d), C.byref(h)) == getattr(pxr, "ERR_" + code)
    assert not h.value


def test_without_a_layer():
    L = pxr.lib()
    r, v, n = pxr.Heads(), C.byref(pxr.Tokens()), C.c_size_t()
    assert L.pxr_head_norm_create(None, C.byref(C.c_void_p())) == pxr.ERR_INVALID_ARG
    assert L.pxr_head_norm_create(C.byref(pxr.HeadNormDesc(8, 0, None, 0.0)), None) == pxr.ERR_INVALID_ARG
    assert L.pxr_head_norm_destroy(None) == pxr.OK
    assert L.pxr_head_norm_forward(None, C.byref(r), v, v, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_head_norm_workspace(None, C.byref(r), C.byref(n)) == pxr.ERR_INVALID_ARG
    assert L.pxr_head_norm_backward(None, C.byref(r), v, v, v, v, None, None, None, 0, None) == pxr.ERR_INVALID_ARG


def _turns(f):
    """f / 2 pi modulo 1 as the library forms it: pxr::turns_of, by its mangled name."""
    fn = pxr.lib()._ZN3pxr8turns_ofEd
    fn.argtypes, fn.restype = [C.c_double], C.c_uint64
    return fn(f)


def test_angles_of_far_positions():
    """frequency x position in turns, modulo whole ones, against whole numbers of 200 bits."""
    two_pi = 6283185307179586476925286766559005768394338798750211641949889184615632812572417997256069650684234135964296173026564613294187689219101164463450718816256962
    digits = 10 ** (len(str(two_pi)) - 1)
    rng = np.random.default_rng(0)
    for f in [1.0, 0.5, 10000.0 ** -0.3, -0.7, 0.0, 1e-9, 2.0 ** 20, 2 * math.pi, *rng.standard_normal(20)]:
        num, den = float(f).as_integer_ratio()
        want = num * 2 ** 200 * digits // (den * two_pi)  # turns in fractions of 2^200
        got = _turns(float(f))
        for position in (1, 2, 3, 1000, 2 ** 20 + 1, 2 ** 31 - 1, -1, -2 ** 31):
            off = ((got * position) % 2 ** 64 * 2 ** 136 - want * position) % 2 ** 200
            off = min(off, 2 ** 200 - off) / 2 ** 200
            # f in turns has a rounding of 2^-64 of its size (long double) or of one turn, whichever is more
            assert off <= abs(position) * 2.0 ** -63 * max(1.0, abs(f)), (f, position)


def test_turns_are_rounded_once():
    """Of any frequency that a layer takes, and whatever its size: frequency / 2 pi as the nearest fraction of 2^64 (or, where two are within 2^-31 of as near, either), so that an angle keeps 2^-22 turns up to positions of 2^31
    (2^-34 of its fraction, 2^-32 of the fraction's upper half, the rest of fp32)."""
    two_pi = 6283185307179586476925286766559005768394338798750211641949889184615632812572417997256069650684234135964296173026564613294187689219101164463450718816256962
    digits = 10 ** (len(str(two_pi)) - 1)
    rng = np.random.default_rng(1)
    some = [1000003.7, 2.0 ** 20, 1e6, 16384.0, 2 * math.pi, 40 * math.pi, 1.0, 1e-9, 1e-30, 5e-324, 0.0, -0.0, *(2.0 ** rng.uniform(-70, 20, 200)), *(rng.integers(1, 2 ** 20, 50) + 0.0)]
    for f in [s * float(x) for x in some for s in (1, -1)]:
        num, den = f.as_integer_ratio()
        off = (_turns(f) * 2 ** 136 - num * 2 ** 200 * digits // (den * two_pi)) % 2 ** 200
        assert min(off, 2 ** 200 - off) <= 2 ** 135 * (1 + 2.0 ** -30), f
