"""Refusals of a learner's update that need no device."""
import ctypes as C

import numpy as np
import pytest

from paper_2502_00021_amd import pxr

QUINTIC = (3.4445, -4.7750, 2.0315)


def _call(workspace=1 << 60, buffers=(64, 64, 64), coefficients=(QUINTIC,) * 5, **change):
    c = np.ascontiguousarray(coefficients, np.float32)
    d = pxr.OrthogonaliseDesc(0, 1, 8, 16, 0, 16, 0, 16, len(c), c.ctypes.data, 1e-7)
    for name, value in change.items():
        setattr(d, name, value)
    n = C.c_size_t()
    return (pxr.lib().pxr_orthogonalise_workspace(C.byref(d), C.byref(n)), pxr.lib().pxr_orthogonalise(C.byref(d), *buffers, workspace, None), n.value)


@pytest.mark.parametrize("change", [
    dict(dtype=2), dict(rows=0), dict(cols=0), dict(n_matrices=65536), dict(n_steps=0), dict(n_steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(x_row=15), dict(out_row=15), dict(out_row=-16), dict(out_row=2 ** 62), dict(coefficients=None, n_steps=1), dict(n_matrices=2, out_matrix=127), dict(n_matrices=2, out_matrix=-127),
    dict(coefficients=[(float("nan"), 0, 0)]), dict(coefficients=[(0, float("inf"), 0)]), dict(coefficients=[(0, 0, -float("inf"))]),
    dict(coefficients=[(2.0 ** 21, 0, 0)]), dict(coefficients=[(1e4, 0, 0)] * 2), dict(coefficients=[(100, 0, 0)] * 10), dict(coefficients=[(0, 0, 1e30)]),
    # small values grow by 10^13, the largest one stays: 10^13 (t - t^3)
    dict(coefficients=[(1e13, -1e13, 0)])])
def test_descriptions(change):
    null = change.get("coefficients", 0) is None
    if null:
        d = pxr.OrthogonaliseDesc(0, 1, 8, 16, 0, 16, 0, 16, 1, None, 1e-7)
        assert pxr.lib().pxr_orthogonalise(C.byref(d), 64, 64, 64, 1 << 60, None) == pxr.ERR_INVALID_ARG
        assert pxr.lib().pxr_orthogonalise_workspace(C.byref(d), C.byref(C.c_size_t())) == pxr.ERR_INVALID_ARG
        return
    assert _call(**change)[:2] == (pxr.ERR_INVALID_ARG, pxr.ERR_INVALID_ARG)
    assert pxr.lib().pxr_last_error()


@pytest.mark.parametrize("change", [dict(rows=2 ** 15 + 1, cols=2 ** 15 + 1), dict(rows=2 ** 31, cols=4), dict(rows=2, cols=2 ** 32 - 1), dict(rows=2 ** 28 + 1, cols=1)])
def test_sizes(change):
    row = dict(x_row=change["cols"], out_row=change["cols"])
    assert _call(**change, **row)[:2] == (pxr.ERR_UNSUPPORTED, pxr.ERR_UNSUPPORTED)


def test_buffers():
    assert pxr.lib().pxr_orthogonalise(None, 64, 64, 64, 1 << 60, None) == pxr.ERR_INVALID_ARG
    assert pxr.lib().pxr_orthogonalise_workspace(None, C.byref(C.c_size_t())) == pxr.ERR_INVALID_ARG
    for i in range(3):
        for bad in (None, 66 if i < 2 else 72):
            b = [64, 64, 64]
            b[i] = bad
            if i < 2:
                assert _call(buffers=b)[1] == pxr.ERR_INVALID_ARG, (i, bad)
            large = dict(rows=300, cols=400, x_row=400, out_row=400)
            assert _call(buffers=b, **large)[1] == pxr.ERR_INVALID_ARG, (i, bad)
    need = _call(**large)[2]
    assert need > 0 and _call(workspace=need - 1, **large)[1] == pxr.ERR_INVALID_ARG
    assert _call(n_matrices=0, buffers=(None, None, None), workspace=0) == (pxr.OK, pxr.OK, 0)  # nothing to do


def test_bounds_of_singular_values():
    """pxr::orthogonalise_bounds, by its mangled name, against many values of the polynomial."""
    class Bounds(C.Structure):
        _fields_ = [("most", C.c_double), ("factor", C.c_double)]
    fn = pxr.lib()._ZN3pxr20orthogonalise_boundsEdddd
    fn.argtypes, fn.restype = [C.c_double] * 4, Bounds
    rng = np.random.default_rng(0)
    cases = [QUINTIC, (1.5, -0.5, 0), (2, 0, 0), (0, 0, 0), (0, 1, 0), (1, 1, 1), (15 / 8, -10 / 8, 3 / 8), *rng.standard_normal((200, 3)) * 5]
    for a, b, c in cases:
        for most in (1.0, 0.3, 1.2, 7.0):
            t = np.linspace(0, most, 20001)
            got = fn(a, b, c, most)
            value, factor = np.abs(a * t + b * t ** 3 + c * t ** 5).max(), np.abs(a + b * t ** 2 + c * t ** 4).max()
            assert value <= got.most <= value * 1.002 + 1e-6 and factor <= got.factor * (1 + 1e-12) <= factor * 1.001 + 1e-6, (a, b, c, most)


def _need(coefficients=(QUINTIC,) * 5, **change):
    """The workspace's bytes: nothing is launched."""
    c = np.ascontiguousarray(coefficients, np.float32)
    d = pxr.OrthogonaliseDesc(0, 1, 8, 16, 0, 16, 0, 16, len(c), c.ctypes.data, 1e-7)
    for name, value in change.items():
        setattr(d, name, value)
    n = C.c_size_t()
    assert pxr.lib().pxr_orthogonalise_workspace(C.byref(d), C.byref(n)) == pxr.OK
    return n.value


@pytest.mark.parametrize("steps", [(QUINTIC,) * 7, ((1.5, -0.5, 0.0),) * 19, ((1100.0, 0.0, 0.0), (0.001, 0.0, 0.0))])
def test_long_matrices_of_few_rows_take_many_steps_in_rounds(steps):
    """A has to be formed from X again before the steps have multiplied its roundings by their factors' squares, 1024^2 and more: X is held between two rounds, [rows,cols] in fp64."""
    one, two = (_need(rows=8, cols=5000, x_row=5000, out_row=5000, coefficients=c) for c in (steps[:-1], steps))
    assert two == one + 8 * 8 * 5000
    assert _need(rows=5000, cols=8, x_row=8, out_row=8, n_matrices=3, out_matrix=40000, coefficients=steps) == 3 * two
    assert _call(rows=5000, cols=8, x_row=8, out_row=8, coefficients=steps, workspace=two - 1)[1] == pxr.ERR_INVALID_ARG
    # smaller ones, and those of more rows, form it in every step
    for m, n in ((8, 300), (40, 5000)):
        one, two = (_need(rows=m, cols=n, x_row=n, out_row=n, coefficients=c) for c in (steps[:1], steps))
        assert one == two


def test_results_that_share_values_with_the_update():
    """Refused before the workspace is looked at: a row, a value or a matrix on; parts of one buffer side by side, and x itself, are not."""
    base = 1 << 24
    for m, n, B, pitch in ((40, 5000, 1, 5000), (600, 64, 3, 200), (5000, 7, 2, 21)):
        d = dict(rows=m, cols=n, n_matrices=B, x_row=pitch, out_row=pitch, x_matrix=m * pitch, out_matrix=m * pitch)
        assert _need(**d) > 0
        why = lambda x, out: (_call(buffers=(4 * x, 4 * out, None), **d)[1], pxr.lib().pxr_last_error().decode())
        for by in (1, -1, pitch, 1 - n, (m - 1) * pitch, B * m * pitch - 1 if B > 1 else pitch, -pitch + 1):
            shared = any(abs(by + i * m * pitch + j * pitch) < n for i in range(1 - B, B) for j in range(1 - m, m))
            code, message = why(base, base + by)
            assert code == pxr.ERR_INVALID_ARG and ("overlaps x" if shared else "workspace") in message, (m, n, by)
        for x, out in ((base, base), (base, base + B * m * pitch), (base, base - B * m * pitch), *(((base, base + n), (base + 2 * n, base)) if pitch >= 3 * n else ())):
            assert "workspace" in why(x, out)[1]
        d["out_row"], d["out_matrix"] = pitch + 1, m * (pitch + 1)
        assert "overlaps x" in why(base, base)[1]
