"""Refusals of a gated recurrence that need no device."""
import ctypes as C

import pytest

from paper_2502_00021_amd import pxr


def _rollout(**change):
    r = pxr.GatedRollout(0, 2, 3, 8, 1, pxr.Steps(64, 24, 8), pxr.Steps(64, 24, 8), None, 0, 0, None)
    for name, value in change.items():
        setattr(r, name, value)
    return r


VIEW = pxr.Steps(64, 24, 8)
SIZES = [dict(n_envs=0), dict(width=0), dict(n_steps=2 ** 31), dict(n_envs=2 ** 22 + 1), dict(n_envs=2 ** 22, width=65), dict(n_envs=2 ** 32 - 1, width=2 ** 32 - 1),
         dict(n_envs=2 ** 22, n_steps=129), dict(n_envs=1, width=2 ** 28 + 1), dict(n_envs=2 ** 12, width=2 ** 12, n_steps=2 ** 20)]


def _all(r, view=VIEW, state=64):
    L = pxr.lib()
    r1 = pxr.GatedRollout.from_buffer_copy(r)
    return (L.pxr_gated_recurrence_forward(C.byref(r), C.byref(view), None, 64, 1 << 60, None),
            L.pxr_gated_recurrence_backward(C.byref(r), C.byref(VIEW), None, C.byref(view), C.byref(view), None, 64, 1 << 60, None),
            L.pxr_gated_recurrence_step(C.byref(r1), state, C.byref(view), None))


@pytest.mark.parametrize("change", SIZES + [dict(dtype=2), dict(coupled=2), dict(d_state=66)])
def test_descriptions(change):
    assert set(_all(_rollout(**change))) == {pxr.ERR_INVALID_ARG}
    assert pxr.lib().pxr_last_error()


@pytest.mark.parametrize("change", SIZES)
def test_workspace(change):
    r = _rollout(**change)
    n = C.c_size_t()
    for backward in (0, 1):
        assert pxr.lib().pxr_gated_recurrence_workspace(r.n_envs, r.n_steps, r.width, backward, C.byref(n)) == pxr.ERR_INVALID_ARG
        assert pxr.lib().pxr_gated_recurrence_workspace(2, 3, 8, backward, None) == pxr.ERR_INVALID_ARG
        assert pxr.lib().pxr_gated_recurrence_workspace(2, 3, 8, backward, C.byref(n)) == pxr.OK and n.value == 0
        assert pxr.lib().pxr_gated_recurrence_workspace(1, 50000, 512, backward, C.byref(n)) == pxr.OK and n.value > 0


def test_buffers():
    L = pxr.lib()
    for data in (None, 66):
        bad = pxr.Steps(data, 24, 8)
        for change in (dict(x=bad), dict(gate=bad)):
            assert set(_all(_rollout(**change))) == {pxr.ERR_INVALID_ARG}
            assert L.pxr_gated_recurrence_step(C.byref(_rollout(n_steps=1, **change)), 64, C.byref(VIEW), None) == pxr.ERR_INVALID_ARG
        assert set(_all(_rollout(), bad)) == {pxr.ERR_INVALID_ARG}
        assert L.pxr_gated_recurrence_step(C.byref(_rollout(n_steps=1)), 64, C.byref(bad), None) == pxr.ERR_INVALID_ARG
        assert L.pxr_gated_recurrence_step(C.byref(_rollout(n_steps=1)), data, C.byref(VIEW), None) == pxr.ERR_INVALID_ARG
    r, v = _rollout(), C.byref(VIEW)
    assert L.pxr_gated_recurrence_step(C.byref(r), 64, v, None) == pxr.ERR_INVALID_ARG  # three steps
    assert L.pxr_gated_recurrence_forward(None, v, None, None, 0, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_gated_recurrence_forward(C.byref(r), None, None, None, 0, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_gated_recurrence_forward(C.byref(r), v, 66, None, 0, None) == pxr.ERR_INVALID_ARG
    for after, first in ((66, 64), (64, 66), (64, 64), (64, 68)):
        assert L.pxr_gated_recurrence_backward(C.byref(r), v, after, v, v, first, None, 0, None) == pxr.ERR_INVALID_ARG
    # states that overlap: 2 x 8 values of 4 bytes
    for out in (64, 68, 64 + 60, 4):
        assert L.pxr_gated_recurrence_forward(C.byref(_rollout(d_state=64)), v, out, None, 0, None) == pxr.ERR_INVALID_ARG
    # a workspace that is missing, misaligned or too small
    long = _rollout(n_steps=50000)
    n = C.c_size_t()
    for backward in (0, 1):
        assert L.pxr_gated_recurrence_workspace(2, 50000, 8, backward, C.byref(n)) == pxr.OK and n.value
        for ws, size in ((None, n.value), (72, n.value), (64, n.value - 1)):
            if backward:
                assert L.pxr_gated_recurrence_backward(C.byref(long), v, None, v, v, None, ws, size, None) == pxr.ERR_INVALID_ARG
            else:
                assert L.pxr_gated_recurrence_forward(C.byref(long), v, None, ws, size, None) == pxr.ERR_INVALID_ARG
