"""Refusals of a gated recurrence that need no device."""
import ctypes as C

import numpy as np
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


def _why(call, *args):
    """What a call says that has no workspace: whether it got as far as that."""
    assert call(*args) == pxr.ERR_INVALID_ARG
    return pxr.lib().pxr_last_error().decode()


def _places(v, B, T, D):
    return set(((np.arange(B)[:, None, None] * v.env + np.arange(T)[:, None] * v.step + np.arange(D)).ravel() + v.data // 4).tolist())


def test_views_that_are_written_share_no_value_with_the_others():
    """Against the values' places themselves, over strides that a view that does not overlap itself may have, those that programs have among them: parts of one buffer, the same one a step or an environment on,
    the other way round."""
    L, rng = pxr.lib(), np.random.default_rng(0)
    seen = [0, 0]
    for n in range(400):
        B, T, D = (int(rng.integers(1, 4)) for _ in range(3))
        T = 5000 if n % 2 else 700  # (a forward, a backward pass that needs a workspace)
        inner = int(rng.integers(D, 3 * D + 1))
        if rng.random() < 0.5:
            env, step = inner * T + int(rng.integers(0, 4)), inner
        else:
            env, step = inner, inner * B + int(rng.integers(0, 4))
        env, step = env * int(rng.choice([-1, 1])), step * int(rng.choice([-1, 1]))
        first = 1 << 22
        moved = int(rng.choice([0, 1, -1, D, -D, inner, step, env, -env + 1, step + D, 2 * step - D + 1, int(rng.integers(-inner * B * T, inner * B * T)), 1 << 20]))
        a, b, far = pxr.Steps(4 * first, env, step), pxr.Steps(4 * (first + moved), env, step), pxr.Steps(4 << 30, env, step)
        shared = bool(_places(a, B, T, D) & _places(b, B, T, D))
        seen[shared] += 1
        r = lambda x, gate: C.byref(pxr.GatedRollout(0, B, T, D, 1, x, gate, None, 0, 0, None))
        for x, gate in ((b, far), (far, b)):
            if n % 2:
                why = _why(L.pxr_gated_recurrence_forward, r(x, gate), C.byref(a), None, None, 0, None)
                assert ("overlaps" if shared else "workspace") in why, (B, T, D, env, step, moved)
        if n % 2 == 0:
            free = [pxr.Steps(4 << 31, env, step), pxr.Steps(4 << 32, env, step), pxr.Steps(4 << 33, env, step)]
            for views in ((b, *free[:2], a, free[2]), (b, *free[:2], free[2], a), (free[0], b, free[1], a, free[2]), (*free[:2], b, free[2], a), (*free, a, b)):
                x, gate, dout, dx, dgate = views
                why = _why(L.pxr_gated_recurrence_backward, r(x, gate), C.byref(dout), None, C.byref(dx), C.byref(dgate), None, None, 0, None)
                assert ("overlap" if shared else "workspace") in why, (B, T, D, env, step, moved)
    assert min(seen) > 100
    # strides that are not the same: apart, or from the same value on; inputs that environments or steps share; strides of any size
    for x, out, shared in ((pxr.Steps(4 << 20, 10, 5), pxr.Steps(4 << 20, 5000, 1), True), (pxr.Steps(4 << 20, 0, 0), pxr.Steps(8 << 20, 5000, 1), False), (pxr.Steps(8 << 20, 0, 0), pxr.Steps(8 << 20, 5000, 1), True),
                           (pxr.Steps(4 << 20, 2 ** 62, 2 ** 62), pxr.Steps(8 << 20, 5000, 1), False), (pxr.Steps(4 << 20, -2 ** 63, 1), pxr.Steps(4 << 20, -2 ** 63, 1), True)):
        why = _why(L.pxr_gated_recurrence_forward, C.byref(pxr.GatedRollout(0, 2, 5000, 1, 1, x, pxr.Steps(64, 0, 0), None, 0, 0, None)), C.byref(out), None, None, 0, None)
        assert ("overlaps" if shared else "workspace") in why
    # a single step: of the same place another environment on (its own place, which it may have, is for the GPU's tests)
    step = pxr.GatedRollout(0, 3, 1, 8, 1, pxr.Steps(4096, 8, 0), pxr.Steps(8192, 8, 0), None, 0, 0, None)
    for at in (4096 + 32, 4096 + 4, 8192 - 32):
        assert "overlaps" in _why(L.pxr_gated_recurrence_step, C.byref(step), 64, C.byref(pxr.Steps(at, 8, 0)), None)
