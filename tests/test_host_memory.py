"""Refusals of a policy's memory that need no device: descriptions of layer norms and of linear attention."""
import ctypes as C

import numpy as np
import pytest

from paper_2502_00021_amd import pxr


def _norm(**change):
    d = dict(dtype=0, param_dtype=0, n_rows=4, width=8, eps=1e-5, x_stride=8, y_stride=8, dx_stride=8)
    d.update(change)
    return pxr.LayerNormDesc(**d)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(param_dtype=1), dict(dtype=1, param_dtype=2), dict(width=0), dict(width=2 ** 30 + 1), dict(n_rows=2 ** 31),
                                    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x_stride=7), dict(y_stride=0), dict(x_stride=-8)])
def test_layer_norm_descriptions(change):
    L, d = pxr.lib(), _norm(**change)
    assert L.pxr_layer_norm_forward(C.byref(d), 64, None, None, 64, None, None, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_layer_norm_backward(C.byref(d), 64, 64, 64, 64, None, 64, None, None, None, 0, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_layer_norm_workspace(C.byref(d), C.byref(C.c_size_t())) == pxr.ERR_INVALID_ARG
    assert L.pxr_last_error()


def test_layer_norm_buffers():
    L, d = pxr.lib(), _norm()
    size = C.c_size_t()
    assert L.pxr_layer_norm_workspace(None, C.byref(size)) == L.pxr_layer_norm_workspace(C.byref(d), None) == pxr.ERR_INVALID_ARG
    assert L.pxr_layer_norm_workspace(C.byref(d), C.byref(size)) == pxr.OK
    forward = [64, 64, 64, 64, 64, 64]
    for i, bad in ((0, None), (3, None), (0, 66), (1, 65), (2, 66), (3, 66), (4, 66), (5, 66)):
        a = list(forward)
        a[i] = bad
        assert L.pxr_layer_norm_forward(C.byref(d), *a, None) == pxr.ERR_INVALID_ARG, (i, bad)
    backward = [64] * 9
    for i, bad in [(i, None) for i in (0, 1, 2, 3, 5)] + [(i, 66) for i in range(8)]:
        a = list(backward)
        a[i] = bad
        assert L.pxr_layer_norm_backward(C.byref(d), *a, 1 << 40, None) == pxr.ERR_INVALID_ARG, (i, bad)
    assert L.pxr_layer_norm_backward(C.byref(_norm(dx_stride=7)), *backward, 1 << 40, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_layer_norm_forward(C.byref(_norm(n_rows=0)), *[None] * 6, None) == pxr.OK  # nothing to do


@pytest.mark.parametrize("change,code", [
    (dict(n_heads=0), "INVALID_ARG"), (dict(n_heads=65536), "INVALID_ARG"), (dict(d_key=0), "INVALID_ARG"), (dict(d_value=0), "INVALID_ARG"),
    (dict(d_key=257), "UNSUPPORTED"), (dict(d_value=257), "UNSUPPORTED"), (dict(scale=float("nan")), "INVALID_ARG"), (dict(log_decay=None), "INVALID_ARG"),
    (dict(decays=[0.1, -1.0]), "INVALID_ARG"), (dict(decays=[-1.0, float("nan")]), "INVALID_ARG"), (dict(decays=[-float("inf"), 0.0]), "INVALID_ARG")])
def test_linear_attention_descriptions(change, code):
    decays = np.float32(change.pop("decays", [-0.5, -1.0]))
    d = pxr.LinearAttentionDesc(2, 16, 16, 1.0, decays.ctypes.data)
    for name, value in change.items():
        setattr(d, name, value)
    h = C.c_void_p()
    assert pxr.lib().pxr_linear_attention_create(C.byref(d), C.byref(h)) == getattr(pxr, "ERR_" + code)
    assert not h.value


def test_linear_attention_without_a_layer():
    L = pxr.lib()
    assert L.pxr_linear_attention_create(None, C.byref(C.c_void_p())) == pxr.ERR_INVALID_ARG
    assert L.pxr_linear_attention_destroy(None) == pxr.OK
    assert L.pxr_linear_attention_workspace(None, 0, 1, 1, 0, C.byref(C.c_size_t())) == pxr.ERR_INVALID_ARG
    assert L.pxr_linear_attention_forward(None, C.byref(pxr.Rollout()), C.byref(pxr.Tokens()), None, None, 0, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_linear_attention_step(None, C.byref(pxr.Rollout()), None, C.byref(pxr.Tokens()), None) == pxr.ERR_INVALID_ARG
