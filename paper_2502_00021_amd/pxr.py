"""ctypes binding of libpxr.so — argument marshalling only; every step runs in the HIP library.

Mirrors include/pxr.h one to one: create_scene / destroy_scene /
apply_distractor / render_batch, set_skeleton / pose_batch /
render_batch_kinematic (+ scene_info, set_block_threads, host_tables), the policy's first layer (Conv) and its memory
(layer_norm, layer_norm_backward, LinearAttention, gated_recurrence, HeadNorm),
a learner's update (orthogonalise).  PyTorch is used only to hold device memory and name the stream.
There is no fallback: a missing library or a failing call raises.
"""
import ctypes as C
import math
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpxr.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_OOM, ERR_DEVICE = range(5)
ID_GROUND = 0xFFFFFFFE
ID_BG = 0xFFFFFFFF
KINDS = {"capsule": 0, "sphere": 1, "box": 2, "mesh": 3}
MODES = {"none": 0, "color": 1, "video": 2}


class PxrError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"pxr error {code}: {message}")
        self.code = code


class BodyDesc(C.Structure):
    _fields_ = [("type", C.c_uint32), ("shape", C.c_float * 4), ("rgb", C.c_float * 3),
                ("n_lon", C.c_uint32), ("n_lat", C.c_uint32),
                ("mesh_verts", C.c_void_p), ("mesh_tris", C.c_void_p), ("mesh_tri_mul", C.c_void_p),
                ("n_mesh_verts", C.c_uint32), ("n_mesh_tris", C.c_uint32)]


class SceneDesc(C.Structure):
    _fields_ = [("width", C.c_uint32), ("height", C.c_uint32), ("n_bodies", C.c_uint32), ("root_body", C.c_uint32),
                ("bodies", C.POINTER(BodyDesc)),
                ("fov_y_deg", C.c_float), ("cam_offset", C.c_float * 3), ("cam_up", C.c_float * 3),
                ("z_near", C.c_float), ("z_far", C.c_float),
                ("light_dir", C.c_float * 3), ("ambient", C.c_float), ("diffuse", C.c_float),
                ("ground_enabled", C.c_uint32), ("ground_cell", C.c_float), ("ground_grey", C.c_float * 2),
                ("background_rgb", C.c_float * 3)]


class DistractorDesc(C.Structure):
    _fields_ = [("mode", C.c_uint32), ("seed", C.c_uint64),
                ("scale_lo", C.c_float), ("scale_hi", C.c_float), ("offset_lo", C.c_float), ("offset_hi", C.c_float),
                ("d_video", C.c_void_p), ("n_frames", C.c_uint32), ("alpha", C.c_float),
                ("d_env_offset", C.c_void_p), ("n_videos", C.c_uint32), ("d_env_video", C.c_void_p)]


class SkeletonDesc(C.Structure):
    _fields_ = [("n_bodies", C.c_uint32), ("n_free", C.c_uint32), ("n_angles", C.c_uint32),
                ("parent", C.c_void_p), ("slot", C.c_void_p), ("anchor", C.c_void_p), ("axis", C.c_void_p),
                ("offset", C.c_void_p)]


class ConvDesc(C.Structure):
    _fields_ = [("in_h", C.c_uint32), ("in_w", C.c_uint32), ("n_stack", C.c_uint32),
                ("c_out", C.c_uint32), ("kernel", C.c_uint32), ("stride", C.c_uint32),
                ("weights", C.c_void_p), ("bias", C.c_void_p), ("relu", C.c_uint32)]


class LayerNormDesc(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("param_dtype", C.c_uint32), ("n_rows", C.c_uint64), ("width", C.c_uint32),
                ("eps", C.c_float), ("x_stride", C.c_int64), ("y_stride", C.c_int64), ("dx_stride", C.c_int64)]


class LinearAttentionDesc(C.Structure):
    _fields_ = [("n_heads", C.c_uint32), ("d_key", C.c_uint32), ("d_value", C.c_uint32), ("scale", C.c_float),
                ("log_decay", C.c_void_p)]


class Tokens(C.Structure):
    _fields_ = [("data", C.c_void_p), ("env", C.c_int64), ("step", C.c_int64), ("head", C.c_int64)]


class Rollout(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("n_envs", C.c_uint32), ("n_steps", C.c_uint32),
                ("q", Tokens), ("k", Tokens), ("v", Tokens),
                ("d_resets", C.c_void_p), ("resets_env", C.c_int64), ("resets_step", C.c_int64), ("d_state", C.c_void_p)]


class Steps(C.Structure):
    _fields_ = [("data", C.c_void_p), ("env", C.c_int64), ("step", C.c_int64)]


class GatedRollout(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("n_envs", C.c_uint32), ("n_steps", C.c_uint32), ("width", C.c_uint32), ("coupled", C.c_uint32),
                ("x", Steps), ("gate", Steps),
                ("d_resets", C.c_void_p), ("resets_env", C.c_int64), ("resets_step", C.c_int64), ("d_state", C.c_void_p)]


class HeadNormDesc(C.Structure):
    _fields_ = [("d_head", C.c_uint32), ("d_rotary", C.c_uint32), ("frequencies", C.c_void_p), ("eps", C.c_float)]


class Heads(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("param_dtype", C.c_uint32), ("n_envs", C.c_uint32), ("n_steps", C.c_uint32),
                ("n_heads", C.c_uint32), ("n_key_heads", C.c_uint32), ("q", Tokens), ("k", Tokens),
                ("d_q_weight", C.c_void_p), ("d_k_weight", C.c_void_p), ("d_positions", C.c_void_p), ("position_bits", C.c_uint32),
                ("positions_env", C.c_int64), ("positions_step", C.c_int64), ("first", C.c_int64)]


class OrthogonaliseDesc(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("n_matrices", C.c_uint32), ("rows", C.c_uint32), ("cols", C.c_uint32),
                ("x_matrix", C.c_int64), ("x_row", C.c_int64), ("out_matrix", C.c_int64), ("out_row", C.c_int64),
                ("n_steps", C.c_uint32), ("coefficients", C.c_void_p), ("eps", C.c_float)]


# Calls' structures as bytes: a call packs its arguments in a fraction of the time that it takes to fill the structures.
_pack_norm = struct.Struct("@IIQIfqqq").pack
_pack_tokens = struct.Struct("@Pqqq").pack
_pack_rollout = struct.Struct("@III4xPqqqPqqqPqqqPqqP").pack
_pack_heads = struct.Struct("@IIIIIIPqqqPqqqPPPI4xqqq").pack
_pack_orthogonalise = struct.Struct("@IIIIqqqqI4xPf4x").pack
_pack_steps = struct.Struct("@Pqq").pack
_pack_gated = struct.Struct("@IIIII4xPqqPqqPqqP").pack


_lib = None
_lib_path = LIB_PATH


def use_library_file(path):
    """Profiling only (bench.py --profile-lib): load another build of the same sources, e.g. one with phase
    clocks compiled in (paper_2502_00021_amd/build.py --define ... --out FILE).  Must be called before the
    library is first used; nothing in the product path calls it, and no environment variable can."""
    global _lib_path
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    _lib_path = os.path.abspath(path)


def lib():
    """Load libpxr.so (built in-tree by __graft_entry__.build / paper_2502_00021_amd.build)."""
    global _lib
    if _lib is None:
        path = _lib_path
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` first")
        try:  # PyTorch's HIP runtime first: a process that loads this library before it finds no device afterwards
            import torch  # noqa: F401
        except ImportError:
            pass
        L = C.CDLL(path)
        vp, u32 = C.c_void_p, C.c_uint32
        L.pxr_create_scene.argtypes = [C.POINTER(SceneDesc), C.POINTER(vp)]
        L.pxr_destroy_scene.argtypes = [vp]
        L.pxr_apply_distractor.argtypes = [vp, C.POINTER(DistractorDesc)]
        L.pxr_render_batch.argtypes = [vp, vp, vp, u32, u32, u32, u32, vp, vp, vp]
        L.pxr_scene_info.argtypes = [vp, vp, vp, vp, vp]
        L.pxr_set_block_threads.argtypes = [vp, u32]
        L.pxr_host_tables.argtypes = [C.POINTER(SceneDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.pxr_set_skeleton.argtypes = [vp, C.POINTER(SkeletonDesc)]
        L.pxr_pose_batch.argtypes = [vp, vp, vp, u32, vp, vp]
        L.pxr_render_batch_kinematic.argtypes = [vp, vp, vp, vp, u32, u32, u32, u32, vp, vp, vp, vp]
        L.pxr_render_batch_kinematic_static.argtypes = [vp, vp, vp, vp, u32, u32, u32, u32, vp, vp, vp]
        L.pxr_render_batch_kinematic_static.restype = C.c_int
        L.pxr_kinematic_info.argtypes = [vp, u32, C.POINTER(u32)]
        L.pxr_kinematic_info.restype = C.c_int
        L.pxr_conv_create.argtypes = [C.POINTER(ConvDesc), C.POINTER(vp)]
        L.pxr_conv_destroy.argtypes = [vp]
        L.pxr_conv_forward.argtypes = [vp, vp, u32, vp, vp]
        L.pxr_conv_info.argtypes = [vp, vp, vp, vp, vp, vp]
        L.pxr_conv_set_tuning.argtypes = [vp, u32, u32]
        for name in ("pxr_conv_create", "pxr_conv_destroy", "pxr_conv_forward", "pxr_conv_info", "pxr_conv_set_tuning"):
            getattr(L, name).restype = C.c_int
        L.pxr_pipeline_create.argtypes = [vp, vp, u32, C.POINTER(vp)]
        L.pxr_pipeline_destroy.argtypes = [vp]
        L.pxr_pipeline_step.argtypes = [vp, vp, vp, u32, u32, u32, vp, vp, vp]
        L.pxr_pipeline_set_overlap_from.argtypes = [vp, C.c_uint64]
        L.pxr_pipeline_info.argtypes = [vp, u32, C.POINTER(u32)]
        for name in ("pxr_pipeline_create", "pxr_pipeline_destroy", "pxr_pipeline_step", "pxr_pipeline_set_overlap_from",
                     "pxr_pipeline_info"):
            getattr(L, name).restype = C.c_int
        size = C.POINTER(C.c_size_t)
        tokens = rollout = norm = vp  # (structures, or their packed bytes)
        L.pxr_layer_norm_forward.argtypes = [norm, vp, vp, vp, vp, vp, vp, vp]
        L.pxr_layer_norm_workspace.argtypes = [norm, size]
        L.pxr_layer_norm_backward.argtypes = [norm, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.pxr_linear_attention_create.argtypes = [C.POINTER(LinearAttentionDesc), C.POINTER(vp)]
        L.pxr_linear_attention_destroy.argtypes = [vp]
        L.pxr_linear_attention_workspace.argtypes = [vp, u32, u32, u32, u32, size]
        L.pxr_linear_attention_forward.argtypes = [vp, rollout, tokens, vp, vp, C.c_size_t, vp]
        L.pxr_linear_attention_backward.argtypes = [vp, rollout, tokens, vp, tokens, tokens, tokens, vp, vp, C.c_size_t, vp]
        L.pxr_linear_attention_step.argtypes = [vp, rollout, vp, tokens, vp]
        for name in ("layer_norm_forward", "layer_norm_workspace", "layer_norm_backward", "linear_attention_create",
                     "linear_attention_destroy", "linear_attention_workspace", "linear_attention_forward",
                     "linear_attention_backward", "linear_attention_step"):
            getattr(L, "pxr_" + name).restype = C.c_int
        steps = vp
        L.pxr_gated_recurrence_workspace.argtypes = [u32, u32, u32, u32, size]
        L.pxr_gated_recurrence_forward.argtypes = [rollout, steps, vp, vp, C.c_size_t, vp]
        L.pxr_gated_recurrence_backward.argtypes = [rollout, steps, vp, steps, steps, vp, vp, C.c_size_t, vp]
        L.pxr_gated_recurrence_step.argtypes = [rollout, vp, steps, vp]
        for name in ("workspace", "forward", "backward", "step"):
            getattr(L, "pxr_gated_recurrence_" + name).restype = C.c_int
        heads = vp
        L.pxr_head_norm_create.argtypes = [C.POINTER(HeadNormDesc), C.POINTER(vp)]
        L.pxr_head_norm_destroy.argtypes = [vp]
        L.pxr_head_norm_forward.argtypes = [vp, heads, tokens, tokens, vp]
        L.pxr_head_norm_workspace.argtypes = [vp, heads, size]
        L.pxr_head_norm_backward.argtypes = [vp, heads, tokens, tokens, tokens, tokens, vp, vp, vp, C.c_size_t, vp]
        for name in ("create", "destroy", "forward", "workspace", "backward"):
            getattr(L, "pxr_head_norm_" + name).restype = C.c_int
        L.pxr_orthogonalise_workspace.argtypes = [vp, size]
        L.pxr_orthogonalise.argtypes = [vp, vp, vp, vp, C.c_size_t, vp]
        L.pxr_orthogonalise_workspace.restype = L.pxr_orthogonalise.restype = C.c_int
        L.pxr_selftest_arithmetic.argtypes = [vp]
        L.pxr_selftest_arithmetic.restype = C.c_int
        L.pxr_measure_peaks.argtypes = [vp, vp, vp, vp, vp]
        L.pxr_measure_peaks.restype = C.c_int
        L.pxr_last_error.restype = C.c_char_p
        for name in ("pxr_create_scene", "pxr_destroy_scene", "pxr_apply_distractor", "pxr_render_batch",
                     "pxr_scene_info", "pxr_set_block_threads", "pxr_host_tables", "pxr_set_skeleton",
                     "pxr_pose_batch", "pxr_render_batch_kinematic"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


_torch = None


def _torch_module():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _stream_handle(stream, tensor):
    """The caller's stream handle (an integer), or that of the current stream of the tensor's GPU (without building a
    Stream object on every call)."""
    if stream is None:
        return _torch._C._cuda_getCurrentRawStream(tensor.get_device())
    return C.c_void_p(stream)  # (an integer or a TypeError: as a pointer argument, ctypes would take text and bytes)


def _check(rc):
    if rc != OK:
        raise PxrError(rc, lib().pxr_last_error().decode())


def _written(torch, *tensors):
    """Tensors of the caller's that a call has written through their pointers: autograd learns that they are other values
    now, and refuses a backward pass that saved the ones before."""
    torch.autograd.graph.increment_version(tensors)


def make_scene_desc(desc):
    """Plain-dict scene description (see workloads.default_scene) -> (SceneDesc, keep-alive list)."""
    bodies = desc["bodies"]
    arr = (BodyDesc * max(1, len(bodies)))()
    keep = [arr]
    for i, b in enumerate(bodies):
        arr[i].type = KINDS[b["kind"]] if isinstance(b["kind"], str) else int(b["kind"])
        arr[i].shape = (C.c_float * 4)(*b["shape"])
        arr[i].rgb = (C.c_float * 3)(*b["rgb"])
        arr[i].n_lon = int(b["n_lon"])
        arr[i].n_lat = int(b.get("n_lat", 0))
        if b.get("verts") is not None:  # caller-supplied mesh
            v = np.ascontiguousarray(b["verts"], dtype=np.float32).reshape(-1, 3)
            t = np.ascontiguousarray(b["tris"], dtype=np.uint32).reshape(-1, 3)
            keep += [v, t]
            arr[i].mesh_verts, arr[i].mesh_tris = v.ctypes.data, t.ctypes.data
            arr[i].n_mesh_verts, arr[i].n_mesh_tris = v.shape[0], t.shape[0]
            if b.get("mul") is not None:
                m = np.ascontiguousarray(b["mul"], dtype=np.float32)
                assert m.shape == (t.shape[0],)
                keep.append(m)
                arr[i].mesh_tri_mul = m.ctypes.data
    d = SceneDesc()
    d.width, d.height = int(desc["width"]), int(desc["height"])
    d.n_bodies, d.root_body = len(bodies), int(desc["root_body"])
    d.bodies = C.cast(arr, C.POINTER(BodyDesc))
    d.fov_y_deg = desc["fov_y_deg"]
    d.cam_offset = (C.c_float * 3)(*desc["cam_offset"])
    d.cam_up = (C.c_float * 3)(*desc["cam_up"])
    d.z_near, d.z_far = desc["z_near"], desc["z_far"]
    d.light_dir = (C.c_float * 3)(*desc["light_dir"])
    d.ambient, d.diffuse = desc["ambient"], desc["diffuse"]
    d.ground_enabled = 1 if desc["ground_enabled"] else 0
    d.ground_cell = desc["ground_cell"]
    d.ground_grey = (C.c_float * 2)(*desc["ground_grey"])
    d.background_rgb = (C.c_float * 3)(*desc["background_rgb"])
    return d, keep


def host_tables(desc):
    """pxr_host_tables: the scene builder's tables as numpy arrays (no device needed)."""
    d, keep = make_scene_desc(desc)
    nv, nt, npair = C.c_uint32(), C.c_uint32(), C.c_uint32()
    _check(lib().pxr_host_tables(C.byref(d), C.byref(nv), C.byref(nt), None, None, None, None, None,
                                 C.byref(npair), None))
    V, T, P = nv.value, nt.value, npair.value
    pt = np.empty((P, 3), np.uint32)
    vt = np.empty((V, 4), np.float32)
    ti = np.empty((T, 2), np.uint32)
    ts = np.empty((T, 4), np.float32)
    cxcy = np.empty(d.width + d.height, np.float32)
    consts = np.empty(16, np.float32)
    _check(lib().pxr_host_tables(C.byref(d), None, None, vt.ctypes.data, ti.ctypes.data, ts.ctypes.data,
                                 cxcy.ctypes.data, consts.ctypes.data, None, pt.ctypes.data))
    del keep
    code = vt[:, 3].copy().view(np.uint32)
    return dict(V=V, T=T, uverts=np.concatenate([vt[:, :3], ((code & 3).astype(np.float32) - 1.0)[:, None]], axis=1),
                vert_body=code >> 2,
                tris=np.stack([ti[:, 0] & 0xFFFF, ti[:, 0] >> 16, ti[:, 1] & 0xFFFF], axis=1).astype(np.uint32),
                tri_body=ti[:, 1] >> 16, normals=ts[:, :3].copy(), mul=ts[:, 3].copy(),
                cx=cxcy[:d.width].copy(), cy=cxcy[d.width:].copy(),
                Rv=consts[:9].reshape(3, 3).copy(), f=float(consts[9]), gs=consts[10:12].copy(), l=consts[12:15].copy(),
                lds_bytes=int(consts[15]),
                pair_quads=np.stack([pt[:, 0] & 0xFFFF, pt[:, 0] >> 16, pt[:, 1] & 0xFFFF, pt[:, 1] >> 16], axis=1),
                pair_tris=np.stack([pt[:, 2] & 0xFFFF, pt[:, 2] >> 16], axis=1))


class Scene:
    """Owns one pxr_scene handle.  Tensors passed to render_batch must live on the scene's GPU."""

    def __init__(self, desc):
        d, keep = make_scene_desc(desc)
        h = C.c_void_p()
        _check(lib().pxr_create_scene(C.byref(d), C.byref(h)))
        del keep
        self._h = h
        self.W, self.H, self.K = d.width, d.height, d.n_bodies
        self._bound = []  # keeps bound distractor tensors alive
        self._skel = None  # (n_free, n_angles) of the bound skeleton

    def close(self):
        if getattr(self, "_h", None):
            _check(lib().pxr_destroy_scene(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def info(self):
        v, t, l, b = C.c_uint32(), C.c_uint32(), C.c_uint32(), C.c_uint32()
        _check(lib().pxr_scene_info(self._h, C.byref(v), C.byref(t), C.byref(l), C.byref(b)))
        return dict(n_verts=v.value, n_tris=t.value, lds_bytes=l.value, block_threads=b.value)

    def set_block_threads(self, n):
        _check(lib().pxr_set_block_threads(self._h, int(n)))

    def apply_distractor(self, d=None):
        """d: None / {"mode": "none"} to unbind, or a dict as produced by the workload generators,
        with `video` / `env_offset` given as CUDA uint8 / int32 tensors."""
        self._bound = []
        if d is None or d.get("mode", "none") == "none":
            _check(lib().pxr_apply_distractor(self._h, None))
            return
        unknown = set(d) - {"mode", "seed", "scale", "offset", "video", "alpha", "env_offset", "env_video"}
        if unknown:  # (a misspelt key would silently leave its default in place)
            raise ValueError(f"unknown distractor keys: {sorted(unknown)}")
        s = DistractorDesc()
        s.mode = MODES[d["mode"]]
        s.seed = int(d.get("seed", 0))
        s.scale_lo, s.scale_hi = d.get("scale", (1.0, 1.0))
        s.offset_lo, s.offset_hi = d.get("offset", (0.0, 0.0))
        if d["mode"] == "video":
            v = d["video"]
            assert v.is_cuda and v.is_contiguous() and v.dtype.itemsize == 1 and tuple(v.shape[-3:]) == (self.H, self.W, 3)
            s.d_video = v.data_ptr()
            if v.dim() == 5:  # a set of clips [n_videos, n_frames, H, W, 3]
                s.n_videos, s.n_frames = v.shape[0], v.shape[1]
                ev = d.get("env_video")
                if ev is not None:
                    assert ev.is_cuda and ev.is_contiguous() and ev.dtype.itemsize == 4
                    s.d_env_video = ev.data_ptr()
                    self._bound.append(ev)
            else:
                assert v.dim() == 4
                s.n_frames = v.shape[0]
            s.alpha = float(d.get("alpha", 0.5))
            self._bound.append(v)
            eo = d.get("env_offset")
            if eo is not None:
                assert eo.is_cuda and eo.is_contiguous() and eo.dtype.itemsize == 4
                s.d_env_offset = eo.data_ptr()
                self._bound.append(eo)
        _check(lib().pxr_apply_distractor(self._h, C.byref(s)))

    def render_batch(self, poses, shapes=None, step0=0, env0=0, frames=None, ids=None, want_ids=False, stream=None):
        """poses: CUDA float32 [B,S,K,7]; shapes: CUDA float32 [B,K,4] or None.
        Returns (frames uint8 [B,S,H,W,3], ids int32-typed uint32 bits [B,S,H,W] or None); enqueue only."""
        torch = _torch or _torch_module()
        assert poses.is_cuda and poses.dtype == torch.float32 and poses.is_contiguous()
        B, S = poses.shape[0], poses.shape[1]
        assert poses.shape == (B, S, self.K, 7), tuple(poses.shape)
        if shapes is not None:
            assert shapes.is_cuda and shapes.dtype == torch.float32 and shapes.is_contiguous()
            assert shapes.shape == (B, self.K, 4)
        if frames is None:
            frames = torch.empty((B, S, self.H, self.W, 3), dtype=torch.uint8, device=poses.device)
        else:
            assert frames.is_cuda and frames.is_contiguous() and frames.dtype == torch.uint8
            assert frames.shape == (B, S, self.H, self.W, 3)
        if ids is None and want_ids:
            ids = torch.empty((B, S, self.H, self.W), dtype=torch.int32, device=poses.device)
        if ids is not None:
            assert ids.is_cuda and ids.is_contiguous() and ids.dtype == torch.int32
            assert ids.shape == (B, S, self.H, self.W)
        stream = _stream_handle(stream, poses)
        _check(_lib.pxr_render_batch(self._h, poses.data_ptr(), None if shapes is None else shapes.data_ptr(),
                                     B, S, int(step0), int(env0), frames.data_ptr(),
                                     None if ids is None else ids.data_ptr(), stream))
        return frames, ids

    # ---- kinematics stage

    def set_skeleton(self, skel, n_free, n_angles):
        """skel: dict(parent, slot, anchor, axis, offset) of length-K host arrays (workloads._skeleton), or None."""
        if skel is None:
            _check(lib().pxr_set_skeleton(self._h, None))
            self._skel = None
            return
        d, keep = make_skeleton_desc(skel, n_free, n_angles)
        _check(lib().pxr_set_skeleton(self._h, C.byref(d)))
        del keep
        self._skel = (int(n_free), int(n_angles))

    def _fk_args(self, free_poses, angles):
        torch = _torch or _torch_module()
        if self._skel is None:
            raise PxrError(ERR_INVALID_ARG, "no skeleton bound (Scene.set_skeleton)")
        F, J = self._skel
        lead = tuple(free_poses.shape[:-2]) if F else tuple(angles.shape[:-1])
        n = math.prod(lead)
        if F:
            assert free_poses.is_cuda and free_poses.dtype == torch.float32 and free_poses.is_contiguous()
            assert free_poses.shape == lead + (F, 7), tuple(free_poses.shape)
        if J:
            assert angles.is_cuda and angles.dtype == torch.float32 and angles.is_contiguous()
            assert angles.shape == lead + (J,), tuple(angles.shape)
        return lead, n, free_poses if F else angles, (free_poses.data_ptr() if F else None), (angles.data_ptr() if J else None)

    def pose_batch(self, free_poses, angles, poses=None, stream=None):
        """free_poses: CUDA float32 [..., F, 7]; angles: CUDA float32 [..., J] -> poses [..., K, 7]; enqueue only."""
        torch = _torch or _torch_module()
        lead, n, source, pf, pa = self._fk_args(free_poses, angles)
        if poses is None:
            poses = torch.empty(lead + (self.K, 7), dtype=torch.float32, device=source.device)
        else:
            assert poses.is_cuda and poses.is_contiguous() and poses.dtype == torch.float32
            assert poses.shape == lead + (self.K, 7)
        stream = _stream_handle(stream, source)
        _check(_lib.pxr_pose_batch(self._h, pf, pa, n, poses.data_ptr(), stream))
        return poses

    def kinematic_launches(self, n_frames):
        """How many kernels render_batch_kinematic launches for that many frames (1 or 2)."""
        n = C.c_uint32()
        _check(lib().pxr_kinematic_info(self._h, int(n_frames), C.byref(n)))
        return n.value

    def render_batch_kinematic(self, free_poses, angles, shapes=None, step0=0, env0=0, poses=None, frames=None,
                               want_ids=False, stream=None):
        """free_poses [B,S,F,7], angles [B,S,J] -> (frames, ids or None, poses [B,S,K,7]); enqueue only."""
        torch = _torch or _torch_module()
        lead, n, source, pf, pa = self._fk_args(free_poses, angles)
        B, S = lead
        if poses is None:
            poses = torch.empty((B, S, self.K, 7), dtype=torch.float32, device=source.device)
        if frames is None:
            frames = torch.empty((B, S, self.H, self.W, 3), dtype=torch.uint8, device=source.device)
        assert poses.is_contiguous() and poses.shape == (B, S, self.K, 7) and poses.dtype == torch.float32
        assert frames.is_contiguous() and frames.shape == (B, S, self.H, self.W, 3) and frames.dtype == torch.uint8
        if shapes is not None:
            assert shapes.is_cuda and shapes.dtype == torch.float32 and shapes.is_contiguous()
            assert shapes.shape == (B, self.K, 4)
        ids = torch.empty((B, S, self.H, self.W), dtype=torch.int32, device=source.device) if want_ids else None
        stream = _stream_handle(stream, source)
        _check(_lib.pxr_render_batch_kinematic(self._h, pf, pa, None if shapes is None else shapes.data_ptr(), B, S,
                                               int(step0), int(env0), poses.data_ptr(), frames.data_ptr(),
                                               None if ids is None else ids.data_ptr(), stream))
        return frames, ids, poses


    def render_batch_kinematic_static(self, free_poses, angles, shapes=None, step0=0, env0=0, frames=None, ids=None,
                                      stream=None):
        """pxr_render_batch_kinematic_static: like render_batch_kinematic, the poses staying in the library's own
        static device buffer.  `frames` (and `ids`, if wanted) must be given: this call allocates nothing."""
        torch = _torch or _torch_module()
        lead, n, source, pf, pa = self._fk_args(free_poses, angles)
        B, S = lead
        assert frames is not None and frames.is_cuda and frames.is_contiguous() and frames.dtype == torch.uint8
        assert tuple(frames.shape) == (B, S, self.H, self.W, 3)
        if ids is not None:
            assert ids.is_cuda and ids.is_contiguous() and ids.dtype == torch.int32 and tuple(ids.shape) == (B, S, self.H, self.W)
        if shapes is not None:
            assert shapes.is_cuda and shapes.dtype == torch.float32 and shapes.is_contiguous()
            assert tuple(shapes.shape) == (B, self.K, 4)
        stream = _stream_handle(stream, source)
        _check(_lib.pxr_render_batch_kinematic_static(self._h, pf, pa, None if shapes is None else shapes.data_ptr(), B, S,
                                                      int(step0), int(env0), frames.data_ptr(),
                                                      None if ids is None else ids.data_ptr(), stream))
        return frames, ids


class Conv:
    """Owns one pxr_conv handle: the policy's first convolutional layer (3x3, stride 2, 32 channels) on the frame stack."""

    def __init__(self, in_h, in_w, n_stack, weights, bias, relu=True, c_out=32, kernel=3, stride=2):
        w = np.ascontiguousarray(weights, dtype=np.float32)
        b = np.ascontiguousarray(bias, dtype=np.float32)
        assert w.shape == (kernel, kernel, 3 * n_stack, c_out) and b.shape == (c_out,), (w.shape, b.shape)
        d = ConvDesc()
        d.in_h, d.in_w, d.n_stack = int(in_h), int(in_w), int(n_stack)
        d.c_out, d.kernel, d.stride = int(c_out), int(kernel), int(stride)
        d.weights, d.bias, d.relu = w.ctypes.data, b.ctypes.data, 1 if relu else 0
        h = C.c_void_p()
        _check(lib().pxr_conv_create(C.byref(d), C.byref(h)))
        self._h = h
        self.H, self.W, self.S, self.C = int(in_h), int(in_w), int(n_stack), int(c_out)
        i = self.info()
        self.Ho, self.Wo = i["out_h"], i["out_w"]

    def close(self):
        if getattr(self, "_h", None):
            _check(lib().pxr_conv_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def info(self):
        v = [C.c_uint32() for _ in range(5)]
        _check(lib().pxr_conv_info(self._h, *[C.byref(x) for x in v]))
        return dict(zip(("out_h", "out_w", "band_rows", "lds_bytes", "n_groups"), (x.value for x in v)))

    def set_tuning(self, band_rows=0, n_groups=0):
        _check(lib().pxr_conv_set_tuning(self._h, int(band_rows), int(n_groups)))

    def forward(self, frames, out=None, stream=None):
        """frames: CUDA uint8 [B,S,H,W,3] -> CUDA bfloat16 [B,Ho,Wo,32]; enqueue only."""
        torch = _torch or _torch_module()
        assert frames.is_cuda and frames.dtype == torch.uint8 and frames.is_contiguous()
        B = frames.shape[0]
        assert frames.shape == (B, self.S, self.H, self.W, 3), tuple(frames.shape)
        given = out is not None
        if out is None:
            out = torch.empty((B, self.Ho, self.Wo, self.C), dtype=torch.bfloat16, device=frames.device)
        else:
            assert out.is_cuda and out.is_contiguous() and out.dtype == torch.bfloat16
            assert out.shape == (B, self.Ho, self.Wo, self.C)
        stream = _stream_handle(stream, frames)
        _check(_lib.pxr_conv_forward(self._h, frames.data_ptr(), B, out.data_ptr(), stream))
        if given:
            _written(torch, out)
        return out


class Pipeline:
    """Owns one pxr_pipeline handle: render + conv layer per step, chunk c's layer beside chunk c + 1's render."""

    def __init__(self, scene, conv, n_chunks=4):
        h = C.c_void_p()
        _check(lib().pxr_pipeline_create(scene._h, conv._h, int(n_chunks), C.byref(h)))
        self._h, self.scene, self.conv = h, scene, conv

    def close(self):
        if getattr(self, "_h", None):
            _check(lib().pxr_pipeline_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_overlap_from(self, n_bytes):
        """Bytes of frames and features from which steps are cut into chunks (0 = always)."""
        _check(lib().pxr_pipeline_set_overlap_from(self._h, int(n_bytes)))

    def chunks(self, B):
        """Into how many chunks a step of B environments is cut."""
        n = C.c_uint32()
        _check(lib().pxr_pipeline_info(self._h, int(B), C.byref(n)))
        return n.value

    def step(self, poses, shapes, frames, features, step0=0, env0=0, stream=None):
        """poses [B,S,K,7], shapes [B,K,4] or None -> frames [B,S,H,W,3] uint8, features [B,Ho,Wo,32] bf16 (both given)."""
        torch = _torch or _torch_module()
        sc, cv = self.scene, self.conv
        B = poses.shape[0]
        assert poses.is_cuda and poses.dtype == torch.float32 and poses.is_contiguous() and poses.shape == (B, cv.S, sc.K, 7)
        if shapes is not None:
            assert shapes.is_cuda and shapes.dtype == torch.float32 and shapes.is_contiguous() and shapes.shape == (B, sc.K, 4)
        assert frames.is_cuda and frames.is_contiguous() and frames.dtype == torch.uint8 and frames.shape == (B, cv.S, sc.H, sc.W, 3)
        assert features.is_cuda and features.is_contiguous() and features.dtype == torch.bfloat16
        assert features.shape == (B, cv.Ho, cv.Wo, cv.C)
        stream = _stream_handle(stream, poses)
        _check(_lib.pxr_pipeline_step(self._h, poses.data_ptr(), None if shapes is None else shapes.data_ptr(), B,
                                      int(step0), int(env0), frames.data_ptr(), features.data_ptr(), stream))
        _written(torch, frames, features)
        return frames, features


_dtype_codes = {}


def _dtype_code(torch, dtype):
    if not _dtype_codes:
        _dtype_codes.update({torch.float32: 0, torch.bfloat16: 1})
    code = _dtype_codes.get(dtype)
    assert code is not None, f"float32 or bfloat16, not {dtype}"
    return code


def _empty(torch, like, stream, shape, dtype):
    """Device memory for a call's outputs and workspace.  On a stream of the caller's it comes from that stream's pool: the
    allocator may hand it out again as soon as it is let go, which is in order on that stream and on no other."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=like.device)):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _empty_like(torch, like, stream):
    """Device memory of a tensor's shape and type, contiguous (at less cost than _empty)."""
    if stream is None:
        return torch.empty_like(like) if like.is_contiguous() else torch.empty_like(like, memory_format=torch.contiguous_format)
    return _empty(torch, like, stream, like.shape, like.dtype)


def _rows(x):
    """Rows, width and the values from row to row of [..., D] (raises if there is no single such number)."""
    assert x.is_cuda and x.dim() >= 1 and x.shape[-1] > 0, "a CUDA tensor [..., width]"
    r = x if x.dim() == 2 else x.view(-1, x.shape[-1])
    n, width = r.shape
    step, inner = r.stride()
    assert inner == 1 or width == 1 or n == 0, "the values of a row must be adjacent"
    return n, width, step if n > 1 else width


def _params(torch, x, width, *params):
    """dtype of the weight and bias (those that there are), checked."""
    dtype = None
    for p in params:
        if p is not None:
            assert p.is_cuda and p.is_contiguous() and p.dim() == 1 and p.shape[0] == width, tuple(p.shape)
            assert p.dtype in (torch.float32, x.dtype) and dtype in (None, p.dtype), "weight and bias: both float32 or both of x's type"
            dtype = p.dtype
    return torch.float32 if dtype is None else dtype


def _ptr(x):
    return None if x is None else x.data_ptr()


def _here(torch, *tensors):
    """Tensors (and None) of the current GPU: a call's kernels go there, whatever its tensors are on."""
    device = torch._C._cuda_getDevice()
    for t in tensors:
        assert t is None or t.get_device() == device, f"a tensor of cuda:{t.get_device()}, and the current device is cuda:{device}"


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """x: CUDA float32 or bfloat16 [..., D] (rows a constant stride apart, their values adjacent); weight, bias: [D], float32
    or of x's type, or None.  Returns (y like x, mean, rstd: float32, x's leading shape), the latter two for
    layer_norm_backward; enqueue only."""
    torch = _torch or _torch_module()
    n, width, x_stride = _rows(x)
    dtype = x.dtype
    params = _params(torch, x, width, weight, bias)
    given = out is not None
    if out is None:
        out, y_stride = _empty_like(torch, x, stream), width
    else:
        assert out.is_cuda and out.dtype == dtype and out.shape == x.shape
        y_stride = _rows(out)[2]
    mean = _empty(torch, x, stream, x.shape[:-1], torch.float32)
    rstd = _empty_like(torch, mean, stream)
    d = _pack_norm(_dtype_code(torch, dtype), _dtype_code(torch, params), n, width, eps, x_stride, y_stride, width)
    _check((_lib or lib()).pxr_layer_norm_forward(d, x.data_ptr(), _ptr(weight), _ptr(bias), out.data_ptr(), mean.data_ptr(),
                                                  rstd.data_ptr(), _stream_handle(stream, x)))
    if given:
        _written(torch, out)
    return out, mean, rstd


_norm_asked = (None, 0)


def layer_norm_backward(dy, x, mean, rstd, weight=None, dx=None, params_dtype=None, stream=None):
    """Gradients of layer_norm for dy (x's shape and type), with the mean and rstd that it returned.  Returns (dx, dweight,
    dbias), the latter two [D] of the weight's type (without a weight: params_dtype, float32 unless given); enqueue only."""
    global _norm_asked
    torch = _torch or _torch_module()
    n, width, x_stride = _rows(x)
    dtype = x.dtype
    assert dy.dtype == dtype and dy.shape == x.shape
    dy_stride = _rows(dy)[2]
    for s in (mean, rstd):
        assert s.is_cuda and s.dtype == torch.float32 and s.is_contiguous() and s.numel() == n, "mean and rstd: one float32 for each row"
    params = _params(torch, x, width, weight) if weight is not None else params_dtype or torch.float32
    assert params in (torch.float32, dtype)
    given = dx is not None
    if dx is None:
        dx, dx_stride = _empty_like(torch, x, stream), width
    else:
        assert dx.is_cuda and dx.dtype == dtype and dx.shape == x.shape
        dx_stride = _rows(dx)[2]
    dweight = _empty(torch, x, stream, (width,), params)
    dbias = _empty_like(torch, dweight, stream)
    d = _pack_norm(_dtype_code(torch, dtype), _dtype_code(torch, params), n, width, 0.0, x_stride, dy_stride, dx_stride)
    L = _lib or lib()
    asked, need = _norm_asked  # (the bytes for the description that was asked for last are known)
    if asked != d:
        size = C.c_size_t()
        _check(L.pxr_layer_norm_workspace(d, size))
        need = size.value
        _norm_asked = (d, need)
    ws = _empty(torch, x, stream, (need,), torch.uint8) if need else None
    _check(L.pxr_layer_norm_backward(d, dy.data_ptr(), x.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _ptr(weight), dx.data_ptr(),
                                     dweight.data_ptr(), dbias.data_ptr(), _ptr(ws), need, _stream_handle(stream, x)))
    if given:
        _written(torch, dx)
    return dx, dweight, dbias


class LinearAttention:
    """Owns one pxr_linear_attention handle: a state [d_key, d_value] per environment and head that decays by
    exp(log_decay[h]) with every step, takes in k v^T and answers scale S^T q; cut where an episode begins."""

    def __init__(self, n_heads, d_key, d_value, log_decay, scale=None):
        """log_decay: n_heads natural logarithms, <= 0 (constants: no gradient); scale: d_key ** -0.5 unless given."""
        ld = np.ascontiguousarray(log_decay, dtype=np.float32)
        assert ld.shape == (n_heads,), ld.shape
        d = LinearAttentionDesc(int(n_heads), int(d_key), int(d_value), float(d_key ** -0.5 if scale is None else scale), ld.ctypes.data)
        h = C.c_void_p()
        _check(lib().pxr_linear_attention_create(C.byref(d), C.byref(h)))
        self._h = h
        self._asked = (None, 0)
        self.H, self.dk, self.dv, self.scale = int(n_heads), int(d_key), int(d_value), d.scale

    def close(self):
        if getattr(self, "_h", None):
            _check(lib().pxr_linear_attention_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _view(self, x, shape, dtype):
        """The fields of pxr_tokens for a [B, T, H, d] or (one step) [B, H, d] tensor of this shape and type."""
        assert x.is_cuda and x.dtype == dtype and x.shape == shape, (tuple(x.shape), shape, x.dtype)
        s = x.stride()
        assert s[-1] == 1 or shape[-1] == 1 or x.numel() == 0, "a head's values must be adjacent"
        return (x.data_ptr(), s[0], s[1], s[2]) if len(s) == 4 else (x.data_ptr(), s[0], 0, s[1])

    def _state(self, torch, state, B):
        assert state.is_cuda and state.dtype == torch.float32 and state.is_contiguous()
        assert state.shape == (B, self.H, self.dk, self.dv), tuple(state.shape)
        return state.data_ptr()

    def _rollout(self, torch, q, k, v, resets, state):
        """The bytes of pxr_rollout; the shapes of keys and of values; environments and steps."""
        keys, dtype = q.shape, q.dtype
        lead = keys[:-2]
        values = (*lead, self.H, self.dv)
        B, T = lead if len(lead) == 2 else (lead[0], 1)
        assert keys[-2] == self.H and keys[-1] == self.dk, (tuple(keys), self.H, self.dk)
        marks = (0, 0, 0)
        if resets is not None:
            assert resets.is_cuda and resets.dtype in (torch.bool, torch.uint8) and resets.shape == lead, tuple(resets.shape)
            s = resets.stride()
            marks = (resets.data_ptr(), s[0], s[1] if len(s) == 2 else 0)
        packed = _pack_rollout(_dtype_code(torch, dtype), B, T, *self._view(q, keys, dtype), *self._view(k, keys, dtype),
                               *self._view(v, values, dtype), *marks, 0 if state is None else self._state(torch, state, B))
        return packed, keys, values, B, T

    def _workspace(self, torch, like, B, T, backward, stream):
        sizes = (like.dtype, B, T, backward)
        asked, need = self._asked  # (the bytes for the sizes that were asked for last are known)
        if asked != sizes:
            n = C.c_size_t()
            _check(_lib.pxr_linear_attention_workspace(self._h, _dtype_code(torch, like.dtype), B, T, backward, n))
            need = n.value
            self._asked = (sizes, need)
        return _empty(torch, like, stream, (need,), torch.uint8) if need else None, need

    def forward(self, q, k, v, resets=None, state=None, out=None, state_out=None, stream=None):
        """q, k: CUDA float32 or bfloat16 [B,T,H,d_key], v: [B,T,H,d_value] (any strides, a head's values adjacent); resets:
        bool or uint8 [B,T], true where a step begins an episode, or None; state: float32 [B,H,d_key,d_value] before the
        first step, or None = zeros.  Returns (out [B,T,H,d_value], the state after the last step); enqueue only."""
        torch = _torch or _torch_module()
        assert q.dim() == 4
        r, keys, values, B, T = self._rollout(torch, q, k, v, resets, state)
        given = [t for t in (out, state_out) if t is not None]
        out = _empty_like(torch, v, stream) if out is None else out
        if state_out is None:
            state_out = (_empty(torch, q, stream, (B, self.H, self.dk, self.dv), torch.float32) if state is None else
                         _empty_like(torch, state, stream))
        ws, need = self._workspace(torch, q, B, T, 0, stream)
        _check(_lib.pxr_linear_attention_forward(self._h, r, _pack_tokens(*self._view(out, values, q.dtype)), self._state(torch, state_out, B),
                                                 _ptr(ws), need, _stream_handle(stream, q)))
        if given:
            _written(torch, *given)
        return out, state_out

    def backward(self, dout, q, k, v, resets=None, state=None, dstate=None, stream=None):
        """Gradients for dout [B,T,H,d_value] and dstate [B,H,d_key,d_value] (of the state after the last step, or None = zeros)
        of a forward call with these inputs.  Returns (dq, dk, dv, the gradient of the state before the first step or, where
        there was none, None); enqueue only."""
        torch = _torch or _torch_module()
        assert q.dim() == 4
        r, keys, values, B, T = self._rollout(torch, q, k, v, resets, state)
        dtype = q.dtype
        dq = _empty_like(torch, q, stream)
        dk, dv = _empty_like(torch, dq, stream), _empty_like(torch, v, stream)
        dfirst = None if state is None else _empty_like(torch, state, stream)
        ws, need = self._workspace(torch, q, B, T, 1, stream)
        _check(_lib.pxr_linear_attention_backward(
            self._h, r, _pack_tokens(*self._view(dout, values, dtype)), None if dstate is None else self._state(torch, dstate, B),
            _pack_tokens(*self._view(dq, keys, dtype)), _pack_tokens(*self._view(dk, keys, dtype)), _pack_tokens(*self._view(dv, values, dtype)),
            _ptr(dfirst), _ptr(ws), need, _stream_handle(stream, q)))
        return dq, dk, dv, dfirst

    def step(self, q, k, v, state, resets=None, out=None, stream=None):
        """One step of every environment: q, k [B,H,d_key], v [B,H,d_value], resets [B] or None; state float32
        [B,H,d_key,d_value] is updated in place (autograd is told).  Returns out [B,H,d_value]; enqueue only."""
        torch = _torch or _torch_module()
        assert q.dim() == 3
        r, _, values, B, _ = self._rollout(torch, q, k, v, resets, None)
        given = (state,) if out is None else (state, out)
        out = _empty_like(torch, v, stream) if out is None else out
        _check(_lib.pxr_linear_attention_step(self._h, r, self._state(torch, state, B), _pack_tokens(*self._view(out, values, q.dtype)),
                                              _stream_handle(stream, q)))
        _written(torch, *given)
        return out


class HeadNorm:
    """Owns one pxr_head_norm handle: each head of queries and keys is divided by its root mean square, multiplied by a weight, and
    the pairs (i, i + d_rotary / 2) of its first d_rotary values are turned by position * frequencies[i]."""

    def __init__(self, d_head, d_rotary=None, frequencies=None, base=10000.0, eps=1e-6):
        """d_rotary: even, all of d_head (or all but one) unless given, 0 = no rotation; frequencies: d_rotary / 2 radians a position,
        base ** (-2 i / d_rotary) unless given."""
        d_head = int(d_head)
        d_rotary = d_head // 2 * 2 if d_rotary is None else int(d_rotary)
        if frequencies is None:
            frequencies = [float(base) ** (-2 * i / d_rotary) for i in range(d_rotary // 2)]
        f = np.ascontiguousarray(frequencies, dtype=np.float64)
        assert f.shape == (d_rotary // 2,), f.shape
        d = HeadNormDesc(d_head, d_rotary, f.ctypes.data, float(eps))
        h = C.c_void_p()
        _check(lib().pxr_head_norm_create(C.byref(d), C.byref(h)))
        self._h = h
        self._device = _torch_module().cuda.current_device()  # that has the frequencies
        self._asked = (None, 0)
        self.d, self.rotary, self.eps = d_head, d_rotary, d.eps

    def close(self):
        if getattr(self, "_h", None):
            _check(lib().pxr_head_norm_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _view(self, x, shape, dtype):
        """The fields of pxr_tokens for a tensor of this shape and type, [B, T, H, d] or (one step) [B, H, d]."""
        assert x.is_cuda and x.dtype == dtype and x.shape == shape, (tuple(x.shape), tuple(shape), x.dtype)
        s = x.stride()
        assert s[-1] == 1 or shape[-1] == 1 or x.numel() == 0, "a head's values must be adjacent"
        return (x.data_ptr(), s[0], s[1], s[2]) if len(s) == 4 else (x.data_ptr(), s[0], 0, s[1])

    def _heads(self, torch, q, k, q_weight, k_weight, positions, first):
        """The bytes of pxr_heads; the shapes of q and of k; the heads' and the weights' type."""
        some = q if q is not None else k
        assert some is not None and some.dim() in (3, 4), "queries or keys [B, T, heads, d] or [B, heads, d]"
        dtype, shape = some.dtype, some.shape
        lead = shape[:-2]
        B, T = lead if len(shape) == 4 else (shape[0], 1)
        qs = ks = None
        qv = kv = (0, 0, 0, 0)
        if q is not None:
            qs = shape
            assert qs[-1] == self.d, (tuple(qs), self.d)
            qv = self._view(q, qs, dtype)
        if k is not None:
            ks = k.shape
            assert ks[:-2] == lead and ks[-1] == self.d, (tuple(ks), tuple(shape))
            kv = self._view(k, ks, dtype)
        params = torch.float32 if q_weight is None and k_weight is None else _params(torch, some, self.d, q_weight, k_weight)
        bits, at, at_env, at_step = 32, 0, 0, 0
        if positions is not None:
            kind = positions.dtype
            assert positions.is_cuda and kind in (torch.int32, torch.int64) and positions.shape == lead, tuple(positions.shape)
            assert first == 0, "positions say where every step is"
            s = positions.stride()
            at, at_env, at_step, bits = positions.data_ptr(), s[0], s[1] if len(s) == 2 else 0, 64 if kind == torch.int64 else 32
        packed = _pack_heads(_dtype_code(torch, dtype), _dtype_code(torch, params), B, T, 0 if qs is None else qs[-2], 0 if ks is None else ks[-2], *qv, *kv,
                             _ptr(q_weight) or 0, _ptr(k_weight) or 0, at, bits, at_env, at_step, first)
        return packed, qs, ks, dtype, params

    def _check_device(self, torch, *tensors):
        _here(torch, *tensors)
        assert self._device == torch._C._cuda_getDevice(), f"a layer of cuda:{self._device}"

    def _new(self, torch, x, shape, stream):
        """A contiguous tensor like x, and its pxr_tokens."""
        out = _empty_like(torch, x, stream)
        H, d = shape[-2:]
        return out, _pack_tokens(out.data_ptr(), (shape[1] if len(shape) == 4 else 1) * H * d, H * d, d)

    def forward(self, q, k, q_weight=None, k_weight=None, positions=None, first=0, q_out=None, k_out=None, stream=None):
        """q, k: CUDA float32 or bfloat16 [B,T,H,d] (or, one step, [B,H,d]; any strides, a head's values adjacent; the numbers of heads may
        differ, either may be None); weights: [d], float32 or of their type, or None; positions: int32 or int64 [B,T] (one step:
        [B]), or None: step t is at first + t.  Returns (q, k) normalised and turned, in q_out and k_out if given (they may be
        the inputs themselves); enqueue only."""
        torch = _torch or _torch_module()
        r, qs, ks, dtype, _ = self._heads(torch, q, k, q_weight, k_weight, positions, first)
        self._check_device(torch, q, k, q_weight, k_weight, positions, q_out, k_out)
        to_q = to_k = None
        given = [t for t in (q_out, k_out) if t is not None]
        if q_out is not None:
            assert q is not None
            to_q = _pack_tokens(*self._view(q_out, qs, dtype))
        elif q is not None:
            q_out, to_q = self._new(torch, q, qs, stream)
        if k_out is not None:
            assert k is not None
            to_k = _pack_tokens(*self._view(k_out, ks, dtype))
        elif k is not None:
            k_out, to_k = self._new(torch, k, ks, stream)
        _check(_lib.pxr_head_norm_forward(self._h, r, to_q, to_k, _stream_handle(stream, q if q is not None else k)))
        if given:
            _written(torch, *given)
        return q_out, k_out

    def backward(self, dq, dk, q, k, q_weight=None, k_weight=None, positions=None, first=0, params_dtype=None, stream=None):
        """Gradients for dq and dk (of the outputs) of a forward call with these inputs.  Returns (of q, of k, of q_weight, of k_weight), the latter two [d] of the
        weights' type (without weights: params_dtype, float32 unless given); None in the place of what is of no heads; enqueue only."""
        torch = _torch or _torch_module()
        r, qs, ks, dtype, params = self._heads(torch, q, k, q_weight, k_weight, positions, first)
        self._check_device(torch, q, k, q_weight, k_weight, positions, dq, dk)
        some = q if q is not None else k
        if q_weight is None and k_weight is None and params_dtype is not None:
            assert params_dtype in (torch.float32, dtype)
            params = params_dtype
            r = r[:4] + struct.pack("@I", _dtype_code(torch, params)) + r[8:]
        grads, sums, given, into = [None, None], [None, None], [None, None], [None, None]
        for i, (x, d, shape) in enumerate(((q, dq, qs), (k, dk, ks))):
            if x is not None:
                given[i] = _pack_tokens(*self._view(d, shape, dtype))
                grads[i], into[i] = self._new(torch, x, shape, stream)
                sums[i] = _empty(torch, x, stream, (self.d,), params)
        sizes = r[:24]
        asked, need = self._asked  # (the bytes for the sizes that were asked for last are known)
        if asked != sizes:
            n = C.c_size_t()
            _check(_lib.pxr_head_norm_workspace(self._h, r, n))
            need = n.value
            self._asked = (sizes, need)
        ws = _empty(torch, some, stream, (need,), torch.uint8) if need else None
        _check(_lib.pxr_head_norm_backward(self._h, r, *given, *into, *(_ptr(s) for s in sums), _ptr(ws), need, _stream_handle(stream, some)))
        return (*grads, *sums)


def _steps_view(x, shape, dtype):
    """The fields of pxr_steps for a [B, T, D] or (one step) [B, D] tensor of this shape and type."""
    assert x.is_cuda and x.dtype == dtype and x.shape == shape, (tuple(x.shape), tuple(shape), x.dtype)
    s = x.stride()
    assert s[-1] == 1 or shape[-1] == 1 or x.numel() == 0, "a step's values must be adjacent"
    return (x.data_ptr(), s[0], s[1]) if len(s) == 3 else (x.data_ptr(), s[0], 0)


def _channels(torch, state, B, D):
    assert state.is_cuda and state.dtype == torch.float32 and state.is_contiguous() and state.shape == (B, D), tuple(state.shape)
    return state.data_ptr()


def _gated_rollout(torch, x, gate, resets, state, coupled):
    """The bytes of pxr_gated_rollout; environments, steps and channels."""
    shape, dtype = x.shape, x.dtype
    B, T, D = shape if len(shape) == 3 else (shape[0], 1, shape[1])
    marks = (0, 0, 0)
    if resets is not None:
        assert resets.is_cuda and resets.dtype in (torch.bool, torch.uint8) and resets.shape == shape[:-1], tuple(resets.shape)
        s = resets.stride()
        marks = (resets.data_ptr(), s[0], s[1] if len(s) == 2 else 0)
    packed = _pack_gated(_dtype_code(torch, dtype), B, T, D, 1 if coupled else 0, *_steps_view(x, shape, dtype), *_steps_view(gate, shape, dtype),
                         *marks, 0 if state is None else _channels(torch, state, B, D))
    return packed, B, T, D


_gated_asked = (None, 0)


def _gated_workspace(torch, like, B, T, D, backward, stream):
    global _gated_asked
    sizes = (B, T, D, backward)
    asked, need = _gated_asked  # (the bytes for the sizes that were asked for last are known)
    if asked != sizes:
        n = C.c_size_t()
        _check((_lib or lib()).pxr_gated_recurrence_workspace(B, T, D, backward, n))
        need = n.value
        _gated_asked = (sizes, need)
    return _empty(torch, like, stream, (need,), torch.uint8) if need else None, need


def gated_recurrence(x, gate, resets=None, state=None, coupled=True, out=None, state_out=None, stream=None):
    """h_t = (an episode begins ? 0 : a h_{t-1}) + (coupled ? 1 - a : 1) x_t with a = 1 / (1 + exp(-gate_t)), for each environment
    and channel.  x, gate: CUDA float32 or bfloat16 [B,T,D] (any strides, a step's values adjacent); resets: bool or uint8
    [B,T], true where a step begins an episode, or None; state: float32 [B,D] before the first step, or None = zeros.  out must not
    overlap an input.  Returns (out [B,T,D], the state after the last step); enqueue only."""
    torch = _torch or _torch_module()
    assert x.dim() == 3
    r, B, T, D = _gated_rollout(torch, x, gate, resets, state, coupled)
    _here(torch, x, gate, resets, state, out, state_out)
    given = [t for t in (out, state_out) if t is not None]
    out = _empty_like(torch, x, stream) if out is None else out
    if state_out is None:
        state_out = _empty(torch, x, stream, (B, D), torch.float32) if state is None else _empty_like(torch, state, stream)
    ws, need = _gated_workspace(torch, x, B, T, D, 0, stream)
    _check((_lib or lib()).pxr_gated_recurrence_forward(r, _pack_steps(*_steps_view(out, x.shape, x.dtype)), _channels(torch, state_out, B, D),
                                                        _ptr(ws), need, _stream_handle(stream, x)))
    if given:
        _written(torch, *given)
    return out, state_out


def gated_recurrence_backward(dout, x, gate, resets=None, state=None, dstate=None, coupled=True, stream=None):
    """Gradients for dout [B,T,D] and dstate [B,D] (of the state after the last step, or None = zeros) of a gated_recurrence call
    with these inputs.  Returns (dx, dgate, the gradient of the state before the first step or, where there was none, None);
    enqueue only."""
    torch = _torch or _torch_module()
    assert x.dim() == 3
    r, B, T, D = _gated_rollout(torch, x, gate, resets, state, coupled)
    _here(torch, dout, x, gate, resets, state, dstate)
    dx = _empty_like(torch, x, stream)
    dgate = _empty_like(torch, dx, stream)
    dfirst = None if state is None else _empty_like(torch, state, stream)
    ws, need = _gated_workspace(torch, x, B, T, D, 1, stream)
    _check((_lib or lib()).pxr_gated_recurrence_backward(
        r, _pack_steps(*_steps_view(dout, x.shape, x.dtype)), None if dstate is None else _channels(torch, dstate, B, D),
        _pack_steps(*_steps_view(dx, x.shape, x.dtype)), _pack_steps(*_steps_view(dgate, x.shape, x.dtype)), _ptr(dfirst), _ptr(ws), need,
        _stream_handle(stream, x)))
    return dx, dgate, dfirst


def gated_recurrence_step(x, gate, state, resets=None, coupled=True, out=None, stream=None):
    """One step of every environment: x, gate [B,D], resets [B] or None; state float32 [B,D] is updated in place (autograd is
    told); out may be x or gate itself.  Returns out [B,D]; enqueue only."""
    torch = _torch or _torch_module()
    assert x.dim() == 2
    r, B, _, D = _gated_rollout(torch, x, gate, resets, None, coupled)
    _here(torch, x, gate, state, resets, out)
    given = (state,) if out is None else (state, out)
    out = _empty_like(torch, x, stream) if out is None else out
    _check((_lib or lib()).pxr_gated_recurrence_step(r, _channels(torch, state, B, D), _pack_steps(*_steps_view(out, x.shape, x.dtype)),
                                                     _stream_handle(stream, x)))
    _written(torch, *given)
    return out


# A step that takes singular values from nearly nothing to about one within five.
ORTHOGONALISE_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
_coefficients = (None, None, None)


def _steps_of(coefficients, steps):
    """float32 [n][3] for one triple, taken `steps` times (5 unless given), or for a triple for each step."""
    global _coefficients
    known, n, array = _coefficients  # (those of the call before, most often)
    plain = type(coefficients) is tuple and all(type(c) is float for c in coefficients)
    if not plain or known != coefficients or n != steps:
        array = np.asarray(coefficients, np.float32)
        if array.ndim == 1:
            array = np.tile(array, (5 if steps is None else int(steps), 1))
        assert array.ndim == 2 and array.shape[1] == 3 and (steps is None or array.shape[0] == steps), "a triple, or one for each step"
        array = np.ascontiguousarray(array)
        if plain:
            _coefficients = (coefficients, steps, array)
    return array


_orthogonalise_asked = (None, 0)


def orthogonalise_workspace(n_matrices, rows, cols, dtype=None, steps=None, coefficients=ORTHOGONALISE_COEFFICIENTS, eps=1e-7):
    """Bytes of workspace of an orthogonalise call on n_matrices [rows, cols] (float32 unless dtype says otherwise); raises what that call would refuse of its sizes
    and steps.  Host only."""
    torch = _torch or _torch_module()
    c = _steps_of(coefficients, steps)
    n = C.c_size_t()
    _check(lib().pxr_orthogonalise_workspace(_pack_orthogonalise(0 if dtype is None else _dtype_code(torch, dtype), n_matrices, rows, cols, rows * cols, cols, rows * cols, cols,
                                                                 c.shape[0], c.ctypes.data, eps), n))
    return n.value


def orthogonalise(x, steps=None, coefficients=ORTHOGONALISE_COEFFICIENTS, eps=1e-7, out=None, stream=None):
    """A learner's update [m,n], or several [B,m,n], CUDA float32 or bfloat16 (rows at any stride, their values adjacent), with its
    singular values pushed towards one: X = x / (|x| + eps), then for each step X <- a X + (b A + c A^2) X with A = X X^T (of the
    transpose where m > n).  coefficients: (a, b, c), taken `steps` times (5 unless given), or a triple for each step.
    Returns the result like x (out may be x); enqueue only."""
    global _orthogonalise_asked
    torch = _torch or _torch_module()
    shape, s = x.shape, x.stride()
    assert x.is_cuda and len(shape) in (2, 3) and shape[-2] > 0 and shape[-1] > 0, "a CUDA tensor [m,n] or [B,m,n]"
    assert s[-1] == 1 or shape[-1] == 1, "the values of a row must be adjacent"
    _here(torch, x, out)
    given = out is not None
    if out is None:
        out = _empty_like(torch, x, stream)
    else:
        assert out.is_cuda and out.dtype == x.dtype and out.shape == shape and (out.stride(-1) == 1 or shape[-1] == 1)
    t = out.stride()
    c = _steps_of(coefficients, steps)
    B = shape[0] if len(shape) == 3 else 1
    d = _pack_orthogonalise(_dtype_code(torch, x.dtype), B, shape[-2], shape[-1], s[0] if len(s) == 3 else 0, s[-2], t[0] if len(t) == 3 else 0, t[-2],
                            c.shape[0], c.ctypes.data, eps)
    L = _lib or lib()
    sizes = d[:16] + c.tobytes()
    asked, need = _orthogonalise_asked  # (the bytes for the sizes and steps that were asked for last are known)
    if asked != sizes:
        n = C.c_size_t()
        _check(L.pxr_orthogonalise_workspace(d, n))
        need = n.value
        _orthogonalise_asked = (sizes, need)
    ws = _empty(torch, x, stream, (need,), torch.uint8) if need else None
    _check(L.pxr_orthogonalise(d, x.data_ptr(), out.data_ptr(), _ptr(ws), need, _stream_handle(stream, x)))
    if given:
        _written(torch, out)
    return out


def make_skeleton_desc(skel, n_free, n_angles):
    """dict(parent, slot, anchor, axis, offset) -> (SkeletonDesc, keep-alive list)."""
    parent = np.ascontiguousarray(skel["parent"], dtype=np.int32)
    slot = np.ascontiguousarray(skel["slot"], dtype=np.int32)
    arrs = [np.ascontiguousarray(skel[k], dtype=np.float32).reshape(-1) for k in ("anchor", "axis", "offset")]
    K = parent.shape[0]
    assert slot.shape == (K,) and all(a.shape == (K * 3,) for a in arrs)
    d = SkeletonDesc()
    d.n_bodies, d.n_free, d.n_angles = K, int(n_free), int(n_angles)
    d.parent, d.slot = parent.ctypes.data, slot.ctypes.data
    d.anchor, d.axis, d.offset = (a.ctypes.data for a in arrs)
    return d, [parent, slot] + arrs


def selftest_arithmetic():
    """pxr_selftest_arithmetic: dict(recip_mismatches, floor_mismatches, recip_checked, floor_checked) on the current device."""
    c = (C.c_uint64 * 4)()
    _check(lib().pxr_selftest_arithmetic(c))
    return dict(recip_mismatches=int(c[0]), floor_mismatches=int(c[1]), recip_checked=int(c[2]), floor_checked=int(c[3]))


def measure_peaks():
    """pxr_measure_peaks: dict(fma_tlaneops, imad_tlaneops, copy_gbs, read_gbs, write_gbs) measured on the current device."""
    v = [C.c_double() for _ in range(5)]
    _check(lib().pxr_measure_peaks(*[C.byref(x) for x in v]))
    return dict(zip(("fma_tlaneops", "imad_tlaneops", "copy_gbs", "read_gbs", "write_gbs"), (x.value for x in v)))


def ids_to_numpy(ids):
    """int32 CUDA tensor holding uint32 id bits -> numpy uint32."""
    return ids.cpu().numpy().view(np.uint32)
