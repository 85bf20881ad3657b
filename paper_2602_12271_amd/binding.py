"""Thin ctypes binding over libmonarchrt.so (the C ABI in include/monarchrt.h).

Argument marshalling only: PyTorch supplies device memory and the HIP stream, every
step of the operator runs in the library's kernels.  There is no CPU fallback: a
missing library raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import NamedTuple, Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmonarchrt.so")

MRT_OK = 0
MRT_ERR_NULL, MRT_ERR_SHAPE, MRT_ERR_BLOCK, MRT_ERR_UNSUPPORTED, MRT_ERR_WORKSPACE, MRT_ERR_HIP = range(1, 7)
MRT_F32, MRT_BF16 = 0, 1
MRT_COMPUTE_DEFAULT, MRT_COMPUTE_F32 = 0, 1

EXPORTED = [
    "monarch_attn_check", "monarch_attn_workspace_min_bytes", "monarch_attn_workspace_bytes",
    "monarch_attn_fwd", "dense_attn_check", "dense_attn_fwd", "mrt_status_string", "mrt_last_error",
    "mrt_profile_enable", "mrt_profile_read", "mrt_set_head_groups",
    "monarch_attn_bwd", "monarch_attn_bwd_workspace_bytes", "monarch_attn_bwd_workspace_min_bytes",
    "monarch_attn_fwd_noalloc",
    "monarch_attn_bwd_saved_workspace_bytes", "monarch_attn_fwd_save", "monarch_attn_bwd_saved",
    "dense_attn_workspace_bytes", "dense_attn_fwd_ws",
    "dense_attn_fwd_save", "dense_attn_fwd_save_workspace_bytes", "dense_attn_fwd_save_queries", "dense_attn_bwd", "dense_attn_bwd_check", "dense_attn_bwd_workspace_bytes",
    "mrt_rotary_check", "mrt_rotary_fwd", "mrt_rotary_bwd",
    "mrt_norm_rotary_check", "mrt_norm_rotary_fwd", "mrt_norm_rotary_bwd", "mrt_norm_rotary_bwd_workspace_bytes",
    "mrt_cache8_check", "mrt_cache8_write", "mrt_cache8_read",
    "dense_attn_cache8_check", "dense_attn_fwd_cache8", "dense_attn_fwd_cache8_workspace_bytes",
]
NOALLOC_SCRATCH_BYTES = 128 << 20
ASSIGNMENTS = {"fh_w": 0, "w_fh": 1, "fw_h": 2, "h_fw": 3, "f_hw": 4, "hw_f": 5}
KERNEL_STAGE_R, KERNEL_STAGE_L, KERNEL_DENSE, KERNEL_FIRST, KERNEL_LAST = 1, 2, 4, 16, 32
KERNEL_DENSE_BWD, KERNEL_ROTARY, KERNEL_CACHE = 8, 64, 128
ROTARY_LAYOUTS = {"adjacent": 0, "halves": 1}
ROTARY_LADDERS = {"axis": 0, "shared": 1}


class MrtStrides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_longlong), ("head", ctypes.c_longlong), ("token", ctypes.c_longlong)]


class MrtProblem(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int),
        ("f_q", ctypes.c_int), ("f_kv", ctypes.c_int), ("h", ctypes.c_int), ("w", ctypes.c_int),
        ("q_frame_offset", ctypes.c_int),
        ("q", MrtStrides), ("k", MrtStrides), ("v", MrtStrides), ("o", MrtStrides),
        ("dtype", ctypes.c_int), ("compute", ctypes.c_int), ("scale", ctypes.c_float),
        ("assignment", ctypes.c_int), ("tile_h", ctypes.c_int), ("head_groups", ctypes.c_int),
    ]


class MrtDenseTrain(ctypes.Structure):
    _fields_ = [("kv_heads", ctypes.c_int), ("kv_len", ctypes.c_void_p),
                ("dout", MrtStrides), ("dq", MrtStrides), ("dk", MrtStrides), ("dv", MrtStrides)]


class MrtRotary(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int), ("pairs", ctypes.c_int * 3), ("layout", ctypes.c_int),
                ("ladder", ctypes.c_int), ("theta", ctypes.c_double)]


class MrtRotaryTensor(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("heads", ctypes.c_int), ("f", ctypes.c_int), ("h", ctypes.c_int),
                ("w", ctypes.c_int), ("frame_offset", ctypes.c_int), ("x", MrtStrides), ("y", MrtStrides),
                ("x_dtype", ctypes.c_int), ("y_dtype", ctypes.c_int), ("positions", ctypes.c_void_p),
                ("position_batch", ctypes.c_longlong), ("position_axis", ctypes.c_longlong)]


class MrtNormTensor(ctypes.Structure):
    _fields_ = [("t", MrtRotaryTensor), ("weight", ctypes.c_void_p), ("weight_dtype", ctypes.c_int),
                ("weight_head", ctypes.c_longlong), ("dx", MrtStrides), ("dweight", ctypes.c_void_p)]


class MrtCache8(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("capacity", ctypes.c_int),
                ("block", ctypes.c_int), ("format", ctypes.c_int), ("k", MrtStrides), ("v", MrtStrides),
                ("k_scale_batch", ctypes.c_longlong), ("k_scale_head", ctypes.c_longlong),
                ("v_scale_batch", ctypes.c_longlong), ("v_scale_head", ctypes.c_longlong),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class MrtCache8Rows(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int), ("at", ctypes.c_int), ("at_each", ctypes.c_void_p), ("tokens_each", ctypes.c_void_p),
                ("k", MrtStrides), ("v", MrtStrides), ("dtype", ctypes.c_int)]


class MrtError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"monarchrt status {status}: {text}")
        self.status = status


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2602_12271_amd.build). "
            "There is no fallback path.")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(MrtProblem)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.monarch_attn_check.argtypes = [P, ci, ci, ci, ci, ci]
    lib.monarch_attn_check.restype = ci
    lib.monarch_attn_workspace_min_bytes.argtypes = [P, ci, ci, ci, ci]
    lib.monarch_attn_workspace_min_bytes.restype = sz
    lib.monarch_attn_workspace_bytes.argtypes = [P, ci, ci, ci, ci]
    lib.monarch_attn_workspace_bytes.restype = sz
    lib.monarch_attn_fwd.argtypes = [vp, vp, vp, vp, P, ci, ci, ci, ci, ci, vp, sz, vp]
    lib.monarch_attn_fwd.restype = ci
    lib.monarch_attn_fwd_noalloc.argtypes = [vp, vp, vp, vp, P, ci, ci, ci, ci, ci, vp]
    lib.monarch_attn_fwd_noalloc.restype = ci
    fp = ctypes.c_void_p
    lib.monarch_attn_bwd_workspace_min_bytes.argtypes = [P, ci, ci, ci, ci]
    lib.monarch_attn_bwd_workspace_min_bytes.restype = sz
    lib.monarch_attn_bwd_workspace_bytes.argtypes = [P, ci, ci, ci, ci]
    lib.monarch_attn_bwd_workspace_bytes.restype = sz
    lib.monarch_attn_bwd.argtypes = [vp, vp, vp, vp, fp, fp, fp, P, ci, ci, ci, ci, ci, vp, sz, vp]
    lib.monarch_attn_bwd.restype = ci
    lib.monarch_attn_bwd_saved_workspace_bytes.argtypes = [P, ci, ci, ci, ci]
    lib.monarch_attn_bwd_saved_workspace_bytes.restype = sz
    lib.monarch_attn_fwd_save.argtypes = [vp, vp, vp, vp, P, ci, ci, ci, ci, ci, vp, sz, vp]
    lib.monarch_attn_fwd_save.restype = ci
    lib.monarch_attn_bwd_saved.argtypes = [vp, vp, vp, vp, fp, fp, fp, P, ci, ci, ci, ci, ci, vp, sz, vp]
    lib.monarch_attn_bwd_saved.restype = ci
    lib.dense_attn_check.argtypes = [P, ci]
    lib.dense_attn_check.restype = ci
    lib.dense_attn_fwd.argtypes = [vp, vp, vp, vp, P, ci, vp]
    lib.dense_attn_fwd.restype = ci
    lib.dense_attn_workspace_bytes.argtypes = [P, ci]
    lib.dense_attn_workspace_bytes.restype = sz
    lib.dense_attn_fwd_ws.argtypes = [vp, vp, vp, vp, P, ci, vp, sz, vp]
    lib.dense_attn_fwd_ws.restype = ci
    T = ctypes.POINTER(MrtDenseTrain)
    lib.dense_attn_fwd_save.argtypes = [vp, vp, vp, vp, vp, P, T, ci, vp, sz, vp]
    lib.dense_attn_fwd_save.restype = ci
    lib.dense_attn_fwd_save_workspace_bytes.argtypes = [P, T, ci]
    lib.dense_attn_fwd_save_workspace_bytes.restype = sz
    lib.dense_attn_fwd_save_queries.argtypes = [P, T, ci, sz]
    lib.dense_attn_fwd_save_queries.restype = ci
    lib.dense_attn_bwd_check.argtypes = [P, T, ci]
    lib.dense_attn_bwd_check.restype = ci
    lib.dense_attn_bwd_workspace_bytes.argtypes = [P, T, ci]
    lib.dense_attn_bwd_workspace_bytes.restype = sz
    lib.dense_attn_bwd.argtypes = [vp] * 9 + [P, T, ci, vp, sz, vp]
    lib.dense_attn_bwd.restype = ci
    R, X = ctypes.POINTER(MrtRotary), ctypes.POINTER(MrtRotaryTensor)
    lib.mrt_rotary_check.argtypes = [R, X, ci]
    lib.mrt_rotary_check.restype = ci
    for f in (lib.mrt_rotary_fwd, lib.mrt_rotary_bwd):
        f.argtypes = [R, X, ci, vp, vp, vp]
        f.restype = ci
    N = ctypes.POINTER(MrtNormTensor)
    cd = ctypes.c_double
    lib.mrt_norm_rotary_check.argtypes = [R, cd, N, ci, ci]
    # (descriptions with a call's addresses are bytes that a struct.Struct has packed: 0.4 us where fields one by one take 1)
    lib.mrt_norm_rotary_fwd.argtypes = [R, cd, vp, ci, vp, vp, vp]
    lib.mrt_norm_rotary_bwd.argtypes = [R, cd, vp, ci, vp, vp, vp, vp, sz, vp]
    lib.mrt_norm_rotary_bwd_workspace_bytes.argtypes = [R, vp, ci]
    lib.mrt_norm_rotary_bwd_workspace_bytes.restype = sz
    C, W = ctypes.POINTER(MrtCache8), ctypes.POINTER(MrtCache8Rows)
    lib.mrt_cache8_check.argtypes = [C, W]
    lib.mrt_cache8_write.argtypes = lib.mrt_cache8_read.argtypes = [vp, vp, vp, vp, vp]
    lib.dense_attn_cache8_check.argtypes = [P, C, ci]
    lib.dense_attn_fwd_cache8_workspace_bytes.argtypes = [P, vp, ci]
    lib.dense_attn_fwd_cache8_workspace_bytes.restype = sz
    lib.dense_attn_fwd_cache8.argtypes = [vp, vp, vp, vp, P, vp, ci, vp, sz, vp]
    for f in (lib.mrt_norm_rotary_check, lib.mrt_norm_rotary_fwd, lib.mrt_norm_rotary_bwd, lib.mrt_cache8_check,
              lib.mrt_cache8_write, lib.mrt_cache8_read, lib.dense_attn_cache8_check, lib.dense_attn_fwd_cache8):
        f.restype = ci
    lib.mrt_status_string.argtypes = [ci]
    lib.mrt_status_string.restype = ctypes.c_char_p
    lib.mrt_last_error.argtypes = []
    lib.mrt_last_error.restype = ctypes.c_char_p
    lib.mrt_set_head_groups.argtypes = [ci]
    lib.mrt_set_head_groups.restype = None
    lib.mrt_profile_enable.argtypes = [ci]
    lib.mrt_profile_enable.restype = None
    lib.mrt_profile_read.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ci), ci]
    lib.mrt_profile_read.restype = ci
    _lib = lib
    return lib


def _raise(lib, st: int):
    raise MrtError(st, f"{lib.mrt_status_string(st).decode()}: {lib.mrt_last_error().decode()}")


def make_problem(*, batch, heads, head_dim, f_q, f_kv, h, w, q_frame_offset=0, dtype=MRT_BF16,
                 compute=MRT_COMPUTE_DEFAULT, scale=1.0, q_strides=None, k_strides=None,
                 v_strides=None, o_strides=None, assign="fh_w", tile_h=0, head_groups=0) -> MrtProblem:
    """Problem descriptor; default strides are those of contiguous [batch, heads, tokens, d]."""
    nq, nkv = f_q * h * w, f_kv * h * w

    def contiguous(n):
        return (heads * n * head_dim, n * head_dim, head_dim)
    qs, ks = q_strides or contiguous(nq), k_strides or contiguous(nkv)
    vs, os_ = v_strides or contiguous(nkv), o_strides or contiguous(nq)
    return MrtProblem(batch, heads, head_dim, f_q, f_kv, h, w, q_frame_offset,
                      MrtStrides(*qs), MrtStrides(*ks), MrtStrides(*vs), MrtStrides(*os_),
                      dtype, compute, scale, assign if isinstance(assign, int) else ASSIGNMENTS[assign],
                      tile_h, head_groups)


def monarch_attn_check(prob: MrtProblem, b1, b2, tile, iters, causal_chunk=0) -> int:
    return load_library().monarch_attn_check(ctypes.byref(prob), b1, b2, tile, iters, causal_chunk)


def dense_attn_check(prob: MrtProblem, causal_chunk=0) -> int:
    return load_library().dense_attn_check(ctypes.byref(prob), causal_chunk)


def last_error() -> str:
    return load_library().mrt_last_error().decode()


def monarch_attn_workspace_bytes(prob: MrtProblem, b1, b2, tile, iters, minimum=False) -> int:
    lib = load_library()
    f = lib.monarch_attn_workspace_min_bytes if minimum else lib.monarch_attn_workspace_bytes
    return int(f(ctypes.byref(prob), b1, b2, tile, iters))


def set_head_groups(n: int) -> None:
    load_library().mrt_set_head_groups(int(n))


def profile_enable(repeats) -> None:
    """0/False: off; r >= 1: every launch is issued r times inside one event bracket."""
    load_library().mrt_profile_enable(int(repeats))


def profile_read(capacity: int = 65536):
    """[(milliseconds, kernel kind)] of the launches recorded since the last read."""
    ms = (ctypes.c_float * capacity)()
    kind = (ctypes.c_int * capacity)()
    n = load_library().mrt_profile_read(ms, kind, capacity)
    return [(ms[i], kind[i]) for i in range(n)]


# ---- torch-facing helpers ------------------------------------------------------------
def _torch_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign="fh_w", tile_h=0,
                   head_groups=0):
    import torch
    assert Q.dim() == 4 and K.dim() == 4 and V.dim() == 4
    assert Q.is_cuda and K.is_cuda and V.is_cuda and O.is_cuda
    assert Q.dtype == K.dtype == V.dtype == O.dtype
    dt = {torch.float32: MRT_F32, torch.bfloat16: MRT_BF16}[Q.dtype]
    B, H, nq, d = Q.shape
    assert K.shape == (B, H, f_kv * h * w, d) and V.shape == K.shape and nq == f_q * h * w
    assert O.shape == Q.shape
    for t in (Q, K, V, O):
        assert t.stride(3) == 1, "head_dim must be contiguous"

    def st(t):
        return (t.stride(0), t.stride(1), t.stride(2))
    return make_problem(batch=B, heads=H, head_dim=d, f_q=f_q, f_kv=f_kv, h=h, w=w,
                        q_frame_offset=q_frame_offset, dtype=dt, compute=compute, scale=scale,
                        q_strides=st(Q), k_strides=st(K), v_strides=st(V), o_strides=st(O),
                        assign=assign, tile_h=tile_h, head_groups=head_groups)


# Problem descriptors of recent calls, by the VALUES they are built from (shapes, strides, types and
# arguments, never a tensor's identity): a decoding loop describes the same problem on every call, and
# building and checking the descriptor took 5 of the 10 microseconds a small call spent in Python.
# Read-only once built; bounded.
_problems: dict = {}
_MAX_PROBLEMS = 256


def _call_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign="fh_w", tile_h=0,
                  head_groups=0):
    if not (type(f_q) is type(f_kv) is type(h) is type(w) is type(q_frame_offset) is type(compute) is type(tile_h)
            is type(head_groups) is int and type(scale) is float and type(assign) is str):   # (others: no key to trust)
        return _torch_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h, head_groups)
    key = (Q.shape, Q.stride(), Q.dtype, Q.is_cuda, K.shape, K.stride(), K.dtype, K.is_cuda,
           V.shape, V.stride(), V.dtype, V.is_cuda, O.shape, O.stride(), O.dtype, O.is_cuda,
           f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h, head_groups)
    prob = _problems.get(key)
    if prob is None:
        prob = _torch_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h, head_groups)
        if len(_problems) >= _MAX_PROBLEMS:
            _problems.clear()
        _problems[key] = prob
    return prob


def _stream_of(Q, stream):
    """The stream the call runs on: the caller's, or the current one of Q's device."""
    if stream is not None:
        return stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # 0.06 us; the public way takes 1.9
    return raw(Q.get_device()) if raw is not None else torch.cuda.current_stream(Q.device).cuda_stream


def monarch_attn_fwd(Q, K, V, *, f_q, f_kv, h, w, b1, b2, tile, iters, causal_chunk=0,
                     q_frame_offset=0, scale=1.0, compute=MRT_COMPUTE_DEFAULT, out=None,
                     workspace=None, stream=None, assign="fh_w", tile_h=0, head_groups=0):
    """MonarchRT attention forward on device tensors [batch, heads, tokens, head_dim]."""
    import torch
    lib = load_library()
    O = torch.empty_like(Q) if out is None else out
    prob = _call_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h,
                         head_groups)
    if workspace is None:
        nbytes = lib.monarch_attn_workspace_bytes(ctypes.byref(prob), b1, b2, tile, iters)
        if nbytes == 0:
            _raise(lib, lib.monarch_attn_check(ctypes.byref(prob), b1, b2, tile, iters, causal_chunk))
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
    s = _stream_of(Q, stream)
    st = lib.monarch_attn_fwd(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(),
                              ctypes.byref(prob), b1, b2, tile, iters, causal_chunk,
                              workspace.data_ptr(), workspace.numel() * workspace.element_size(), s)
    if st != MRT_OK:
        _raise(lib, st)
    return O


def monarch_attn_fwd_noalloc(Q, K, V, out, *, f_q, f_kv, h, w, b1, b2, tile, iters, causal_chunk=0,
                             q_frame_offset=0, scale=1.0, compute=MRT_COMPUTE_DEFAULT, stream=None,
                             assign="fh_w", tile_h=0):
    """monarch_attn_fwd on the library's built-in scratch memory: the call allocates nothing, so the
    output tensor must be passed in."""
    import torch
    lib = load_library()
    prob = _call_problem(Q, K, V, out, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h)
    s = _stream_of(Q, stream)
    st = lib.monarch_attn_fwd_noalloc(Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(),
                                      ctypes.byref(prob), b1, b2, tile, iters, causal_chunk, s)
    if st != MRT_OK:
        _raise(lib, st)
    return out


def monarch_attn_bwd(Q, K, V, dO, *, f_q, f_kv, h, w, b1, b2, tile, iters, causal_chunk=0,
                     q_frame_offset=0, scale=1.0, workspace=None, stream=None, assign="fh_w", tile_h=0,
                     compute=MRT_COMPUTE_DEFAULT):
    """Gradients (dQ, dK, dV), fp32, of sum(O * dO) for the forward call with the same arguments.
    compute=MRT_COMPUTE_F32 forces fp32 arithmetic everywhere (bf16 storage otherwise uses the bf16
    matrix unit where the library has such kernels)."""
    import torch
    lib = load_library()
    assert dO.shape == Q.shape and dO.dtype == Q.dtype and dO.is_cuda
    prob = _call_problem(Q, K, V, dO, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h)
    if workspace is None:
        nbytes = lib.monarch_attn_bwd_workspace_bytes(ctypes.byref(prob), b1, b2, tile, iters)
        if nbytes == 0:
            st = lib.monarch_attn_check(ctypes.byref(prob), b1, b2, tile, iters, causal_chunk)
            _raise(lib, st if st != MRT_OK else MRT_ERR_UNSUPPORTED)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
    dQ = torch.empty(Q.shape, dtype=torch.float32, device=Q.device)
    dK = torch.empty(K.shape, dtype=torch.float32, device=Q.device)
    dV = torch.empty(V.shape, dtype=torch.float32, device=Q.device)
    s = _stream_of(Q, stream)
    st = lib.monarch_attn_bwd(Q.data_ptr(), K.data_ptr(), V.data_ptr(), dO.data_ptr(), dQ.data_ptr(),
                              dK.data_ptr(), dV.data_ptr(), ctypes.byref(prob), b1, b2, tile, iters,
                              causal_chunk, workspace.data_ptr(),
                              workspace.numel() * workspace.element_size(), s)
    if st != MRT_OK:
        _raise(lib, st)
    return dQ, dK, dV


def monarch_attn_fwd_save(Q, K, V, *, f_q, f_kv, h, w, b1, b2, tile, iters, causal_chunk=0,
                          q_frame_offset=0, scale=1.0, workspace=None, out=None, stream=None, assign="fh_w",
                          tile_h=0, compute=MRT_COMPUTE_DEFAULT):
    """Forward call of a training step: returns (O, workspace); the workspace holds the intermediates of
    every iteration for monarch_attn_bwd_saved."""
    import torch
    lib = load_library()
    O = torch.empty_like(Q) if out is None else out
    prob = _call_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h)
    if workspace is None:
        nbytes = lib.monarch_attn_bwd_saved_workspace_bytes(ctypes.byref(prob), b1, b2, tile, iters)
        if nbytes == 0:
            st = lib.monarch_attn_check(ctypes.byref(prob), b1, b2, tile, iters, causal_chunk)
            _raise(lib, st if st != MRT_OK else MRT_ERR_UNSUPPORTED)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
    s = _stream_of(Q, stream)
    st = lib.monarch_attn_fwd_save(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), ctypes.byref(prob),
                                   b1, b2, tile, iters, causal_chunk, workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), s)
    if st != MRT_OK:
        _raise(lib, st)
    return O, workspace


def monarch_attn_bwd_saved(Q, K, V, dO, workspace, *, f_q, f_kv, h, w, b1, b2, tile, iters, causal_chunk=0,
                           q_frame_offset=0, scale=1.0, stream=None, assign="fh_w", tile_h=0,
                           compute=MRT_COMPUTE_DEFAULT):
    """Gradients (dQ, dK, dV) from the intermediates monarch_attn_fwd_save left in `workspace` (same
    Q, K, V and arguments): only the reverse sweep runs."""
    import torch
    lib = load_library()
    assert dO.shape == Q.shape and dO.dtype == Q.dtype and dO.is_cuda
    prob = _call_problem(Q, K, V, dO, f_q, f_kv, h, w, q_frame_offset, scale, compute, assign, tile_h)
    dQ = torch.empty(Q.shape, dtype=torch.float32, device=Q.device)
    dK = torch.empty(K.shape, dtype=torch.float32, device=Q.device)
    dV = torch.empty(V.shape, dtype=torch.float32, device=Q.device)
    s = _stream_of(Q, stream)
    st = lib.monarch_attn_bwd_saved(Q.data_ptr(), K.data_ptr(), V.data_ptr(), dO.data_ptr(), dQ.data_ptr(),
                                    dK.data_ptr(), dV.data_ptr(), ctypes.byref(prob), b1, b2, tile, iters,
                                    causal_chunk, workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), s)
    if st != MRT_OK:
        _raise(lib, st)
    return dQ, dK, dV


def dense_attn_workspace_bytes(prob: MrtProblem, causal_chunk=0) -> int:
    """Scratch a dense call makes use of (0: none)."""
    return int(load_library().dense_attn_workspace_bytes(ctypes.byref(prob), causal_chunk))


def _dense_scratch(prob, causal_chunk, Q, s):
    """Scratch of one dense call, or None: on a stream that is not the current one, by which torch's allocator
    orders the memory; under a graph capture, because torch does not tell whether its allocator knows of the
    capture (then the graph would keep the memory) or not (then an allocation could end the capture, and replays
    would find the memory in other hands); where the allocator refuses."""
    import torch
    known = prob.__dict__.setdefault("dense_bytes", {})      # by value, like the descriptor itself
    nbytes = known.get(causal_chunk)
    if nbytes is None:
        nbytes = known[causal_chunk] = dense_attn_workspace_bytes(prob, causal_chunk)
    if nbytes == 0 or s != _stream_of(Q, None) or torch.cuda.is_current_stream_capturing():
        return None
    try:
        return torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
    except torch.cuda.OutOfMemoryError:       # a call that fits without its scratch still runs
        return None


def dense_attn_fwd(Q, K, V, *, f_q, f_kv, h, w, causal_chunk=0, q_frame_offset=0, scale=1.0,
                   compute=MRT_COMPUTE_DEFAULT, out=None, stream=None, workspace=None):
    """Dense softmax attention baseline on device tensors [batch, heads, tokens, head_dim].

    bf16 calls of few queries split their keys over several workgroups if they have scratch memory
    (dense_attn_workspace_bytes): `workspace`, or memory of torch's allocator.  Without `workspace` a call under a
    graph capture, with a `stream` that is not torch's current one, or one whose scratch the allocator refuses
    splits nothing: it takes longer (2 heads of 816 queries of 3264 keys 44 us instead of 19), and its results are
    two roundings to bf16 from a split call's (3e-3 in the 2-norm), equally far from the exact ones.  Give such
    calls a workspace to have them split like the others.  How the keys are split also depends on the number of
    heads, so a head's last bits may."""
    import torch
    lib = load_library()
    O = torch.empty_like(Q) if out is None else out
    prob = _call_problem(Q, K, V, O, f_q, f_kv, h, w, q_frame_offset, scale, compute)
    s = _stream_of(Q, stream)
    if workspace is None:
        workspace = _dense_scratch(prob, causal_chunk, Q, s)
    ws, nbytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = lib.dense_attn_fwd_ws(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(),
                               ctypes.byref(prob), causal_chunk, ws, nbytes, s)
    if st != MRT_OK:
        _raise(lib, st)
    return O


# ---- a training step of the dense attention, rotary positions ------------------------------------
def _require(ok, text, status=MRT_ERR_SHAPE):
    if not ok:
        raise MrtError(status, text)


def _run_on(Q, stream, call):
    """call(stream) with Q's device and the call's stream as torch's current ones: memory that it takes from torch is
    then ordered by the stream that uses it."""
    import torch
    get = getattr(torch._C, "_cuda_getDevice", None)
    same_device = Q.get_device() == (get() if get is not None else torch.cuda.current_device())
    s = _stream_of(Q, None)
    if same_device and (stream is None or stream == s):
        return call(s)
    with torch.cuda.device(Q.device):
        if stream is None:
            return call(_stream_of(Q, None))
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, Q.device) if stream else torch.cuda.default_stream(Q.device)):
            return call(stream)


def _dtype_of(x, name):
    import torch
    _require(x.dtype in (torch.float32, torch.bfloat16), f"{name}: fp32 or bf16, got {x.dtype}")
    return MRT_F32 if x.dtype == torch.float32 else MRT_BF16


def _same_device(first, *others):
    at = first.get_device()
    _require(at >= 0, "tensors must be on a GPU")
    for x in others:
        if x is not None and x.get_device() != at:
            _require(False, "tensors are on different devices")


# (problem, training description without kv_len, backward scratch) of recent calls by their values, like _problems
_train_problems: dict = {}


def _train_problem(Q, K, V, O, grads, f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale, compute):
    key = (Q.shape, K.shape, V.shape, O.shape, Q.dtype, K.dtype, V.dtype, O.dtype, Q.stride(), K.stride(), V.stride(), O.stride(),
           tuple([(g.shape, g.dtype, g.stride()) for g in grads]), f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale, compute)
    found = _train_problems.get(key)
    if found is not None:
        return found
    _require(Q.dim() == 4 and K.dim() == 4 and K.shape == V.shape, "Q, K and V are [batch, heads, tokens, head_dim], K like V")
    B, H, nq, d = Q.shape
    _require(nq == f_q * h * w, f"Q has {nq} tokens, the grid {f_q * h * w}")
    _require(K.shape[0] == B and K.shape[2] == f_kv * h * w and K.shape[3] == d,
             f"K and V are [{B}, heads, {f_kv * h * w}, {d}], got {tuple(K.shape)}")
    for x, like in zip((O, *grads), (Q, Q, Q, K, V)):
        _require(x.shape == like.shape, "O, dO and the gradients have the shapes of Q, K and V")
    for x in (Q, K, V, O, *grads):
        _require(x.dtype == Q.dtype, "all tensors have one type")
        _require(x.stride(3) == 1, "head_dim must be contiguous")

    def st(x):
        return x.stride()[:3]
    prob = make_problem(batch=B, heads=H, head_dim=d, f_q=f_q, f_kv=f_kv, h=h, w=w, q_frame_offset=q_frame_offset,
                        dtype=_dtype_of(Q, "Q"), compute=compute, scale=scale, q_strides=st(Q), k_strides=st(K),
                        v_strides=st(V), o_strides=st(O))
    train = MrtDenseTrain(K.shape[1], None, *[MrtStrides(*st(x)) for x in grads])
    if not grads:
        scratch = dense_attn_fwd_save_workspace_bytes(prob, train, causal_chunk)
    else:
        scratch = dense_attn_bwd_workspace_bytes(prob, train, causal_chunk)
        if scratch == 0:
            lib = load_library()
            _raise(lib, lib.dense_attn_bwd_check(ctypes.byref(prob), ctypes.byref(train), causal_chunk))
    if len(_train_problems) >= _MAX_PROBLEMS:
        _train_problems.clear()
    _train_problems[key] = found = prob, train, scratch
    return found


def _with_lengths(train, kv_len, batch):
    if kv_len is None:
        return train
    import torch
    _require(kv_len.dtype == torch.int32 and kv_len.shape == (batch,) and kv_len.is_contiguous(), f"kv_len: int32 [{batch}], contiguous")
    return MrtDenseTrain(train.kv_heads, kv_len.data_ptr(), train.dout, train.dq, train.dk, train.dv)


def _require_lse(lse, Q):
    import torch
    _require(lse.shape == Q.shape[:3] and lse.dtype == torch.float32 and lse.is_contiguous(),
             "lse is fp32 [batch, heads, tokens], contiguous")


def _require_scratch(workspace):
    """(the library writes as many bytes from its address on as it is told that there are)"""
    _require(workspace is None or workspace.is_contiguous(), "workspace must be contiguous", MRT_ERR_WORKSPACE)


def dense_attn_fwd_save(Q, K, V, *, f_q, f_kv, h, w, causal_chunk=0, q_frame_offset=0, scale=1.0, kv_len=None,
                        compute=MRT_COMPUTE_DEFAULT, out=None, lse=None, workspace=None, stream=None):
    """Forward call of a training step of the dense attention: (O, lse) for dense_attn_bwd.

    Q [batch, heads, tokens, head_dim]; K and V [batch, kv_heads, tokens, head_dim], where kv_heads divides heads.
    lse [batch, heads, tokens], fp32: the natural logarithm of the sum of a row's exponentials, -inf for a row that
    sees no key (its O is 0).  kv_len (int32 [batch], on the device): keys from there on are padding.

    Calls of few queries share their keys over several workgroups if they have scratch memory
    (dense_attn_fwd_save_workspace_bytes): `workspace`, or memory of torch's allocator.  Without `workspace` a call under a
    graph capture, or one whose scratch the allocator refuses, does without, as dense_attn_fwd does.  O differs from dense_attn_fwd's by
    roundings at most."""
    import torch
    lib = load_library()
    _same_device(Q, K, V, out, lse, kv_len, workspace)
    _require_scratch(workspace)

    def call(s):
        O = torch.empty_like(Q) if out is None else out
        prob, train, nbytes = _train_problem(Q, K, V, O, (), f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale, compute)
        stats = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device) if lse is None else lse
        _require_lse(stats, Q)
        train = _with_lengths(train, kv_len, Q.shape[0])
        scratch = workspace
        if scratch is None and nbytes and not torch.cuda.is_current_stream_capturing():
            try:
                scratch = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
            except torch.cuda.OutOfMemoryError:       # a call that fits without its scratch still runs
                pass
        ws, nbytes = (None, 0) if scratch is None else (scratch.data_ptr(), scratch.numel() * scratch.element_size())
        st = lib.dense_attn_fwd_save(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), stats.data_ptr(),
                                     ctypes.byref(prob), ctypes.byref(train), causal_chunk, ws, nbytes, s)
        if st != MRT_OK:
            _raise(lib, st)
        return O, stats
    return _run_on(Q, stream, call)


def dense_attn_fwd_save_workspace_bytes(prob: MrtProblem, train: MrtDenseTrain, causal_chunk=0) -> int:
    """Scratch a forward call that keeps its row statistics makes use of (0: none)."""
    return int(load_library().dense_attn_fwd_save_workspace_bytes(ctypes.byref(prob), ctypes.byref(train), causal_chunk))


def dense_attn_fwd_save_queries(prob: MrtProblem, train: MrtDenseTrain, causal_chunk=0, workspace_bytes=0) -> int:
    """Queries of a workgroup of that call with so much scratch (64, 128 or 256: one of its kernels each)."""
    return int(load_library().dense_attn_fwd_save_queries(ctypes.byref(prob), ctypes.byref(train), causal_chunk, workspace_bytes))


def dense_attn_bwd_workspace_bytes(prob: MrtProblem, train: MrtDenseTrain, causal_chunk=0) -> int:
    """Scratch a backward call needs (0: invalid arguments)."""
    return int(load_library().dense_attn_bwd_workspace_bytes(ctypes.byref(prob), ctypes.byref(train), causal_chunk))


def dense_attn_bwd(Q, K, V, O, dO, lse, *, f_q, f_kv, h, w, causal_chunk=0, q_frame_offset=0, scale=1.0, kv_len=None,
                   compute=MRT_COMPUTE_DEFAULT, out=None, workspace=None, stream=None):
    """Gradients (dQ, dK, dV) of sum(O * dO), in the type of Q, K and V, from the forward call's O and lse
    (dense_attn_fwd_save with the same arguments).  The probabilities are formed again, nothing of their size is kept.
    out: (dQ, dK, dV) to write.  workspace: scratch of dense_attn_bwd_workspace_bytes() bytes (torch's by default)."""
    import torch
    lib = load_library()
    _same_device(Q, K, V, O, dO, lse, kv_len, workspace, *(out or ()))
    _require_scratch(workspace)
    _require_lse(lse, Q)

    def call(s):
        dQ, dK, dV = out if out is not None else (torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V))
        prob, train, nbytes = _train_problem(Q, K, V, O, (dO, dQ, dK, dV), f_q, f_kv, h, w, causal_chunk, q_frame_offset,
                                             scale, compute)
        train = _with_lengths(train, kv_len, Q.shape[0])
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=Q.device) if workspace is None else workspace
        st = lib.dense_attn_bwd(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), dO.data_ptr(), lse.data_ptr(),
                                dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), ctypes.byref(prob), ctypes.byref(train),
                                causal_chunk, scratch.data_ptr(), scratch.numel() * scratch.element_size(), s)
        if st != MRT_OK:
            _raise(lib, st)
        return dQ, dK, dV
    return _run_on(Q, stream, call)


def rotary_pairs_split(head_dim: int):
    """Rotary pairs of (frame, height, width) by default: thirds, the rest to the frame (64 pairs -> 22, 21, 21)."""
    pairs = head_dim // 2
    return pairs - 2 * (pairs // 3), pairs // 3, pairs // 3


def _rotary_tensor(x, y, f, h, w, offset, positions, name):
    import torch
    _require(x.dim() == 4 and x.stride(3) == 1 and y.stride(3) == 1, f"{name}: [batch, heads, tokens, head_dim], head_dim contiguous")
    _require(y.shape == x.shape, f"{name}: the output has another shape")
    B, H, n, _ = x.shape
    if positions is not None:
        _require(positions.dtype == torch.int32 and positions.shape in ((3, n), (B, 3, n)) and (n == 1 or positions.stride(-1) == 1),
                 f"{name}: positions are int32 [3, {n}] or [{B}, 3, {n}]")
        f, h, w, offset = 1, 1, n, 0
        pos = None, positions.stride(0) if positions.dim() == 3 else 0, positions.stride(-2)
    else:
        _require(f is not None and h is not None and w is not None, f"{name}: neither a grid nor positions")
        _require(n == f * h * w, f"{name} has {n} tokens, its grid {f * h * w}")
        pos = None, 0, 0
    return MrtRotaryTensor(B, H, f, h, w, offset, MrtStrides(*x.stride()[:3]), MrtStrides(*y.stride()[:3]),
                           _dtype_of(x, name), _dtype_of(y, name), *pos)


def _layout_of(x):
    return None if x is None else (x.shape, x.stride(), x.dtype)


# (description, tensors without their positions) of recent calls by their values, like _problems
_rotary_problems: dict = {}


def _rotary(entry, Q, K, f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, split, layout, ladder, q_positions,
            k_positions, dtype, out, k_out, stream):
    import torch
    lib = load_library()
    _require(K is not None or (k_out is None and k_positions is None), "k_out and k_positions are for a call with K")
    for y in (out, k_out):
        _require(y is None or dtype is None or y.dtype == dtype, "dtype is not that of the given output")
    _same_device(Q, K, q_positions, k_positions, out, k_out)

    def call(s):
        y = [torch.empty_like(Q, dtype=dtype) if out is None else out]
        x, n = [Q], 1
        if K is not None:
            y.append(torch.empty_like(K, dtype=dtype) if k_out is None else k_out)
            x, n = [Q, K], 2
        key = (Q.shape, Q.stride(), Q.dtype, _layout_of(y[0]), _layout_of(K), _layout_of(y[-1]), _layout_of(q_positions),
               _layout_of(k_positions), f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta,
               None if split is None else tuple(split), layout, ladder)
        found = _rotary_problems.get(key)
        if found is None:
            _require(layout in ROTARY_LAYOUTS, f"layout is one of {sorted(ROTARY_LAYOUTS)}")
            _require(ladder in ROTARY_LADDERS, f"ladder is one of {sorted(ROTARY_LADDERS)}")
            pairs = tuple(rotary_pairs_split(Q.shape[-1]) if split is None else split)
            _require(len(pairs) == 3, "split: rotary pairs of the frame, height and width axis")
            r = MrtRotary(Q.shape[-1], (ctypes.c_int * 3)(*pairs), ROTARY_LAYOUTS[layout], ROTARY_LADDERS[ladder], theta)
            tensors = [_rotary_tensor(Q, y[0], f_q, h, w, q_frame_offset, q_positions, "Q")]
            if K is not None:
                _require(K.shape[-1] == Q.shape[-1], "Q and K have one head_dim")
                tensors.append(_rotary_tensor(K, y[1], f_q if f_kv is None else f_kv, h, w, kv_frame_offset, k_positions, "K"))
            found = r, (MrtRotaryTensor * n)(*tensors), ctypes.c_void_p * n
            if len(_rotary_problems) >= _MAX_PROBLEMS:
                _rotary_problems.clear()
            _rotary_problems[key] = found
        r, tensors, pointers = found
        if q_positions is not None or k_positions is not None:     # (a description that is shared is not written)
            tensors = type(tensors).from_buffer_copy(tensors)
            for t, pos in zip(tensors, (q_positions, k_positions)):
                t.positions = None if pos is None else pos.data_ptr()
        st = getattr(lib, entry)(ctypes.byref(r), tensors, n, pointers(*[t.data_ptr() for t in x]),
                                 pointers(*[t.data_ptr() for t in y]), s)
        if st != MRT_OK:
            _raise(lib, st)
        return tuple(y) if n > 1 else y[0]
    return _run_on(Q, stream, call)


def rotary_fwd(Q, K=None, *, f_q=None, f_kv=None, h=None, w=None, q_frame_offset=0, kv_frame_offset=0, theta=10000.0,
               split=None, layout="adjacent", ladder="axis", q_positions=None, k_positions=None, dtype=None, out=None,
               k_out=None, stream=None):
    """Rotary positions with three axes on Q and K, [batch, heads, tokens, head_dim], in one launch: (Q', K'), or Q'
    where K is None.  The numbers of heads may differ.

    Positions: those of the grids (f_q, h, w) and (f_kv, h, w), frames counted from the offsets, or q_positions /
    k_positions, int32 [3, tokens] or [batch, 3, tokens].  split: rotary pairs of the three axes (by default thirds
    of head_dim); features behind them are copied.  layout "adjacent": a pair is features 2p, 2p + 1; "halves": p and
    p + the number of pairs.  ladder "axis": every axis has the frequencies theta^(-i / its pairs); "shared": one
    ladder theta^(-p / all pairs) is shared out.  dtype: of the results (that of Q and K by default).  out / k_out may
    be Q / K themselves, or the place in a cache where the keys belong."""
    return _rotary("mrt_rotary_fwd", Q, K, f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, split, layout, ladder,
                   q_positions, k_positions, dtype, out, k_out, stream)


def rotary_bwd(dQ, dK=None, *, f_q=None, f_kv=None, h=None, w=None, q_frame_offset=0, kv_frame_offset=0, theta=10000.0,
               split=None, layout="adjacent", ladder="axis", q_positions=None, k_positions=None, dtype=None, out=None,
               k_out=None, stream=None):
    """Gradients with respect to rotary_fwd's inputs from those of its results (the turn by the opposite angle), with
    the arguments of that call.  dtype: of the results, e.g. bf16 for the fp32 gradients of monarch_attn_bwd."""
    return _rotary("mrt_rotary_bwd", dQ, dK, f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, split, layout, ladder,
                   q_positions, k_positions, dtype, out, k_out, stream)


# ---- norms of queries and keys with their rotary positions ---------------------------------------
# (description, tensors without addresses, how to fill these in, arrays of addresses, backward scratch) of recent calls by their values, like _problems
_norm_problems: dict = {}


def _packing(template, offsets):
    """(pack, pieces): pieces of the template's bytes with places for addresses between them; pack(*pieces) joins them."""
    raw, form, pieces, last = bytes(template), "=", [], 0
    for offset in offsets:
        form += f"{offset - last}sQ"
        pieces += (raw[last:offset], 0)
        last = offset + 8
    pieces.append(raw[last:])
    return struct.Struct(f"{form}{len(raw) - last}s").pack, pieces


def _packed(packing, addresses):
    pack, pieces = packing
    pieces = pieces.copy()                       # (what is shared is not written)
    pieces[1::2] = addresses
    return pack(*pieces)


def _norm_weight(weight, x, name):
    if weight is None:
        return None, MRT_F32, 0
    d = x.shape[-1]
    _require(weight.shape in ((d,), (x.shape[1], d)) and (d == 1 or weight.stride(-1) == 1),
             f"{name}: the weight is [{d}] or [{x.shape[1]}, {d}], head_dim contiguous")
    return weight, _dtype_of(weight, name + "'s weight"), weight.stride(0) if weight.dim() == 2 and x.shape[1] > 1 else 0


def _own_rows(weight):
    """A weight of every head with a row of its own (expanded ones have one place for all, where their gradients have not)."""
    return weight.contiguous() if weight is not None and weight.dim() == 2 and 0 <= weight.stride(0) < weight.shape[1] else weight


def _norm_problem(x, y, dx, weights, f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, split, layout, ladder, positions,
                  given=None):
    """x, y, dx: the norm's input, its result (or the gradient of that) and the gradient of x, of one or two tensors.  given: None,
    or those of y and dx whose layout does not follow from x (the others come from empty_like), behind the type asked of that."""
    if given is None:
        given = (None, *y, *dx)
    key = [f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, None if split is None else tuple(split), layout, ladder, len(x), len(dx),
           given[0]]
    for t in (*x, *weights, *positions, *given[1:]):
        if t is None:
            key.append(None)
        else:
            key += (t.shape, t.stride(), t.dtype)
    key = tuple(key)
    found = _norm_problems.get(key)
    if found is not None:
        return found
    _require(layout in ROTARY_LAYOUTS, f"layout is one of {sorted(ROTARY_LAYOUTS)}")
    _require(ladder in ROTARY_LADDERS, f"ladder is one of {sorted(ROTARY_LADDERS)}")
    pairs = tuple(rotary_pairs_split(x[0].shape[-1]) if split is None else split)
    _require(len(pairs) == 3, "split: rotary pairs of the frame, height and width axis")
    r = MrtRotary(x[0].shape[-1], (ctypes.c_int * 3)(*pairs), ROTARY_LAYOUTS[layout], ROTARY_LADDERS[ladder], theta)
    tensors = []
    for i, name in zip(range(len(x)), "QK"):
        _require(x[i].shape[-1] == x[0].shape[-1], "Q and K have one head_dim")
        t = _rotary_tensor(x[i], y[i], (f_q if i == 0 or f_kv is None else f_kv), h, w, kv_frame_offset if i else q_frame_offset,
                           positions[i], name)
        _, dtype, apart = _norm_weight(weights[i], x[i], name)
        strides = MrtStrides()
        if dx:
            _require(dx[i].shape == x[i].shape and dx[i].dtype == x[i].dtype and dx[i].stride(3) == 1,
                     f"{name}: the gradient has its shape and type, head_dim contiguous")
            strides = MrtStrides(*dx[i].stride()[:3])
        tensors.append(MrtNormTensor(t, None, dtype, apart, strides, None))
    array = (MrtNormTensor * len(x))(*tensors)
    offsets = [i * ctypes.sizeof(MrtNormTensor) + at for i in range(len(x)) for at in _NORM_ADDRESSES]
    packing, nbytes = _packing(array, offsets), 0
    if dx:                                       # (scratch: of a call whose addresses are there)
        there = _packed(packing, [256 if t is not None else 0 for i in range(len(x)) for t in (positions[i], weights[i], weights[i])])
        nbytes = load_library().mrt_norm_rotary_bwd_workspace_bytes(ctypes.byref(r), there, len(x))
    found = r, array, packing, struct.Struct(f"{len(x)}Q").pack, nbytes
    if len(_norm_problems) >= _MAX_PROBLEMS:
        _norm_problems.clear()
    _norm_problems[key] = found
    return found


_NORM_ADDRESSES = (MrtNormTensor.t.offset + MrtRotaryTensor.positions.offset, MrtNormTensor.weight.offset, MrtNormTensor.dweight.offset)


def _norm_tensors(packing, x, weights, positions, dweights=(None, None)):
    """The description with the call's addresses."""
    addresses = []
    for _, weight, position, dweight in zip(x, weights, positions, dweights):
        addresses += (0 if position is None else position.data_ptr(), 0 if weight is None else weight.data_ptr(),
                      0 if dweight is None else dweight.data_ptr())
    return _packed(packing, addresses)


def norm_rotary_fwd(Q, K=None, q_weight=None, k_weight=None, *, eps=1e-6, f_q=None, f_kv=None, h=None, w=None, q_frame_offset=0,
                    kv_frame_offset=0, theta=10000.0, split=None, layout="adjacent", ladder="axis", q_positions=None,
                    k_positions=None, dtype=None, out=None, k_out=None, stream=None):
    """Root-mean-square norms of Q and K, [batch, heads, tokens, head_dim], every head of a token by itself, and their rotary
    positions, in one launch: (Q', K'), or Q' where K is None.

    q_weight / k_weight: [head_dim], or [heads, head_dim] for a weight of every head, fp32 or bf16; None: ones.  The other
    arguments are those of rotary_fwd.  Statistics and products in fp32, rounded once to `dtype` (that of Q and K by
    default)."""
    lib = load_library()
    import torch
    _require(K is not None or (k_out is None and k_positions is None and k_weight is None),
             "k_out, k_positions and k_weight are for a call with K")
    for y in (out, k_out):
        _require(y is None or dtype is None or y.dtype == dtype, "dtype is not that of the given output")
    _same_device(Q, K, q_weight, k_weight, q_positions, k_positions, out, k_out)

    def call(s):
        x, y = [Q], [torch.empty_like(Q, dtype=dtype) if out is None else out]
        if K is not None:
            x.append(K)
            y.append(torch.empty_like(K, dtype=dtype) if k_out is None else k_out)
        weights, positions = (_own_rows(q_weight), _own_rows(k_weight)), (q_positions, k_positions)
        r, _, packing, pointers, _ = _norm_problem(x, y, (), weights, f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, split,
                                             layout, ladder, positions, (dtype, out, k_out))
        tensors = _norm_tensors(packing, x, weights, positions)
        st = lib.mrt_norm_rotary_fwd(ctypes.byref(r), eps, tensors, len(x), pointers(*[t.data_ptr() for t in x]),
                                     pointers(*[t.data_ptr() for t in y]), s)
        if st != MRT_OK:
            _raise(lib, st)
        return tuple(y) if len(y) > 1 else y[0]
    return _run_on(Q, stream, call)


def norm_rotary_bwd(Q, K, q_weight, k_weight, dQ, dK=None, *, eps=1e-6, f_q=None, f_kv=None, h=None, w=None, q_frame_offset=0,
                    kv_frame_offset=0, theta=10000.0, split=None, layout="adjacent", ladder="axis", q_positions=None,
                    k_positions=None, out=None, k_out=None, workspace=None, stream=None):
    """Gradients with respect to norm_rotary_fwd's inputs, from those of its results, dQ and dK: (dQ, dK, dq_weight,
    dk_weight), with the arguments of that call.  K and dK are None together.  Gradients of Q and K have their types (those
    that come in may have others); gradients of weights are fp32 in the weights' shapes, summed over batch, tokens and the
    heads that share them, None where there is no weight.  out / k_out: where the gradients of Q and K belong.
    workspace: scratch (torch's by default)."""
    lib = load_library()
    import torch
    _require((K is None) == (dK is None) and (K is not None or (k_out is None and k_positions is None and k_weight is None)),
             "K and dK come together; k_out, k_positions and k_weight are for a call with K")
    _same_device(Q, K, q_weight, k_weight, dQ, dK, q_positions, k_positions, out, k_out, workspace)
    _require_scratch(workspace)

    def call(s):
        x, g, dx = [Q], [dQ], [torch.empty_like(Q) if out is None else out]
        if K is not None:
            x.append(K)
            g.append(dK)
            dx.append(torch.empty_like(K) if k_out is None else k_out)
        weights, positions = (_own_rows(q_weight), _own_rows(k_weight)), (q_positions, k_positions)
        r, _, packing, pointers, nbytes = _norm_problem(x, g, dx, weights, f_q, f_kv, h, w, q_frame_offset, kv_frame_offset, theta, split,
                                             layout, ladder, positions, (None, *g, out, k_out))
        # (contiguous: rows of weights are, and rows apart come out side by side)
        dw = [None if u is None else torch.empty_like(u, dtype=torch.float32) for u in weights]
        tensors = _norm_tensors(packing, x, weights, positions, dw)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=Q.device) if workspace is None and nbytes else workspace
        ws, nbytes = (None, 0) if scratch is None else (scratch.data_ptr(), scratch.numel() * scratch.element_size())
        st = lib.mrt_norm_rotary_bwd(ctypes.byref(r), eps, tensors, len(x), pointers(*[t.data_ptr() for t in x]),
                                     pointers(*[t.data_ptr() for t in g]), pointers(*[t.data_ptr() for t in dx]), ws, nbytes, s)
        if st != MRT_OK:
            _raise(lib, st)
        return dx[0], dx[1] if K is not None else None, dw[0], dw[1]
    return _run_on(Q, stream, call)


# ---- a cache of keys and values in 8 bits --------------------------------------------------------
class Cache8(NamedTuple):
    """K, V: codes [batch, heads, capacity, head_dim], torch.float8_e4m3fn or torch.int8.  K_scale, V_scale: uint8
    [batch, heads, ceil(capacity / block)], the exponent + 127 of the power of two that `block` tokens share."""
    K: object
    V: object
    K_scale: object
    V_scale: object
    block: int


def cache8(batch, heads, capacity, head_dim, *, format="e4m3", block=64, device="cuda"):
    """An empty cache (all values zero).  format: "e4m3" or "int8"."""
    import torch
    _require(format in ("e4m3", "int8"), "format is e4m3 or int8")
    _require(block in (16, 32, 64, 128), "block is 16, 32, 64 or 128")
    dtype = torch.float8_e4m3fn if format == "e4m3" else torch.int8
    codes = [torch.zeros(batch, heads, capacity, head_dim, dtype=torch.uint8, device=device).view(dtype) for _ in range(2)]
    scales = [torch.full((batch, heads, -(-capacity // block)), 3, dtype=torch.uint8, device=device) for _ in range(2)]
    return Cache8(*codes, *scales, block)


# descriptions of recent caches without addresses, by their values, like _problems
_caches: dict = {}


_CACHE_ADDRESSES = tuple(getattr(MrtCache8, name).offset for name in ("k_codes", "v_codes", "k_scales", "v_scales"))


def _cache8_bytes(c):
    """The C description of a cache."""
    K, V, ks, vs, block = c.K, c.V, c.K_scale, c.V_scale, c.block
    key = (K.shape, K.stride(), K.dtype, V.shape, V.stride(), V.dtype, ks.shape, ks.stride(), ks.dtype, vs.shape, vs.stride(), vs.dtype,
           block, type(block))
    found = _caches.get(key)
    if found is None:
        import torch
        _require(K.dim() == 4 and V.shape == K.shape and K.dtype == V.dtype and K.dtype in (torch.float8_e4m3fn, torch.int8),
                 "K and V of a cache are [batch, heads, capacity, head_dim], torch.float8_e4m3fn or torch.int8")
        _require(type(block) is int and block in (16, 32, 64, 128), "block is 16, 32, 64 or 128")
        B, H, n, d = K.shape
        blocks = -(-n // block)
        for x in (ks, vs):
            _require(x.dtype == torch.uint8 and x.shape == (B, H, blocks) and (blocks == 1 or x.stride(2) == 1),
                     f"scales of the cache are uint8 [{B}, {H}, {blocks}], blocks contiguous")
        _require(K.stride(3) == 1 and V.stride(3) == 1, "head_dim must be contiguous")
        found = _packing(MrtCache8(B, H, d, n, block, 0 if K.dtype == torch.float8_e4m3fn else 1, MrtStrides(*K.stride()[:3]),
                                   MrtStrides(*V.stride()[:3]), *ks.stride()[:2], *vs.stride()[:2]), _CACHE_ADDRESSES)
        if len(_caches) >= _MAX_PROBLEMS:
            _caches.clear()
        _caches[key] = found
    return _packed(found, (K.data_ptr(), V.data_ptr(), ks.data_ptr(), vs.data_ptr()))


def _cache8_of(c):
    return MrtCache8.from_buffer_copy(_cache8_bytes(c))


# descriptions of recent rows without addresses, by their values, like _problems
_rows: dict = {}


_ROWS = struct.Struct(f"={MrtCache8Rows.at.offset}siQQ{ctypes.sizeof(MrtCache8Rows) - MrtCache8Rows.k.offset}s").pack


def _cache8_rows(cache, K, V, at, lengths, given=True):
    """given: K and V may have any layout; else they are contiguous, of the cache's shape but for their number of rows."""
    number = type(at) is int
    key = (cache.K.shape, (K.shape, K.stride(), K.dtype, V.shape, V.stride(), V.dtype) if given else (K.shape[2], K.dtype),
           number or (at.dtype, at.shape, at.stride()), lengths is None or (lengths.dtype, lengths.shape, lengths.stride()))
    found = _rows.get(key)
    if found is None:
        import torch
        B, H, _, d = cache.K.shape
        _require(K.dim() == 4 and K.shape == V.shape and K.shape[:2] == (B, H) and K.shape[3] == d and K.dtype == V.dtype,
                 f"K and V are [{B}, {H}, tokens, {d}] of one type")
        _require(K.stride(3) == 1 and V.stride(3) == 1, "head_dim must be contiguous")
        for name, x in (("at", None if number else at), ("lengths", lengths)):
            _require(x is None or (x.dtype == torch.int32 and x.shape == (B,) and x.is_contiguous()),
                     f"{name}: int32 [{B}], contiguous" + (", or a number" if name == "at" else ""))
        found = bytes(MrtCache8Rows(K.shape[2], 0, None, None, MrtStrides(*K.stride()[:3]), MrtStrides(*V.stride()[:3]), _dtype_of(K, "K")))
        found = found[:MrtCache8Rows.at.offset], found[MrtCache8Rows.k.offset:]
        if len(_rows) >= _MAX_PROBLEMS:
            _rows.clear()
        _rows[key] = found
    return _ROWS(found[0], at if number else 0, 0 if number else at.data_ptr(), 0 if lengths is None else lengths.data_ptr(), found[1])


def _require_places(at, lengths=None):
    import torch
    _require(isinstance(at, torch.Tensor) or (type(at) is int and 0 <= at <= 1 << 24), "at: a number (0 .. 2^24), or int32 [batch] on the device")
    _require(lengths is None or isinstance(lengths, torch.Tensor), "lengths: int32 [batch] on the device")


def cache8_write(cache, K, V, *, at=0, lengths=None, stream=None):
    """Rows K and V, [batch, heads, tokens, head_dim], fp32 or bf16, into the cache, from token `at` on: a number, or int32
    [batch] on the device (rows outside the cache are then left out).  lengths (int32 [batch], on the device): rows of every
    sequence that are there.  Rows before `at` keep their values.  A write ends its last block: what was behind the new rows in it
    is lost, so rows inside a cache are replaced up to a multiple of the block (4680 tokens are not one), or with those that
    follow up to there.  The rounding is in the header's comment."""
    lib = load_library()
    _require_places(at, lengths)
    _same_device(K, V, cache.K, cache.V, cache.K_scale, cache.V_scale, None if type(at) is int else at, lengths)

    def call(s):
        st = lib.mrt_cache8_write(_cache8_bytes(cache), _cache8_rows(cache, K, V, at, lengths), K.data_ptr(), V.data_ptr(), s)
        if st != MRT_OK:
            _raise(lib, st)
    _run_on(K, stream, call)


def cache8_read(cache, tokens, *, at=0, dtype=None, out=None, v_out=None, stream=None):
    """The cache's values (K, V) of `tokens` tokens from `at` on (a number, or int32 [batch] on the device: tokens outside the
    cache give zeros), [batch, heads, tokens, head_dim], bf16 (the default) or fp32, exactly: for an attention that takes them so."""
    lib = load_library()
    import torch
    for y in (out, v_out):
        _require(y is None or dtype is None or y.dtype == dtype, "dtype is not that of the given output")
    _require_places(at)
    _same_device(cache.K, cache.V, cache.K_scale, cache.V_scale, None if type(at) is int else at, out, v_out)

    def call(s):
        B, H, _, d = cache.K.shape
        given = dtype if dtype is not None else out.dtype if out is not None else v_out.dtype if v_out is not None else torch.bfloat16
        K = torch.empty(B, H, tokens, d, dtype=given, device=cache.K.device) if out is None else out
        V = v_out if v_out is not None else torch.empty_like(K) if out is None else cache.K.new_empty((B, H, tokens, d), dtype=given)
        _require(K.shape[2] == tokens, f"the output has {K.shape[2]} tokens, not {tokens}")
        rows = _cache8_rows(cache, K, V, at, None, out is not None or v_out is not None)
        st = lib.mrt_cache8_read(_cache8_bytes(cache), rows, K.data_ptr(), V.data_ptr(), s)
        if st != MRT_OK:
            _raise(lib, st)
        return K, V
    return _run_on(cache.K, stream, call)


# (problem, scratch) of recent calls by their values, like _problems
_cache8_problems: dict = {}


def _cache8_problem(Q, O, cache, c, f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale):
    key = (Q.shape, Q.stride(), Q.dtype, O.shape, O.stride(), O.dtype, cache.K.shape, cache.K.stride(), cache.V.stride(), cache.K.dtype,
           f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale)
    found = _cache8_problems.get(key)
    if found is None:
        _require(Q.dim() == 4 and O.shape == Q.shape and O.dtype == Q.dtype and Q.stride(3) == 1 and O.stride(3) == 1,
                 "Q and O are [batch, heads, tokens, head_dim] of one type, head_dim contiguous")
        B, H, nq, d = Q.shape
        _require(nq == f_q * h * w, f"Q has {nq} tokens, the grid {f_q * h * w}")
        prob = make_problem(batch=B, heads=H, head_dim=d, f_q=f_q, f_kv=f_kv, h=h, w=w, q_frame_offset=q_frame_offset,
                            dtype=_dtype_of(Q, "Q"), scale=scale, q_strides=Q.stride()[:3], o_strides=O.stride()[:3])
        lib = load_library()
        nbytes = int(lib.dense_attn_fwd_cache8_workspace_bytes(ctypes.byref(prob), c, causal_chunk))
        if nbytes == 0:
            st = lib.dense_attn_cache8_check(ctypes.byref(prob), ctypes.byref(MrtCache8.from_buffer_copy(c)), causal_chunk)
            if st != MRT_OK:
                _raise(lib, st)
        if len(_cache8_problems) >= _MAX_PROBLEMS:
            _cache8_problems.clear()
        _cache8_problems[key] = found = prob, nbytes
    return found


def dense_attn_fwd_cache8_workspace_bytes(Q, cache, *, f_q, f_kv, h, w, causal_chunk=0, q_frame_offset=0, scale=1.0) -> int:
    """Scratch that dense_attn_fwd_cache8 makes use of with these arguments (0: none)."""
    return _cache8_problem(Q, Q, cache, _cache8_bytes(cache), f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale)[1]


def dense_attn_fwd_cache8(Q, cache, *, f_q, f_kv, h, w, causal_chunk=0, q_frame_offset=0, scale=1.0, kv_len=None, out=None,
                          lse=None, workspace=None, stream=None):
    """Dense attention of bf16 queries [batch, heads, tokens, head_dim] over the first f_kv h w tokens of a cache, whose heads
    divide those of Q: (O, lse), as dense_attn_fwd_save gives them.  kv_len (int32 [batch], on the device): tokens that each
    sequence has.  out may be Q itself.  The cache's values take part exactly; the probabilities are rounded to bf16.

    Calls of few queries share their keys over several workgroups if they have scratch memory
    (dense_attn_fwd_cache8_workspace_bytes): `workspace`, or memory of torch's allocator.  Without `workspace` a call under a
    graph capture, or one whose scratch the allocator refuses, does without and takes longer; results differ by roundings."""
    lib = load_library()
    import torch
    _same_device(Q, cache.K, cache.V, cache.K_scale, cache.V_scale, out, lse, kv_len, workspace)
    _require_scratch(workspace)

    def call(s):
        O = torch.empty_like(Q) if out is None else out
        c = _cache8_bytes(cache)
        prob, nbytes = _cache8_problem(Q, O, cache, c, f_q, f_kv, h, w, causal_chunk, q_frame_offset, scale)
        if lse is None:
            B, H, nq, _ = Q.shape
            stats = torch.empty(B, H, nq, dtype=torch.float32, device=Q.device)
        else:
            stats = lse
            _require_lse(stats, Q)
        if kv_len is not None:
            _require(kv_len.dtype == torch.int32 and kv_len.shape == Q.shape[:1] and kv_len.is_contiguous(),
                     f"kv_len: int32 [{Q.shape[0]}], contiguous")
        scratch = workspace
        if scratch is None and nbytes and not torch.cuda.is_current_stream_capturing():
            try:
                scratch = Q.new_empty(nbytes, dtype=torch.uint8)
            except torch.cuda.OutOfMemoryError:       # a call that fits without its scratch still runs
                pass
        ws, nbytes = (None, 0) if scratch is None else (scratch.data_ptr(), scratch.numel() * scratch.element_size())
        st = lib.dense_attn_fwd_cache8(Q.data_ptr(), c, O.data_ptr(), stats.data_ptr(), ctypes.byref(prob),
                                       None if kv_len is None else kv_len.data_ptr(), causal_chunk, ws, nbytes, s)
        if st != MRT_OK:
            _raise(lib, st)
        return O, stats
    return _run_on(Q, stream, call)
