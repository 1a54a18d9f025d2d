"""ctypes binding of the C-ABI library (``include/lf.h``): argument marshalling only.

Every step of the hot path runs inside the library's HIP kernels.  PyTorch is used here
for nothing but device memory (``torch.empty`` on the GPU) and the current HIP stream.
There is no CPU fallback: if the shared library has not been built, or a call returns an
error status, an exception is raised.
"""
from __future__ import annotations

import array
import ctypes as C
import os
from typing import Optional, Tuple

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "liblf_hsa.so")
_lib = None

LF_OK = 0
LF_BF16, LF_F32 = 0, 1
LF_NORM_LAYER, LF_NORM_RMS = 0, 1
LF_SCHED_FIXED, LF_SCHED_LINEAR, LF_SCHED_CAG = 0, 1, 2
LF_OF_CANDIDATES, LF_OF_HISTORY, LF_OF_ALL = 0, 1, 2


class lf_schedule(C.Structure):
    _fields_ = [("mode", C.c_int32), ("n_chunks", C.c_int32), ("frames_per_chunk", C.c_int32),
                ("frame_len", C.c_int32), ("block", C.c_int32), ("n_sink", C.c_int32),
                ("n_win", C.c_int32), ("k_frames", C.c_int32), ("ratio_of", C.c_int32),
                ("current_mandatory", C.c_int32), ("first_chunk_dense", C.c_int32),
                ("reserved", C.c_int32),
                ("keep_fixed", C.c_double), ("keep_first", C.c_double), ("keep_last", C.c_double),
                ("s_base", C.c_double), ("s_target", C.c_double)]


class lf_budget(C.Structure):
    _fields_ = [("n_hist_frames", C.c_int32), ("frames_per_chunk", C.c_int32),
                ("n_sink", C.c_int32), ("n_win", C.c_int32), ("k_frames", C.c_int32),
                ("k_blocks", C.c_int32), ("current_mandatory", C.c_int32), ("list_len", C.c_int32),
                ("keep_ratio", C.c_double)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class lf_shape(C.Structure):
    _fields_ = [("heads", C.c_int32), ("head_dim", C.c_int32), ("frame_len", C.c_int32),
                ("block", C.c_int32), ("q_len", C.c_int32), ("kv_len", C.c_int32),
                ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("q_stride_tok", C.c_int64), ("q_stride_head", C.c_int64),
                ("k_stride_tok", C.c_int64), ("k_stride_head", C.c_int64),
                ("v_stride_tok", C.c_int64), ("v_stride_head", C.c_int64),
                ("o_stride_tok", C.c_int64), ("o_stride_head", C.c_int64)]


class lf_producer_shape(C.Structure):
    _fields_ = [("heads", C.c_int32), ("head_dim", C.c_int32), ("tokens", C.c_int32),
                ("across_heads", C.c_int32), ("pairing", C.c_int32), ("eps", C.c_float),
                ("x_stride_tok", C.c_int64), ("y_stride_tok", C.c_int64), ("y_stride_head", C.c_int64)]


class lf_axes_shape(C.Structure):
    _fields_ = [("heads", C.c_int32), ("head_dim", C.c_int32), ("tokens", C.c_int32),
                ("across_heads", C.c_int32), ("pairing", C.c_int32), ("pairs", C.c_int32 * 3),
                ("eps", C.c_float), ("reserved", C.c_int32),
                ("x_stride_tok", C.c_int64), ("y_stride_tok", C.c_int64), ("y_stride_head", C.c_int64)]


class lf_kvq_shape(C.Structure):
    _fields_ = [("heads", C.c_int32), ("head_dim", C.c_int32), ("capacity", C.c_int32), ("reserved", C.c_int32)]


class lf_kvq_rows(C.Structure):
    _fields_ = [("first", C.c_int32), ("tokens", C.c_int32), ("k_stride_tok", C.c_int64), ("k_stride_head", C.c_int64),
                ("v_stride_tok", C.c_int64), ("v_stride_head", C.c_int64)]


class lf_token_shape(C.Structure):
    _fields_ = [("heads", C.c_int32), ("head_dim", C.c_int32), ("q_len", C.c_int32), ("cached_len", C.c_int32),
                ("extra_len", C.c_int32), ("reserved", C.c_int32),
                ("q_stride_tok", C.c_int64), ("q_stride_head", C.c_int64),
                ("k_stride_tok", C.c_int64), ("k_stride_head", C.c_int64),
                ("v_stride_tok", C.c_int64), ("v_stride_head", C.c_int64),
                ("o_stride_tok", C.c_int64), ("o_stride_head", C.c_int64)]


class lf_norm_shape(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("channels", C.c_int32), ("groups", C.c_int32), ("group_len", C.c_int32),
                ("stream_dtype", C.c_int32), ("kind", C.c_int32), ("eps", C.c_float), ("residual_scale", C.c_float),
                ("x_stride", C.c_int64), ("xo_stride", C.c_int64), ("b_stride", C.c_int64), ("y_stride", C.c_int64),
                ("gate_stride", C.c_int64), ("scale_stride", C.c_int64), ("shift_stride", C.c_int64)]


class lf_packed_shape(C.Structure):
    _fields_ = [("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("seqs", C.c_int32),
                ("q_len", C.c_int32), ("kv_len", C.c_int32), ("causal", C.c_int32), ("dtype", C.c_int32),
                ("q_stride_tok", C.c_int64), ("q_stride_head", C.c_int64),
                ("k_stride_tok", C.c_int64), ("k_stride_head", C.c_int64),
                ("v_stride_tok", C.c_int64), ("v_stride_head", C.c_int64),
                ("o_stride_tok", C.c_int64), ("o_stride_head", C.c_int64)]


class lf_grad_tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("numel", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32)]


class LfError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lf_strerror(status)} (lf_status {status})")


def library_path() -> str:
    return _LIB_PATH


def load() -> C.CDLL:
    """Load liblf_hsa.so (built by ``paper_2602_04789_amd.build``); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} not found: build it with `python -m paper_2602_04789_amd.build` "
            "(there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32p = C.c_void_p, C.POINTER(C.c_int32)
    lib.lf_chunk_budget.argtypes = [C.c_int32, C.POINTER(lf_schedule), C.POINTER(lf_budget)]
    lib.lf_chunk_budget.restype = C.c_int
    lib.lf_workspace_bytes.argtypes = [C.POINTER(lf_shape), C.POINTER(lf_budget)]
    lib.lf_workspace_bytes.restype = C.c_size_t
    lib.lf_workspace_layout.argtypes = [C.POINTER(lf_shape), C.POINTER(lf_budget),
                                        C.POINTER(C.c_size_t)]
    lib.lf_workspace_layout.restype = C.c_int
    lib.lf_select_mask.argtypes = [vp, vp, C.POINTER(lf_shape), C.POINTER(lf_budget), vp, vp,
                                   C.c_size_t, vp]
    lib.lf_select_mask.restype = C.c_int
    lib.lf_sparse_attn.argtypes = [vp, vp, vp, C.POINTER(lf_shape), vp, C.c_int32, C.c_float,
                                   vp, vp]
    lib.lf_sparse_attn.restype = C.c_int
    lib.lf_attn_workspace_bytes.argtypes = [C.POINTER(lf_shape)]
    lib.lf_attn_workspace_bytes.restype = C.c_size_t
    lib.lf_sparse_attn_split.argtypes = [vp, vp, vp, C.POINTER(lf_shape), C.POINTER(lf_budget), vp,
                                         C.c_float, vp, vp, C.c_size_t, vp]
    lib.lf_sparse_attn_split.restype = C.c_int
    lib.lf_sparse_attn_fwd.argtypes = [vp, vp, vp, C.POINTER(lf_shape), vp, C.c_int32, C.c_float,
                                       vp, vp, vp]
    lib.lf_sparse_attn_fwd.restype = C.c_int
    lib.lf_attn_bwd_workspace_bytes.argtypes = [C.POINTER(lf_shape)]
    lib.lf_attn_bwd_workspace_bytes.restype = C.c_size_t
    lib.lf_sparse_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, C.POINTER(lf_shape), vp, C.c_int32,
                                       C.c_float, vp, vp, vp, vp, C.c_size_t, vp]
    lib.lf_sparse_attn_bwd.restype = C.c_int
    lib.lf_qk_norm_rope.argtypes = [vp, vp, vp, vp, C.POINTER(lf_producer_shape), vp, vp]
    lib.lf_qk_norm_rope.restype = C.c_int
    axp, kvp, rwp, tkp = (C.POINTER(t) for t in (lf_axes_shape, lf_kvq_shape, lf_kvq_rows, lf_token_shape))
    lib.lf_qk_norm_rope_axes.argtypes = [vp, vp, vp, vp, axp, vp, vp]
    lib.lf_qk_norm_rope_axes.restype = C.c_int
    lib.lf_qk_norm_rope_axes_bwd_workspace_bytes.argtypes = [axp]
    lib.lf_qk_norm_rope_axes_bwd_workspace_bytes.restype = C.c_size_t
    lib.lf_qk_norm_rope_axes_bwd.argtypes = [vp, vp, vp, vp, axp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.lf_qk_norm_rope_axes_bwd.restype = C.c_int
    lib.lf_kvq_bytes.argtypes = [kvp]
    lib.lf_kvq_bytes.restype = C.c_size_t
    lib.lf_kvq_append.argtypes = [vp, vp, kvp, rwp, vp, C.c_size_t, vp]
    lib.lf_kvq_append.restype = C.c_int
    lib.lf_kvq_read.argtypes = [vp, C.c_size_t, kvp, rwp, vp, vp, vp]
    lib.lf_kvq_read.restype = C.c_int
    lib.lf_sparse_attn_kvq_workspace_bytes.argtypes = [C.POINTER(lf_shape), C.c_int32]
    lib.lf_sparse_attn_kvq_workspace_bytes.restype = C.c_size_t
    lib.lf_sparse_attn_kvq.argtypes = [vp, vp, C.c_size_t, kvp, vp, vp, C.POINTER(lf_shape), vp, C.c_int32, C.c_float, vp, vp,
                                       C.c_size_t, vp]
    lib.lf_sparse_attn_kvq.restype = C.c_int
    lib.lf_token_attn_kvq_workspace_bytes.argtypes = [tkp]
    lib.lf_token_attn_kvq_workspace_bytes.restype = C.c_size_t
    lib.lf_token_attn_kvq.argtypes = [vp, vp, C.c_size_t, kvp, vp, vp, tkp, C.c_float, vp, vp, C.c_size_t, vp]
    lib.lf_token_attn_kvq.restype = C.c_int
    nrp, pkp = C.POINTER(lf_norm_shape), C.POINTER(lf_packed_shape)
    lib.lf_gate_norm.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, nrp, vp, vp, vp]
    lib.lf_gate_norm.restype = C.c_int
    lib.lf_gate_norm_bwd_workspace_bytes.argtypes = [nrp]
    lib.lf_gate_norm_bwd_workspace_bytes.restype = C.c_size_t
    lib.lf_gate_norm_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, nrp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.lf_gate_norm_bwd.restype = C.c_int
    lib.lf_packed_attn_workspace_bytes.argtypes = [pkp]
    lib.lf_packed_attn_workspace_bytes.restype = C.c_size_t
    lib.lf_packed_attn.argtypes = [vp, vp, vp, pkp, vp, vp, C.c_float, vp, vp, vp, C.c_size_t, vp]
    lib.lf_packed_attn.restype = C.c_int
    lib.lf_packed_attn_bwd_workspace_bytes.argtypes = [pkp]
    lib.lf_packed_attn_bwd_workspace_bytes.restype = C.c_size_t
    lib.lf_packed_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, pkp, vp, vp, C.c_float, vp, vp, vp, vp, C.c_size_t, vp]
    lib.lf_packed_attn_bwd.restype = C.c_int
    lib.lf_grad_workspace_bytes.argtypes = [C.c_int32, C.c_int64]
    lib.lf_grad_workspace_bytes.restype = C.c_size_t
    lib.lf_grad_clip.argtypes = [vp, C.c_int32, C.c_float, C.c_float, vp, vp, C.c_size_t, vp]
    lib.lf_grad_clip.restype = C.c_int
    lib.lf_kcache_bytes.argtypes = [C.POINTER(lf_shape), C.c_int32]
    lib.lf_kcache_bytes.restype = C.c_size_t
    lib.lf_kcache_update.argtypes = [vp, C.POINTER(lf_shape), C.c_int32, C.c_int32, C.c_int32, vp,
                                     C.c_size_t, vp]
    lib.lf_kcache_update.restype = C.c_int
    lib.lf_select_mask_cached.argtypes = [vp, vp, vp, C.c_size_t, C.c_int32, C.POINTER(lf_shape),
                                          C.POINTER(lf_budget), vp, vp, C.c_size_t, vp]
    lib.lf_select_mask_cached.restype = C.c_int
    lib.lf_init.argtypes = []
    lib.lf_init.restype = C.c_int
    lib.lf_static_scratch_bytes.argtypes = []
    lib.lf_static_scratch_bytes.restype = C.c_size_t
    lib.lf_select_mask_static.argtypes = [vp, vp, C.POINTER(lf_shape), C.POINTER(lf_budget), vp, vp]
    lib.lf_select_mask_static.restype = C.c_int
    lib.lf_strerror.argtypes = [C.c_int]
    lib.lf_strerror.restype = C.c_char_p
    lib.lf_version.argtypes = []
    lib.lf_version.restype = C.c_int
    _lib = lib
    return lib


def lf_strerror(status: int) -> str:
    return load().lf_strerror(int(status)).decode()


def lf_version() -> int:
    return int(load().lf_version())


def make_schedule(s) -> lf_schedule:
    """Build the C struct from any object with the struct's field names (e.g. synth.Schedule)."""
    out = lf_schedule()
    for name, _ in lf_schedule._fields_:
        if name != "reserved":
            setattr(out, name, getattr(s, name))
    return out


def lf_chunk_budget(chunk_idx: int, schedule) -> lf_budget:
    sch = schedule if isinstance(schedule, lf_schedule) else make_schedule(schedule)
    out = lf_budget()
    rc = load().lf_chunk_budget(int(chunk_idx), C.byref(sch), C.byref(out))
    if rc != LF_OK:
        raise LfError(rc, "lf_chunk_budget")
    return out


def make_shape(Q, K, V=None, O=None, frame_len: int = 0, block: int = 64) -> lf_shape:
    """Geometry of [H, L, d] tensors (any object with .shape and .stride() in elements)."""
    Vt = K if V is None else V
    Ot = Q if O is None else O
    qs, ks, vs, os_, i = Q.shape, K.stride, Vt.stride, Ot.stride, int
    # one positional construction costs a third of sixteen attribute assignments
    return lf_shape(i(qs[0]), i(qs[2]), i(frame_len), i(block), i(qs[1]), i(K.shape[1]), LF_BF16, 0,
                    i(Q.stride(1)), i(Q.stride(0)), i(ks(1)), i(ks(0)), i(vs(1)), i(vs(0)),
                    i(os_(1)), i(os_(0)))


def _shape_of(Q, K, qs, ks, vs, os_, frame_len, block) -> lf_shape:
    """make_shape of tensors whose strides _strides has returned (plain numbers: 0.5 us instead of 1.6)."""
    heads, q_len, d = Q.shape
    return lf_shape(heads, d, int(frame_len), int(block), q_len, K.shape[1], LF_BF16, 0,
                    qs[1], qs[0], ks[1], ks[0], vs[1], vs[0], os_[1], os_[0])


def lf_workspace_bytes(shape: lf_shape, budget: lf_budget) -> int:
    return int(load().lf_workspace_bytes(C.byref(shape), C.byref(budget)))


def lf_workspace_layout(shape: lf_shape, budget: lf_budget) -> Tuple[int, int, int]:
    off = (C.c_size_t * 3)()
    rc = load().lf_workspace_layout(C.byref(shape), C.byref(budget), off)
    if rc != LF_OK:
        raise LfError(rc, "lf_workspace_layout")
    return int(off[0]), int(off[1]), int(off[2])


_torch = None   # the torch module, once a tensor has been seen (the budget functions do without it)


def _get_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _check_tensor(t, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must live in GPU memory")
    if t.dtype != (_torch or _get_torch()).bfloat16:
        raise ValueError(f"{name} must be bfloat16")
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError(f"{name} must be [H, L, d] with d contiguous")


def _strides(t, name: str):
    """Strides of a tensor that _check_tensor accepts, all in one call."""
    if t.is_cuda and t.dtype is (_torch or _get_torch()).bfloat16:
        st = t.stride()
        if len(st) == 3 and st[2] == 1:
            return st
    _check_tensor(t, name)
    return t.stride()


def _stream_ptr(stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    torch = _torch or _get_torch()
    # the current device's current stream; where torch has the function, without building a Stream object
    # around it (2 us).  It is not part of torch's public interface.
    try:
        raw = torch._C._cuda_getCurrentRawStream
    except AttributeError:
        return int(torch.cuda.current_stream().cuda_stream)
    return raw(torch.cuda.current_device())


def lf_select_mask(Q, Kcache, frame_len: int, block: int, budget: lf_budget, indices=None,
                   workspace=None, stream=None):
    """Enqueue mask selection; returns the int32 [H, n_q, list_len] index tensor (device)."""
    torch = _torch or _get_torch()
    qs, ks = _strides(Q, "Q"), _strides(Kcache, "Kcache")
    sh = _shape_of(Q, Kcache, qs, ks, ks, qs, frame_len, block)
    nb = -(-frame_len // block)
    if indices is None:
        n_q = (sh.q_len // frame_len) * nb if frame_len > 0 else 0
        indices = torch.empty((sh.heads, n_q, max(int(budget.list_len), 0)), dtype=torch.int32,
                              device=Q.device)
    if workspace is None:
        workspace = torch.empty(max(lf_workspace_bytes(sh, budget), 256), dtype=torch.uint8, device=Q.device)
    rc = (_lib or load()).lf_select_mask(Q.data_ptr(), Kcache.data_ptr(), C.byref(sh), C.byref(budget),
                            indices.data_ptr(), workspace.data_ptr(),
                            workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_select_mask")
    return indices


def lf_init() -> None:
    rc = load().lf_init()
    if rc != LF_OK:
        raise LfError(rc, "lf_init")


def lf_static_scratch_bytes() -> int:
    return int(load().lf_static_scratch_bytes())


def lf_select_mask_static(Q, Kcache, frame_len: int, block: int, budget: lf_budget, indices,
                          stream=None):
    """Mask selection on the library's own static scratch; ``indices`` (int32
    [H, n_q, list_len], device) is the caller's and is returned.  Allocates nothing."""
    _check_tensor(Q, "Q")
    _check_tensor(Kcache, "Kcache")
    sh = make_shape(Q, Kcache, frame_len=frame_len, block=block)
    rc = load().lf_select_mask_static(Q.data_ptr(), Kcache.data_ptr(), C.byref(sh), C.byref(budget),
                                      indices.data_ptr(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_select_mask_static")
    return indices


def lf_kcache_bytes(shape: lf_shape, max_frames: int) -> int:
    return int(load().lf_kcache_bytes(C.byref(shape), int(max_frames)))


def lf_kcache_update(Kcache, frame_len: int, block: int, frame_begin: int, frame_end: int,
                     max_frames: int, kcache, stream=None):
    """Pool frames [frame_begin, frame_end) of Kcache into the pooled-key cache ``kcache``
    (a uint8 device tensor of >= lf_kcache_bytes())."""
    _check_tensor(Kcache, "Kcache")
    # the shape only has to describe K here: a query of one frame stands in for Q
    sh = make_shape(Kcache[:, :frame_len], Kcache, frame_len=frame_len, block=block)
    rc = load().lf_kcache_update(Kcache.data_ptr(), C.byref(sh), int(frame_begin), int(frame_end),
                                 int(max_frames), kcache.data_ptr(),
                                 kcache.numel() * kcache.element_size(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_kcache_update")


def lf_select_mask_cached(Q, kcache, max_frames: int, kv_len: int, frame_len: int, block: int,
                          budget: lf_budget, Kcache=None, indices=None, workspace=None, stream=None):
    """Mask selection with the pooled keys taken from ``kcache``; returns the index tensor.
    With ``Kcache`` the current chunk's block means are refreshed from it in the same call."""
    torch = _torch or _get_torch()
    qs = _strides(Q, "Q")
    ks = qs if Kcache is None else _strides(Kcache, "Kcache")
    sh = _shape_of(Q, Q if Kcache is None else Kcache, qs, ks, ks, qs, frame_len, block)
    sh.kv_len = int(kv_len)
    nb = -(-frame_len // block)
    if indices is None:
        n_q = (sh.q_len // frame_len) * nb if frame_len > 0 else 0
        indices = torch.empty((sh.heads, n_q, max(int(budget.list_len), 0)), dtype=torch.int32,
                              device=Q.device)
    if workspace is None:
        workspace = torch.empty(max(lf_workspace_bytes(sh, budget), 256), dtype=torch.uint8,
                                device=Q.device)
    rc = (_lib or load()).lf_select_mask_cached(Q.data_ptr(), None if Kcache is None else Kcache.data_ptr(),
                                      kcache.data_ptr(),
                                      kcache.numel() * kcache.element_size(), int(max_frames),
                                      C.byref(sh), C.byref(budget), indices.data_ptr(),
                                      workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(),
                                      _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_select_mask_cached")
    return indices


def lf_sparse_attn(Q, Kcache, Vcache, indices, frame_len: int, block: int,
                   softmax_scale: float = 0.0, O=None, stream=None):
    """Enqueue blockwise sparse attention; returns O (bfloat16 [H, q_len, d], device)."""
    torch = _torch or _get_torch()
    qs, ks, vs = _strides(Q, "Q"), _strides(Kcache, "Kcache"), _strides(Vcache, "Vcache")
    if not indices.is_cuda or indices.dtype != torch.int32 or not indices.is_contiguous():
        raise ValueError("indices must be a contiguous int32 GPU tensor [H, n_q, list_len]")
    if O is None:
        O = torch.empty_like(Q, memory_format=torch.contiguous_format)
    sh = _shape_of(Q, Kcache, qs, ks, vs, _strides(O, "O"), frame_len, block)
    n_q = (sh.q_len // frame_len) * (-(-frame_len // block)) if frame_len > 0 else -1
    ishape = indices.shape
    if len(ishape) != 3 or ishape[0] != sh.heads or ishape[1] != n_q:
        raise ValueError("indices must be [H, n_q, list_len]")
    rc = (_lib or load()).lf_sparse_attn(Q.data_ptr(), Kcache.data_ptr(), Vcache.data_ptr(), C.byref(sh),
                                         indices.data_ptr(), ishape[2], float(softmax_scale),
                                         O.data_ptr(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_sparse_attn")
    return O


def lf_attn_workspace_bytes(shape: lf_shape) -> int:
    return int(load().lf_attn_workspace_bytes(C.byref(shape)))


def lf_sparse_attn_split(Q, Kcache, Vcache, indices, frame_len: int, block: int, budget: lf_budget,
                         softmax_scale: float = 0.0, O=None, workspace=None, stream=None):
    """Blockwise sparse attention over the retrieved blocks of each list and the current chunk's
    blocks, whose entries are not read (one pass, or a dense phase over the current chunk first:
    the library chooses); returns O.  ``indices`` as written by lf_select_mask for ``budget``."""
    torch = _torch or _get_torch()
    qs, ks, vs = _strides(Q, "Q"), _strides(Kcache, "Kcache"), _strides(Vcache, "Vcache")
    if not indices.is_cuda or indices.dtype != torch.int32 or not indices.is_contiguous():
        raise ValueError("indices must be a contiguous int32 GPU tensor [H, n_q, list_len]")
    if O is None:
        O = torch.empty_like(Q, memory_format=torch.contiguous_format)
    sh = _shape_of(Q, Kcache, qs, ks, vs, _strides(O, "O"), frame_len, block)
    n_q = (sh.q_len // frame_len) * (-(-frame_len // block)) if frame_len > 0 else -1
    if indices.dim() != 3 or tuple(indices.shape) != (sh.heads, n_q, int(budget.list_len)):
        raise ValueError("indices must be [H, n_q, budget.list_len]")
    if workspace is None:
        workspace = torch.empty(max(lf_attn_workspace_bytes(sh), 256), dtype=torch.uint8, device=Q.device)
    rc = (_lib or load()).lf_sparse_attn_split(Q.data_ptr(), Kcache.data_ptr(), Vcache.data_ptr(), C.byref(sh),
                                     C.byref(budget), indices.data_ptr(), float(softmax_scale),
                                     O.data_ptr(), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_sparse_attn_split")
    return O


def _check_lists(indices, sh, frame_len):
    torch = _torch or _get_torch()
    if not indices.is_cuda or indices.dtype != torch.int32 or not indices.is_contiguous():
        raise ValueError("indices must be a contiguous int32 GPU tensor [H, n_q, list_len]")
    n_q = (sh.q_len // frame_len) * (-(-frame_len // sh.block)) if frame_len > 0 else -1
    ishape = indices.shape
    if len(ishape) != 3 or ishape[0] != sh.heads or ishape[1] != n_q:
        raise ValueError("indices must be [H, n_q, list_len]")


def lf_sparse_attn_fwd(Q, Kcache, Vcache, indices, frame_len: int, block: int,
                       softmax_scale: float = 0.0, O=None, lse2=None, stream=None):
    """Blockwise sparse attention that also leaves the rows' log-sum-exp (exp2 domain) for
    lf_sparse_attn_bwd; returns (O, lse2)."""
    torch = _torch or _get_torch()
    qs, ks, vs = _strides(Q, "Q"), _strides(Kcache, "Kcache"), _strides(Vcache, "Vcache")
    if O is None:
        O = torch.empty_like(Q, memory_format=torch.contiguous_format)
    sh = _shape_of(Q, Kcache, qs, ks, vs, _strides(O, "O"), frame_len, block)
    _check_lists(indices, sh, frame_len)
    if lse2 is None:
        lse2 = torch.empty((sh.heads, sh.q_len), dtype=torch.float32, device=Q.device)
    if lse2.dtype != torch.float32 or not lse2.is_cuda or not lse2.is_contiguous() \
            or tuple(lse2.shape) != (sh.heads, sh.q_len):
        raise ValueError("lse2 must be a contiguous float32 GPU tensor [H, q_len]")
    rc = (_lib or load()).lf_sparse_attn_fwd(Q.data_ptr(), Kcache.data_ptr(), Vcache.data_ptr(), C.byref(sh),
                                   indices.data_ptr(), int(indices.shape[-1]), float(softmax_scale),
                                   O.data_ptr(), lse2.data_ptr(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_sparse_attn_fwd")
    return O, lse2


def lf_attn_bwd_workspace_bytes(shape: lf_shape) -> int:
    return int(load().lf_attn_bwd_workspace_bytes(C.byref(shape)))


def lf_sparse_attn_bwd(Q, Kcache, Vcache, O, dO, lse2, indices, frame_len: int, block: int,
                       softmax_scale: float = 0.0, workspace=None, stream=None, grads=None):
    """Gradients of the blockwise sparse attention; returns (dQ, dK, dV), bfloat16 with the
    strides of Q, Kcache and Vcache (``grads``: three such tensors to write into instead of new
    ones).  ``indices`` ascending and duplicate-free per list."""
    torch = _torch or _get_torch()
    qs, ks, vs = _strides(Q, "Q"), _strides(Kcache, "Kcache"), _strides(Vcache, "Vcache")
    os_, gs = _strides(O, "O"), _strides(dO, "dO")
    if dO.shape != O.shape or gs != os_:
        raise ValueError("dO must have the shape and strides of O")
    sh = _shape_of(Q, Kcache, qs, ks, vs, os_, frame_len, block)
    _check_lists(indices, sh, frame_len)
    if lse2.dtype != torch.float32 or not lse2.is_cuda or not lse2.is_contiguous() \
            or tuple(lse2.shape) != (sh.heads, sh.q_len):
        raise ValueError("lse2 must be a contiguous float32 GPU tensor [H, q_len]")
    if grads is None:
        dQ = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device)
        dK = torch.empty_strided(Kcache.shape, Kcache.stride(), dtype=Q.dtype, device=Q.device)
        dV = torch.empty_strided(Vcache.shape, Vcache.stride(), dtype=Q.dtype, device=Q.device)
    else:
        dQ, dK, dV = grads
        for g, t, st, name in ((dQ, Q, qs, "dQ"), (dK, Kcache, ks, "dK"), (dV, Vcache, vs, "dV")):
            if _strides(g, name) != st or g.shape != t.shape:
                raise ValueError(f"{name} must have the shape and strides of its input")
    if workspace is None:
        workspace = torch.empty(max(lf_attn_bwd_workspace_bytes(sh), 256), dtype=torch.uint8,
                                device=Q.device)
    rc = (_lib or load()).lf_sparse_attn_bwd(Q.data_ptr(), Kcache.data_ptr(), Vcache.data_ptr(), O.data_ptr(),
                                   dO.data_ptr(), lse2.data_ptr(), C.byref(sh), indices.data_ptr(),
                                   int(indices.shape[-1]), float(softmax_scale), dQ.data_ptr(),
                                   dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_sparse_attn_bwd")
    return dQ, dK, dV


def lf_qk_norm_rope(X, g, cos_table, sin_table, heads: int, Y, eps: float = 1e-6,
                    across_heads: bool = False, pairing: int = 0, stream=None):
    """RMSNorm + rotary embedding of the token-major activation X [L, >= H*d] (bfloat16) into the
    head-major tensor Y [H, L, d] (bfloat16; may be a view into Q or into the K cache)."""
    torch = _torch or _get_torch()
    xs, ys, Xsh, Ysh = X.stride(), Y.stride(), X.shape, Y.shape
    if X.dtype != torch.bfloat16 or Y.dtype != torch.bfloat16 or len(xs) != 2 or len(ys) != 3:
        raise ValueError("X must be bfloat16 [L, H*d] and Y bfloat16 [H, L, d]")
    if xs[1] != 1 or ys[2] != 1 or not (X.is_cuda and Y.is_cuda):
        raise ValueError("X and Y must be GPU tensors with contiguous channels")
    for t in (g, cos_table, sin_table):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("g, cos_table, sin_table must be contiguous float32 GPU tensors")
    heads, tokens, d = int(heads), Xsh[0], Ysh[2]
    p = lf_producer_shape(heads, d, tokens, int(bool(across_heads)), int(pairing), float(eps),
                          xs[0], ys[1], ys[0])
    csh = cos_table.shape
    if Ysh[0] != heads or Ysh[1] != tokens or g.numel() != heads * d \
            or csh != (tokens, d // 2) or csh != sin_table.shape:
        raise ValueError("shapes of Y, g or the angle tables do not fit X")
    rc = (_lib or load()).lf_qk_norm_rope(X.data_ptr(), g.data_ptr(), cos_table.data_ptr(), sin_table.data_ptr(),
                                C.byref(p), Y.data_ptr(), _stream_ptr(stream))
    if rc != LF_OK:
        raise LfError(rc, "lf_qk_norm_rope")
    return Y


def _here(stream):
    """(current device, pointer of the stream): where a launch goes."""
    torch = _torch or _get_torch()
    if stream is not None:
        at = torch.cuda.current_device()
        if getattr(stream, "device_index", at) != at:
            raise ValueError("stream must belong to the current device")
        return at, int(stream.cuda_stream)
    # as _stream_ptr, and without torch.cuda's look at its own state (0.5 us for both)
    try:
        at = torch._C._cuda_getDevice()
        return at, torch._C._cuda_getCurrentRawStream(at)
    except AttributeError:
        return torch.cuda.current_device(), int(torch.cuda.current_stream().cuda_stream)


def _one_device(at: int, tensors):
    """The launch goes to the current device: all tensors must live there."""
    for t in tensors:
        if t.get_device() != at:
            raise ValueError("all tensors must live on the current device")


def _int32(*values):
    """Sizes and places for int32 fields of the C structures, which would drop the bits above."""
    values = tuple(map(int, values))
    for v in values:        # (two thirds of the time that min() and max() take)
        if not -0x80000000 <= v <= 0x7FFFFFFF:
            raise ValueError("a size or place does not fit 32 bits")
    return values


def _small(sizes: int):
    """_int32 for sizes of tensors, which are not negative, joined by `or` (0.1 us for all of them)."""
    if sizes > 0x7FFFFFFF:
        raise ValueError("a size or place does not fit 32 bits")


def _size_of(query, make, *values) -> int:
    """What a size query of the library says of the structure that `make` builds from whole numbers, 0 where one does not fit."""
    try:
        shape, *more = make(*_int32(*values))
    except ValueError:
        return 0
    return int(query(C.byref(shape), *more))


def _new(stream, make, *args, **kw):
    """A tensor for work on `stream`: taken from that stream's memory, so nothing else still uses it there."""
    if stream is None:
        return make(*args, **kw)
    with (_torch or _get_torch()).cuda.stream(stream):
        return make(*args, **kw)


def _rows(t, name: str):
    """(shape, token stride, head stride) of a [H, L, d] tensor; the stride of an axis of length one does not matter."""
    if t.is_cuda and t.dtype is (_torch or _get_torch()).bfloat16:
        st, sh = t.stride(), t.shape
        if len(st) == 3 and st[2] == 1:
            return sh, (st[1] if sh[1] != 1 else sh[2]), (st[0] if sh[0] != 1 else 0)
    _check_tensor(t, name)
    raise ValueError(f"{name} must be [H, L, d]")


def _check_buffer(t, name: str):
    if t.dtype != (_torch or _get_torch()).uint8 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous uint8 GPU tensor")


def _workspace(workspace, need, like, stream, at: int):
    """The caller's scratch, or a new one of need() bytes: a tensor, or None where nothing is needed."""
    if workspace is None:
        n = int(need())
        return _new(stream, like.new_empty, n, dtype=(_torch or _get_torch()).uint8) if n else None
    if workspace.get_device() != at or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the current device")
    return workspace


def _bytes_of(t):
    return (0, 0) if t is None else (t.data_ptr(), t.numel() * t.element_size())


def _axes_shape(X, g, pos, freq, pairs, heads, out, eps, across_heads, pairing) -> lf_axes_shape:
    torch = _torch or _get_torch()
    if len(pairs) != 3:
        raise ValueError("pairs must be three numbers")
    heads, pairing, *pairs = _int32(heads, pairing, *pairs)
    if not X.is_cuda or X.dtype is not torch.bfloat16:
        raise ValueError("X must be a bfloat16 GPU tensor")
    if g.dtype is not torch.float32 or not g.is_contiguous():
        raise ValueError("g must be contiguous float32 [H * d]")
    if pos.dtype is not torch.int32 or not pos.is_contiguous():
        raise ValueError("pos must be contiguous int32 [L, 3]")
    if freq.dtype is not torch.float64 or not freq.is_contiguous():
        raise ValueError("freq must be contiguous float64 [d / 2]")
    (yheads, tokens, d), yt, yh = _rows(*out)
    xs, xsh = X.stride(), X.shape
    if len(xs) != 2 or xs[1] != 1 or xsh[0] != tokens or yheads != heads:
        raise ValueError("X must be [L, >= H * d] with contiguous channels, Y and dY [H, L, d]")
    if xsh[1] < heads * d or g.numel() != heads * d or pos.shape != (tokens, 3) or freq.numel() != d // 2:
        raise ValueError("shapes of X, g, pos, freq or pairs do not fit")
    return lf_axes_shape(heads, d, tokens, 1 if across_heads else 0, pairing, tuple(pairs), float(eps), 0,
                         xs[0] if tokens != 1 else heads * d, yt, yh)


def lf_qk_norm_rope_axes(X, g, pos, freq, pairs, heads: int, Y, eps: float = 1e-6, across_heads: bool = False,
                         pairing: int = 0, stream=None):
    """RMSNorm and rotary positions over three axes of the token-major activation X [L, >= H*d] (bfloat16) into the head-major
    tensor Y [H, L, d] (bfloat16; may be a view into Q or into the K cache).  ``pos`` int32 [L, 3] (time, height, width),
    ``freq`` float64 [d/2] in radians per position, ``pairs`` how many channel pairs each axis has."""
    p = _axes_shape(X, g, pos, freq, pairs, heads, (Y, "Y"), eps, across_heads, pairing)
    at, st = _here(stream)
    _one_device(at, (X, g, pos, freq, Y))
    rc = (_lib or load()).lf_qk_norm_rope_axes(X.data_ptr(), g.data_ptr(), pos.data_ptr(), freq.data_ptr(), C.byref(p),
                                               Y.data_ptr(), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_qk_norm_rope_axes")
    return Y


def lf_qk_norm_rope_axes_bwd_workspace_bytes(heads: int, head_dim: int, tokens: int) -> int:
    return _size_of(load().lf_qk_norm_rope_axes_bwd_workspace_bytes,
                    lambda H, d, L: (lf_axes_shape(H, d, L, 0, 0, (d // 2, 0, 0), 0.0, 0, H * d, d, L * d),), heads, head_dim, tokens)


def lf_qk_norm_rope_axes_bwd(X, g, pos, freq, pairs, heads: int, dY, eps: float = 1e-6, across_heads: bool = False,
                             pairing: int = 0, workspace=None, stream=None, grads=None):
    """Gradients of lf_qk_norm_rope_axes for an upstream gradient dY [H, L, d] (bfloat16); returns (dX, dg): dX bfloat16 with the
    shape and row stride of X, of which the first H*d channels are written, dg float32 [H*d] (``grads``: two such tensors to
    write into instead of new ones)."""
    torch = _torch or _get_torch()
    p = _axes_shape(X, g, pos, freq, pairs, heads, (dY, "dY"), eps, across_heads, pairing)
    at, st = _here(stream)
    _one_device(at, (X, g, pos, freq, dY))
    if grads is None:
        dg = _new(stream, torch.empty_like, g)
        if X.is_contiguous():
            dX = _new(stream, torch.empty_like, X)
        else:
            dX = _new(stream, torch.empty_strided, X.shape, X.stride(), dtype=X.dtype, device=X.device)
    else:
        dX, dg = grads
        if dX.dtype is not torch.bfloat16 or dX.shape != X.shape or dX.stride(1) != 1 or (dX.shape[0] != 1 and dX.stride(0) != X.stride(0)):
            raise ValueError("dX must be bfloat16 with the shape and strides of X")
        if dg.dtype is not torch.float32 or not dg.is_contiguous() or dg.numel() != g.numel():
            raise ValueError("dg must be contiguous float32 [H * d]")
        _one_device(at, grads)
    lib = _lib or load()
    ws = _workspace(workspace, lambda: lib.lf_qk_norm_rope_axes_bwd_workspace_bytes(C.byref(p)), X, stream, at)
    rc = lib.lf_qk_norm_rope_axes_bwd(X.data_ptr(), g.data_ptr(), pos.data_ptr(), freq.data_ptr(), C.byref(p), dY.data_ptr(),
                                      dX.data_ptr(), dg.data_ptr(), *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_qk_norm_rope_axes_bwd")
    return dX, dg


def lf_kvq_bytes(heads: int, head_dim: int, capacity: int) -> int:
    """Bytes of a 4-bit cache for `capacity` tokens (0 on bad input)."""
    return _size_of(load().lf_kvq_bytes, lambda *sizes: (lf_kvq_shape(*sizes),), heads, head_dim, capacity)


def lf_kvq_append(K, V, cache, capacity: int, first: int, stream=None):
    """Write the tokens [first, first + L) of the 4-bit cache from K and V [H, L, d] (bfloat16); returns ``cache`` (a uint8
    device tensor of >= lf_kvq_bytes())."""
    capacity, first = _int32(capacity, first)
    (sh, kt, kh), (vsh, vt, vh) = _rows(K, "K"), _rows(V, "V")
    _check_buffer(cache, "cache")
    if sh != vsh:
        raise ValueError("K and V must have one shape")
    at, st = _here(stream)
    _one_device(at, (K, V, cache))
    rc = (_lib or load()).lf_kvq_append(K.data_ptr(), V.data_ptr(), C.byref(lf_kvq_shape(sh[0], sh[2], capacity)),
                                        C.byref(lf_kvq_rows(first, sh[1], kt, kh, vt, vh)), cache.data_ptr(), cache.numel(), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_kvq_append")
    return cache


def lf_kvq_read(cache, heads: int, head_dim: int, capacity: int, first: int, tokens: int, K=None, V=None, stream=None):
    """The values that tokens [first, first + tokens) of the 4-bit cache stand for: (K, V), bfloat16 [H, tokens, d]."""
    torch = _torch or _get_torch()
    heads, d, capacity, first, tokens = _int32(heads, head_dim, capacity, first, tokens)
    _check_buffer(cache, "cache")
    shape = heads, tokens, d
    if K is None:
        K = _new(stream, cache.new_empty, shape, dtype=torch.bfloat16)
    if V is None:
        V = _new(stream, cache.new_empty, shape, dtype=torch.bfloat16)
    (ksh, kt, kh), (vsh, vt, vh) = _rows(K, "K"), _rows(V, "V")
    if ksh != shape or vsh != shape:
        raise ValueError("K and V must be [H, tokens, d]")
    at, st = _here(stream)
    _one_device(at, (cache, K, V))
    rc = (_lib or load()).lf_kvq_read(cache.data_ptr(), cache.numel(), C.byref(lf_kvq_shape(heads, d, capacity)),
                                      C.byref(lf_kvq_rows(first, tokens, kt, kh, vt, vh)), K.data_ptr(), V.data_ptr(), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_kvq_read")
    return K, V


def lf_sparse_attn_kvq_workspace_bytes(heads: int, head_dim: int, frame_len: int, block: int, q_len: int, kv_len: int,
                                       list_len: int) -> int:
    """Scratch of one call (0 on bad input too).  It can be less for a longer cache: a buffer for several calls has the largest of their sizes."""
    return _size_of(load().lf_sparse_attn_kvq_workspace_bytes,
                    lambda H, d, n, b, q, kv, length: (lf_shape(H, d, n, b, q, kv, LF_BF16, 0, d, 0, d, 0, d, 0, d, 0), length),
                    heads, head_dim, frame_len, block, q_len, kv_len, list_len)


def lf_sparse_attn_kvq(Q, cache, capacity: int, kv_len: int, indices, frame_len: int, block: int, K=None, V=None,
                       softmax_scale: float = 0.0, O=None, workspace=None, stream=None):
    """Blockwise sparse attention over the 4-bit cache; returns O (bfloat16 [H, q_len, d], device).  With ``K`` and ``V`` [H, q_len,
    d] the current chunk's tokens, the last q_len of kv_len, are read from them in bfloat16, without them from the cache."""
    capacity, kv_len, frame_len, block = _int32(capacity, kv_len, frame_len, block)
    _check_buffer(cache, "cache")
    qsh, qt, qh = _rows(Q, "Q")
    heads, q_len, d = qsh
    if O is None:
        O = _new(stream, Q.new_empty, qsh)
    osh, ot, oh = _rows(O, "O")
    if osh != qsh:
        raise ValueError("O must be [H, q_len, d]")
    at, st = _here(stream)
    kt = kh = vt = vh = k_ptr = v_ptr = 0
    if K is not None and V is not None:
        (ksh, kt, kh), (vsh, vt, vh) = _rows(K, "K"), _rows(V, "V")
        if ksh != qsh or vsh != qsh:
            raise ValueError("K and V must be [H, q_len, d], the current chunk's tokens")
        _one_device(at, (Q, cache, indices, K, V, O))
        k_ptr, v_ptr = K.data_ptr(), V.data_ptr()
    elif K is not None or V is not None:
        raise ValueError("K and V go together")
    else:
        _one_device(at, (Q, cache, indices, O))
    sh = lf_shape(heads, d, frame_len, block, q_len, kv_len, LF_BF16, 0, qt, qh, kt, kh, vt, vh, ot, oh)
    _check_lists(indices, sh, frame_len)
    length, = _int32(indices.shape[2])
    lib = _lib or load()
    ws = _workspace(workspace, lambda: lib.lf_sparse_attn_kvq_workspace_bytes(C.byref(sh), length), Q, stream, at)
    rc = lib.lf_sparse_attn_kvq(Q.data_ptr(), cache.data_ptr(), cache.numel(), C.byref(lf_kvq_shape(heads, d, capacity)),
                                k_ptr, v_ptr, C.byref(sh), indices.data_ptr(), length, float(softmax_scale), O.data_ptr(), *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_sparse_attn_kvq")
    return O


def lf_token_attn_kvq_workspace_bytes(heads: int, head_dim: int, q_len: int, cached_len: int, extra_len: int) -> int:
    return _size_of(load().lf_token_attn_kvq_workspace_bytes,
                    lambda H, d, q, held, extra: (lf_token_shape(H, d, q, held, extra, 0, d, 0, d, 0, d, 0, d, 0),),
                    heads, head_dim, q_len, cached_len, extra_len)


def lf_token_attn_kvq(Q, cache, capacity: int, cached_len: int, K=None, V=None, softmax_scale: float = 0.0, O=None,
                      workspace=None, stream=None):
    """Attention of up to 64 query rows [H, q_len, d] over the first ``cached_len`` tokens of the 4-bit cache and the tokens of ``K``
    and ``V`` [H, extra, d] (bfloat16, optional) behind them; returns O (bfloat16 [H, q_len, d], device)."""
    capacity, cached_len = _int32(capacity, cached_len)
    _check_buffer(cache, "cache")
    qsh, qt, qh = _rows(Q, "Q")
    heads, q_len, d = qsh
    if O is None:
        O = _new(stream, Q.new_empty, qsh)
    osh, ot, oh = _rows(O, "O")
    if osh != qsh:
        raise ValueError("O must be [H, q_len, d]")
    at, st = _here(stream)
    extra = kt = kh = vt = vh = k_ptr = v_ptr = 0
    if K is not None and V is not None:
        (ksh, kt, kh), (vsh, vt, vh) = _rows(K, "K"), _rows(V, "V")
        extra = ksh[1]
        if ksh != vsh or ksh[0] != heads or ksh[2] != d:
            raise ValueError("K and V must be [H, extra, d]")
        _one_device(at, (Q, cache, K, V, O))
        k_ptr, v_ptr = K.data_ptr(), V.data_ptr()
    elif K is not None or V is not None:
        raise ValueError("K and V go together")
    else:
        _one_device(at, (Q, cache, O))
    sh = lf_token_shape(heads, d, q_len, cached_len, extra, 0, qt, qh, kt, kh, vt, vh, ot, oh)
    lib = _lib or load()
    ws = _workspace(workspace, lambda: lib.lf_token_attn_kvq_workspace_bytes(C.byref(sh)), Q, stream, at)
    rc = lib.lf_token_attn_kvq(Q.data_ptr(), cache.data_ptr(), cache.numel(), C.byref(lf_kvq_shape(heads, d, capacity)),
                               k_ptr, v_ptr, C.byref(sh), float(softmax_scale), O.data_ptr(), *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_token_attn_kvq")
    return O


_stream_dtypes = {}        # torch type -> lf_dtype, for streams and gradients (filled once a tensor has been seen)


def _dtypes():
    if not _stream_dtypes:
        torch = _torch or _get_torch()
        _stream_dtypes.update({torch.bfloat16: LF_BF16, torch.float32: LF_F32})
    return _stream_dtypes


def _row_stride(t, shape, dtype, at: int, name: str) -> int:
    """Row stride of a [L, C] tensor on device `at` with contiguous channels; that of a single row does not matter."""
    if t.dtype is dtype and t.shape == shape:
        if t.get_device() != at:
            raise ValueError("all tensors must live on the current device")
        st = t.stride()
        if st[1] == 1 or shape[1] == 1:
            return st[0] if shape[0] != 1 else shape[1]
    raise ValueError(f"{name} must be {dtype} {list(shape)} with contiguous channels")


def _vector(t, n: int, dtype, at: int, name: str) -> int:
    """Address of a contiguous tensor of n elements on device `at`."""
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} [{n}]")
    if t.get_device() != at:
        raise ValueError("all tensors must live on the current device")
    return t.data_ptr()


def _norm_groups(L: int, group_len: int, starts, at: int):
    """(groups, group_len, address of starts)"""
    group_len, = _int32(group_len)
    if starts is None:
        if group_len > 0:
            return -(-L // group_len), group_len, None
    elif group_len <= 0:
        if starts.dim() != 1 or starts.shape[0] < 2:
            raise ValueError("starts must be [groups + 1]")
        groups = starts.shape[0] - 1
        _small(groups)
        return groups, 0, _vector(starts, groups + 1, (_torch or _get_torch()).int32, at, "starts")
    raise ValueError("groups are given by group_len > 0 or by starts")


def lf_gate_norm(X, B=None, gate=None, post_weight=None, weight=None, scale=None, shift=None, group_len: int = 0, starts=None,
                 kind: int = LF_NORM_LAYER, eps: float = 1e-6, residual_scale: float = 1.0, Xout=None, Y=None, stream=None):
    """Between two blocks: Xout = X + residual_scale * gate * (B, or its RMSNorm with ``post_weight``) and Y = norm(Xout) * weight * (1 + scale) +
    shift; returns (Xout, Y).  X [L, C] bfloat16 or float32, B [L, C] and Y bfloat16; gate, scale and shift float32 [groups, C], one row for ``group_len``
    tokens or for the tokens [starts[g], starts[g + 1]) (int32, device); without B, Xout is X.  Xout may be X itself."""
    torch = _torch or _get_torch()
    bf, f32 = torch.bfloat16, torch.float32
    rows, dtype = X.shape, X.dtype
    if len(rows) != 2 or dtype not in (_stream_dtypes or _dtypes()):
        raise ValueError("X must be bfloat16 or float32 [L, C]")
    L, n = rows
    _small(L | n)
    at, st = _here(stream)
    groups, group_len, starts_ptr = _norm_groups(L, group_len, starts, at)
    xs = _row_stride(X, rows, dtype, at, "X")
    xos = bs = gs = cs = hs = n
    b_ptr = xo_ptr = gate_ptr = post_ptr = weight_ptr = scale_ptr = shift_ptr = None
    if B is not None:
        bs, b_ptr = _row_stride(B, rows, bf, at, "B"), B.data_ptr()
        if Xout is None:
            Xout = _new(stream, X.new_empty, rows)
        xos, xo_ptr = _row_stride(Xout, rows, dtype, at, "Xout"), Xout.data_ptr()
        if gate is not None:
            gs, gate_ptr = _row_stride(gate, (groups, n), f32, at, "gate"), gate.data_ptr()
        if post_weight is not None:
            post_ptr = _vector(post_weight, n, f32, at, "post_weight")
    elif gate is not None or post_weight is not None or Xout is not None:
        raise ValueError("gate, post_weight and Xout go with B")
    if weight is not None:
        weight_ptr = _vector(weight, n, f32, at, "weight")
    if scale is not None:
        cs, scale_ptr = _row_stride(scale, (groups, n), f32, at, "scale"), scale.data_ptr()
    if shift is not None:
        hs, shift_ptr = _row_stride(shift, (groups, n), f32, at, "shift"), shift.data_ptr()
    if Y is None:
        Y = _new(stream, X.new_empty, rows, dtype=bf)
    ys = _row_stride(Y, rows, bf, at, "Y")
    kind, = _int32(kind)
    p = lf_norm_shape(L, n, groups, group_len, _stream_dtypes[dtype], kind, eps, residual_scale, xs, xos, bs, ys, gs, cs, hs)
    rc = (_lib or load()).lf_gate_norm(X.data_ptr(), b_ptr, gate_ptr, post_ptr, weight_ptr, scale_ptr, shift_ptr, starts_ptr, C.byref(p), xo_ptr, Y.data_ptr(), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_gate_norm")
    return (X if B is None else Xout), Y


def lf_gate_norm_bwd_workspace_bytes(tokens: int, channels: int, groups: int, group_len: int = 0) -> int:
    """Scratch of one call (0 on bad input); group_len = 0: groups are given by ``starts``."""
    return _size_of(load().lf_gate_norm_bwd_workspace_bytes,
                    lambda L, c, g, n: (lf_norm_shape(L, c, g, n, LF_BF16, LF_NORM_LAYER, 0.0, 1.0, c, c, c, c, c, c, c),), tokens, channels, groups,
                    group_len)


def lf_gate_norm_bwd(Xout, dY, dXout=None, B=None, gate=None, post_weight=None, weight=None, scale=None, group_len: int = 0, starts=None,
                     kind: int = LF_NORM_LAYER, eps: float = 1e-6, residual_scale: float = 1.0, dX=None, dB=None, workspace=None, stream=None):
    """Gradients of lf_gate_norm for upstream gradients dY of Y (may be None: zeros) and dXout of Xout (likewise); Xout as the forward call returned it.
    Returns (dX, dB, dgate, dpost_weight, dweight, dscale, dshift): dX with the type of the stream (``dX`` may be dXout itself), dB bfloat16,
    the tables' gradients float32 [groups, C] and [C], None for what the call does not have (dscale and dshift are always there)."""
    torch = _torch or _get_torch()
    bf, f32 = torch.bfloat16, torch.float32
    rows, dtype = Xout.shape, Xout.dtype
    if len(rows) != 2 or dtype not in (_stream_dtypes or _dtypes()):
        raise ValueError("Xout must be bfloat16 or float32 [L, C]")
    L, n = rows
    _small(L | n)
    at, st = _here(stream)
    groups, group_len, starts_ptr = _norm_groups(L, group_len, starts, at)
    xos = _row_stride(Xout, rows, dtype, at, "Xout")
    bs = ys = gs = cs = n
    b_ptr = db_ptr = gate_ptr = post_ptr = weight_ptr = scale_ptr = dy_ptr = dxo_ptr = None
    if dY is not None:
        ys, dy_ptr = _row_stride(dY, rows, bf, at, "dY"), dY.data_ptr()
    if dXout is not None:
        if _row_stride(dXout, rows, dtype, at, "dXout") != xos:
            raise ValueError("dXout must have the strides of Xout")
        dxo_ptr = dXout.data_ptr()
    if dX is None:
        dX = _new(stream, torch.empty_strided, rows, (xos, 1), dtype=dtype, device=Xout.device)
    if dX is not dXout and _row_stride(dX, rows, dtype, at, "dX") != xos:
        raise ValueError("dX must have the strides of Xout")
    tables = 2
    if B is not None:
        bs, b_ptr = _row_stride(B, rows, bf, at, "B"), B.data_ptr()
        if dB is None:
            dB = _new(stream, torch.empty_strided, rows, (bs, 1), dtype=bf, device=B.device)
        if _row_stride(dB, rows, bf, at, "dB") != bs:
            raise ValueError("dB must have the strides of B")
        db_ptr = dB.data_ptr()
        if gate is not None:
            gs, gate_ptr, tables = _row_stride(gate, (groups, n), f32, at, "gate"), gate.data_ptr(), 3
        if post_weight is not None:
            post_ptr = _vector(post_weight, n, f32, at, "post_weight")
    elif gate is not None or post_weight is not None or dB is not None:
        raise ValueError("gate, post_weight and dB go with B")
    if weight is not None:
        weight_ptr = _vector(weight, n, f32, at, "weight")
    if scale is not None:
        cs, scale_ptr = _row_stride(scale, (groups, n), f32, at, "scale"), scale.data_ptr()
    # the tables' gradients are parts of one tensor: an allocation instead of three
    made = _new(stream, Xout.new_empty, (tables, groups, n), dtype=f32)
    dscale, dshift, *more = made.unbind(0)
    dgate = more[0] if more else None
    dpost = None if post_ptr is None else _new(stream, Xout.new_empty, (n,), dtype=f32)
    dweight = None if weight_ptr is None else _new(stream, Xout.new_empty, (n,), dtype=f32)
    size = 4 * groups * n
    base = made.data_ptr()
    kind, = _int32(kind)
    p = lf_norm_shape(L, n, groups, group_len, _stream_dtypes[dtype], kind, eps, residual_scale, xos, xos, bs, ys, gs, cs, n)
    lib = _lib or load()
    ws = _workspace(workspace, lambda: lib.lf_gate_norm_bwd_workspace_bytes(C.byref(p)), Xout, stream, at)
    rc = lib.lf_gate_norm_bwd(Xout.data_ptr(), b_ptr, gate_ptr, post_ptr, weight_ptr, scale_ptr, starts_ptr, C.byref(p), dy_ptr, dxo_ptr, dX.data_ptr(), db_ptr,
                              base + 2 * size if more else None, None if dpost is None else dpost.data_ptr(), None if dweight is None else dweight.data_ptr(),
                              base, base + size, *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_gate_norm_bwd")
    return dX, dB, dgate, dpost, dweight, dscale, dshift


def _packed(Q, K, V, O, q_start, kv_start, causal):
    """The shape of a call with [H, L, d] tensors."""
    i32 = (_torch or _get_torch()).int32
    (qsh, qt, qh), (ksh, kt, kh), (vsh, vt, vh), (osh, ot, oh) = _rows(Q, "Q"), _rows(K, "K"), _rows(V, "V"), _rows(O, "O")
    heads, q_len, d = qsh
    kv_heads, kv_len, kd = ksh
    if ksh != vsh or kd != d or osh != qsh:
        raise ValueError("K and V must be [kv_heads, kv_len, d], O [heads, q_len, d] as Q")
    n = q_start.shape
    if q_start.dtype is not i32 or kv_start.dtype is not i32 or len(n) != 1 or n[0] < 2 or kv_start.shape != n or not q_start.is_contiguous() \
            or not kv_start.is_contiguous():
        raise ValueError("q_start and kv_start must be contiguous int32 [seqs + 1]")
    causal, = _int32(causal)
    _small(heads | kv_heads | d | q_len | kv_len | n[0] - 1)
    return lf_packed_shape(heads, kv_heads, d, n[0] - 1, q_len, kv_len, causal, LF_BF16, qt, qh, kt, kh, vt, vh, ot, oh)


def _packed_sizes(query, heads, kv_heads, head_dim, seqs, q_len, kv_len, causal) -> int:
    return _size_of(query, lambda H, Hk, d, b, q, kv, u: (lf_packed_shape(H, Hk, d, b, q, kv, u, LF_BF16, d, 0, d, 0, d, 0, d, 0),),
                    heads, kv_heads, head_dim, seqs, q_len, kv_len, causal)


def lf_packed_attn_workspace_bytes(heads: int, kv_heads: int, head_dim: int, seqs: int, q_len: int, kv_len: int, causal: int = 0) -> int:
    """Scratch of one forward call (0 on bad input too); q_len and kv_len are the tensors' rows, of all sequences."""
    return _packed_sizes(load().lf_packed_attn_workspace_bytes, heads, kv_heads, head_dim, seqs, q_len, kv_len, causal)


def _packed_fwd(Q, K, V, q_start, kv_start, causal, softmax_scale, O, lse2, with_lse, workspace, stream, where):
    at, st = _here(stream)
    if O is None:
        O = _new(stream, Q.new_empty, Q.shape)
    p = _packed(Q, K, V, O, q_start, kv_start, causal)
    l_ptr = None
    if with_lse:
        f32 = (_torch or _get_torch()).float32
        if lse2 is None:
            lse2 = _new(stream, Q.new_empty, Q.shape[:2], dtype=f32)
        if lse2.dtype is not f32 or lse2.shape != Q.shape[:2] or not lse2.is_contiguous():
            raise ValueError("lse2 must be a contiguous float32 GPU tensor [heads, q_len]")
        _one_device(at, (Q, K, V, O, q_start, kv_start, lse2))
        l_ptr = lse2.data_ptr()
    else:
        _one_device(at, (Q, K, V, O, q_start, kv_start))
    lib = _lib or load()
    ws = _workspace(workspace, lambda: lib.lf_packed_attn_workspace_bytes(C.byref(p)), Q, stream, at)
    rc = lib.lf_packed_attn(Q.data_ptr(), K.data_ptr(), V.data_ptr(), C.byref(p), q_start.data_ptr(), kv_start.data_ptr(), softmax_scale,
                            O.data_ptr(), l_ptr, *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, where)
    return O, lse2


def lf_packed_attn(Q, K, V, q_start, kv_start, causal: int = 0, softmax_scale: float = 0.0, O=None, workspace=None, stream=None):
    """Attention over packed sequences: Q [heads, q_len, d], K and V [kv_heads, kv_len, d] (bfloat16), sequence b with the rows
    [q_start[b], q_start[b + 1]) and the tokens [kv_start[b], kv_start[b + 1]) (int32, device).  ``causal`` 0: rows see their whole sequence, 1: the
    tokens up to their own (the last row the last token), u: up to the end of their chunk of u.  Returns O; rows of no sequence are left as they are
    (those of a new tensor hold anything)."""
    return _packed_fwd(Q, K, V, q_start, kv_start, causal, softmax_scale, O, None, False, workspace, stream, "lf_packed_attn")[0]


def lf_packed_attn_fwd(Q, K, V, q_start, kv_start, causal: int = 0, softmax_scale: float = 0.0, O=None, lse2=None, workspace=None, stream=None):
    """lf_packed_attn that also leaves the rows' log-sum-exp (exp2 domain, float32 [heads, q_len]) for lf_packed_attn_bwd; returns (O, lse2)."""
    return _packed_fwd(Q, K, V, q_start, kv_start, causal, softmax_scale, O, lse2, True, workspace, stream, "lf_packed_attn_fwd")


def lf_packed_attn_bwd_workspace_bytes(heads: int, kv_heads: int, head_dim: int, seqs: int, q_len: int, kv_len: int, causal: int = 0) -> int:
    return _packed_sizes(load().lf_packed_attn_bwd_workspace_bytes, heads, kv_heads, head_dim, seqs, q_len, kv_len, causal)


def lf_packed_attn_bwd(Q, K, V, O, dO, lse2, q_start, kv_start, causal: int = 0, softmax_scale: float = 0.0, workspace=None, stream=None, grads=None):
    """Gradients of lf_packed_attn_fwd; returns (dQ, dK, dV), bfloat16 with the strides of Q, K and V (``grads``: three such tensors to write into).
    Rows and tokens of no sequence are left as they are (those of new tensors hold anything)."""
    torch = _torch or _get_torch()
    at, st = _here(stream)
    p = _packed(Q, K, V, O, q_start, kv_start, causal)
    if dO.shape != O.shape or dO.dtype is not torch.bfloat16 or (dO.stride() != O.stride() and _rows(dO, "dO")[1:] != (p.o_stride_tok, p.o_stride_head)):
        raise ValueError("dO must have the shape and strides of O")
    if lse2.dtype is not torch.float32 or lse2.shape != Q.shape[:2] or not lse2.is_contiguous():
        raise ValueError("lse2 must be a contiguous float32 GPU tensor [heads, q_len]")
    if grads is None:
        grads = [_new(stream, torch.empty_strided, t.shape, t.stride(), dtype=t.dtype, device=t.device) for t in (Q, K, V)]
    else:
        for g, t, name in zip(grads, (Q, K, V), ("dQ", "dK", "dV")):
            if g.shape != t.shape or (g.stride() != t.stride() and _rows(g, name)[1:] != _rows(t, name)[1:]) or g.dtype is not torch.bfloat16:
                raise ValueError(f"{name} must have the shape and strides of its input")
    dQ, dK, dV = grads
    _one_device(at, (Q, K, V, O, dO, lse2, q_start, kv_start, dQ, dK, dV))
    lib = _lib or load()
    ws = _workspace(workspace, lambda: lib.lf_packed_attn_bwd_workspace_bytes(C.byref(p)), Q, stream, at)
    rc = lib.lf_packed_attn_bwd(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), dO.data_ptr(), lse2.data_ptr(), C.byref(p), q_start.data_ptr(),
                                kv_start.data_ptr(), float(softmax_scale), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_packed_attn_bwd")
    return dQ, dK, dV


def lf_grad_workspace_bytes(count: int, numel: int) -> int:
    """Scratch of lf_grad_clip for `count` tensors of `numel` elements in all (0 on bad input)."""
    try:
        count, = _int32(count)
    except ValueError:
        return 0
    return int(load().lf_grad_workspace_bytes(count, numel)) if 0 <= numel <= 1 << 40 else 0


def lf_grad_clip(grads, max_norm: float, out=None, eps: float = 1e-6, norm=None, workspace=None, stream=None):
    """Scales gradients to a largest norm: x * min(1, max_norm / (norm + eps)), in place or into the tensors of ``out`` (one for each, of the
    same size; bfloat16 or float32), and returns the norm over all of them, float32 [1] on the device.  Where that is not finite they are not scaled;
    max_norm = inf takes the norm alone.  ``grads``: tensors of bfloat16 or float32 without holes, each listed once."""
    torch = _torch or _get_torch()
    kinds = _stream_dtypes or _dtypes()
    grads = list(grads)
    at, st = _here(stream)
    to = None if out is None else list(out)
    tensors = grads if to is None else grads + to
    T = torch.Tensor
    if any(x != at for x in map(T.get_device, tensors)):
        raise ValueError("all tensors must live on the current device")
    sizes = list(map(T.numel, grads))
    # the C structures as rows of four 64-bit numbers: address, address or 0, elements, the two types (a third of the time that ctypes takes for them)
    rows = array.array("q", bytes(32 * len(grads)))
    try:
        types = [kinds[x.dtype] for x in grads]
        if to is None:
            if not all(x.is_contiguous() or _dense(x) for x in grads):
                raise ValueError("gradients must be contiguous (in place: without holes)")
        else:
            if len(to) != len(grads):
                raise ValueError("out must have a tensor for each gradient")
            if list(map(T.numel, to)) != sizes or not all(map(T.is_contiguous, tensors)):
                raise ValueError("gradients and out must be contiguous tensors of the same sizes")
            types = [k | kinds[y.dtype] << 32 for k, y in zip(types, to)]
            rows[1::4] = array.array("q", map(T.data_ptr, to))
    except KeyError:
        raise ValueError("gradients and out must be bfloat16 or float32") from None
    rows[0::4], rows[2::4], rows[3::4] = (array.array("q", x) for x in (map(T.data_ptr, grads), sizes, types))
    total = sum(sizes)
    if norm is None:
        norm = _new(stream, torch.empty, (1,), dtype=torch.float32, device=_device(at))
    if norm.dtype is not torch.float32 or norm.numel() != 1 or norm.get_device() != at:
        raise ValueError("norm must be one float32 on the current device")
    lib = _lib or load()
    count = len(grads)
    ws = _workspace(workspace, lambda: lib.lf_grad_workspace_bytes(count, total), norm, stream, at)
    rc = lib.lf_grad_clip(rows.buffer_info()[0], count, float(max_norm), float(eps), norm.data_ptr(), *_bytes_of(ws), st)
    if rc != LF_OK:
        raise LfError(rc, "lf_grad_clip")
    return norm


_devices = {}      # index -> torch.device


def _device(at: int):
    if at not in _devices:
        _devices[at] = (_torch or _get_torch()).device("cuda", at)
    return _devices[at]


def _dense(t) -> bool:
    """Whether the elements of a tensor fill their memory without holes or overlaps, in whatever order."""
    want = 1
    for st, n in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if st != want:
            return False
        want *= n
    return True
