"""Thin ctypes binding of libspeed3r.so: same names as the C ABI (include/speed3r.h), argument
marshalling only.  Tensors are torch tensors on the GPU (torch is used for device memory and
streams, nothing else); every step of the path runs in the library's HIP kernels.  There is no
fallback: if the library is missing or a call fails, an exception is raised."""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspeed3r.so")

S3R_OK, S3R_ERR_INVALID_ARG, S3R_ERR_UNSUPPORTED, S3R_ERR_WORKSPACE, S3R_ERR_HIP = range(5)
S3R_F32, S3R_BF16 = 0, 1
S3R_NORM_NONE, S3R_NORM_RMS, S3R_NORM_LAYER = range(3)
S3R_PAIRS_HALVES, S3R_PAIRS_NEIGHBOURS, S3R_PAIRS_WHOLE = range(3)
S3R_DIAG_FORCED_RANGE, S3R_DIAG_FORCED_ORDER = 1, 2
S3R_DIAG_PAGE, S3R_DIAG_SPANS, S3R_DIAG_LENGTH, S3R_DIAG_POSITION = 4, 8, 16, 32
STAGES = ("pool", "split", "compress", "topk", "select", "dense")
HEAD_DIM = 64

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_int = ctypes.c_int
_flt = ctypes.c_float


class s3r_params(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("out", _vp), ("gate_logits", _vp),
                ("forced_blocks", _vp), ("n_forced", _int), ("status", _vp),
                ("tokens_per_view", _int), ("special_per_view", _int),
                ("grid_h", _int), ("grid_w", _int), ("window", _int), ("compress_queries", _int),
                ("n_tok", _i64), ("stride_tok", _i64), ("stride_head", _i64), ("heads", _int), ("head_dim", _int), ("block", _int),
                ("topk", _int), ("dtype", _int), ("softmax_scale", _flt), ("topk_idx", _vp),
                ("lse_sel", _vp), ("o_comp", _vp), ("o_sel", _vp), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t), ("stream", _vp)]


class s3r_cross_params(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("out", _vp), ("lse", _vp), ("d_out", _vp),
                ("dq", _vp), ("dk", _vp), ("dv", _vp), ("q_start", _vp), ("kv_start", _vp), ("key_mask", _vp),
                ("status", _vp), ("n_q", _i64), ("n_kv", _i64), ("q_stride_tok", _i64), ("q_stride_head", _i64),
                ("kv_stride_tok", _i64), ("kv_stride_head", _i64), ("batch", _int), ("heads", _int),
                ("kv_heads", _int), ("head_dim", _int), ("dtype", _int), ("softmax_scale", _flt),
                ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t), ("stream", _vp), ("accurate_pv", _int)]


class s3r_cache_params(ctypes.Structure):
    _fields_ = [("k_codes", _vp), ("v_codes", _vp), ("k_scales", _vp), ("v_scales", _vp), ("page_table", _vp),
                ("kv_len", _vp), ("row_start", _vp), ("n_pages", _i64), ("n_rows", _i64), ("page", _int),
                ("max_pages", _int), ("batch", _int), ("heads", _int), ("kv_heads", _int), ("head_dim", _int),
                ("dtype", _int), ("q", _vp), ("out", _vp), ("k", _vp), ("v", _vp), ("q_stride_tok", _i64),
                ("q_stride_head", _i64), ("kv_stride_tok", _i64), ("kv_stride_head", _i64), ("cos", _vp), ("sin", _vp),
                ("positions", _vp), ("n_positions", _i64), ("rot_axes", _int), ("rot_neighbours", _int),
                ("causal", _int), ("softmax_scale", _flt), ("lse", _vp), ("status", _vp), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t), ("stream", _vp)]


class s3r_rotary_params(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("q_out", _vp), ("k_out", _vp), ("d_q_out", _vp), ("d_k_out", _vp), ("dq", _vp),
                ("dk", _vp), ("q_weight", _vp), ("q_bias", _vp), ("k_weight", _vp), ("k_bias", _vp), ("dq_weight", _vp),
                ("dq_bias", _vp), ("dk_weight", _vp), ("dk_bias", _vp), ("cos", _vp), ("sin", _vp), ("positions", _vp),
                ("status", _vp), ("n_rows", _i64), ("n_positions", _i64), ("q_stride_tok", _i64), ("q_stride_head", _i64),
                ("k_stride_tok", _i64), ("k_stride_head", _i64), ("dq_stride_tok", _i64), ("dq_stride_head", _i64),
                ("dk_stride_tok", _i64), ("dk_stride_head", _i64), ("heads", _int), ("kv_heads", _int), ("head_dim", _int),
                ("dtype", _int), ("weight_dtype", _int), ("axes", _int), ("axis_pairs", _int * 3), ("pairs", _int),
                ("norm", _int), ("eps", _flt), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t), ("stream", _vp)]


class s3r_residual_params(ctypes.Structure):
    _fields_ = [("x", _vp), ("f", _vp), ("r", _vp), ("y", _vp), ("weight", _vp), ("bias", _vp), ("post_weight", _vp),
                ("post_bias", _vp), ("scale", _vp), ("gate", _vp), ("row_start", _vp), ("d_r", _vp), ("d_y", _vp), ("dx", _vp),
                ("df", _vp), ("d_weight", _vp), ("d_bias", _vp), ("d_post_weight", _vp), ("d_post_bias", _vp), ("d_scale", _vp),
                ("d_gate", _vp), ("status", _vp), ("n_rows", _i64), ("x_stride", _i64), ("f_stride", _i64),
                ("gate_stride", _i64), ("width", _int), ("batch", _int), ("x_dtype", _int), ("dtype", _int),
                ("weight_dtype", _int), ("norm", _int), ("post_norm", _int), ("eps", _flt), ("residual_scale", _flt),
                ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t), ("stream", _vp)]


EXPORTS = {
    "speed3r_workspace_bytes": (ctypes.c_size_t, [_i64, _int, _int, _int, _int, _int, _int]),
    "speed3r_workspace_bytes_ex": (ctypes.c_size_t, [ctypes.POINTER(s3r_params)]),
    "speed3r_num_blocks": (_i64, [ctypes.POINTER(s3r_params)]),
    "speed3r_selected_per_row": (_int, [_i64, _int, _int, _int]),
    "speed3r_sparse_global_attn_ex": (_int, [ctypes.POINTER(s3r_params)]),
    "speed3r_sparse_global_attn": (_int, [_vp, _vp, _vp, _vp, _i64, _int, _int, _int, _int, _vp]),
    "speed3r_sparse_global_attn_noalloc": (_int, [_vp, _vp, _vp, _vp, _i64, _int, _int, _int, _int, _vp]),
    "speed3r_dense_attn": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _int, _int, _int, _flt, _vp]),
    "speed3r_pool_blocks": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _int, _int, _int, _int, _vp]),
    "speed3r_compress_attn_scores": (_int, [_vp, _vp, _vp, _vp, _i64, _vp, _i64, _int, _int, _flt,
                                            _int, _vp]),
    "speed3r_compress_attn_topk": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _int, _int, _int, _flt, _int, _vp]),
    "speed3r_topk_blocks": (_int, [_vp, _i64, _vp, _i64, _int, _int, _vp]),
    "speed3r_select_attn": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _int, _int,
                                   _int, _int, _int, _flt, _vp]),
    "speed3r_cross_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(s3r_cross_params), _int]),
    "speed3r_cross_attn": (_int, [ctypes.POINTER(s3r_cross_params)]),
    "speed3r_cross_attn_backward": (_int, [ctypes.POINTER(s3r_cross_params)]),
    "speed3r_causal_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(s3r_cross_params), _int, _int]),
    "speed3r_causal_attn": (_int, [ctypes.POINTER(s3r_cross_params), _int]),
    "speed3r_causal_attn_backward": (_int, [ctypes.POINTER(s3r_cross_params), _int]),
    "speed3r_cache_append": (_int, [ctypes.POINTER(s3r_cache_params)]),
    "speed3r_cache_read": (_int, [ctypes.POINTER(s3r_cache_params)]),
    "speed3r_cache_attn": (_int, [ctypes.POINTER(s3r_cache_params)]),
    "speed3r_cache_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(s3r_cache_params)]),
    "speed3r_rotary": (_int, [ctypes.POINTER(s3r_rotary_params)]),
    "speed3r_rotary_backward": (_int, [ctypes.POINTER(s3r_rotary_params)]),
    "speed3r_rotary_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(s3r_rotary_params)]),
    "speed3r_residual_norm": (_int, [ctypes.POINTER(s3r_residual_params)]),
    "speed3r_residual_norm_backward": (_int, [ctypes.POINTER(s3r_residual_params)]),
    "speed3r_residual_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(s3r_residual_params)]),
    "speed3r_probe_select_loads": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _int, _int, _int, _int, _int, _int, _vp]),
    "speed3r_set_profiling": (_int, [_int]),
    "speed3r_get_stage_ms": (_int, [ctypes.POINTER(_flt), ctypes.POINTER(_int)]),
    "speed3r_set_kernel_choice": (_int, [_int]),
    "speed3r_release_scratch": (_int, []),
    "speed3r_last_error": (ctypes.c_char_p, []),
}

_lib = None


class Speed3rError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"speed3r status {status}: {message}")
        self.status = status


def load():
    """Load libspeed3r.so (built by paper_2603_08055_amd.build / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it first (python -m paper_2603_08055_amd.build)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _check(status: int):
    if status != S3R_OK:
        raise Speed3rError(status, speed3r_last_error())


def speed3r_last_error() -> str:
    return load().speed3r_last_error().decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return S3R_F32
    if t.dtype == torch.bfloat16:
        return S3R_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev(t, name, dtype=None):
    """data_ptr of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous tensor on the GPU")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _strided_qkv(q, k, v):
    """data_ptrs and the common (stride_tok, stride_head) of q, k, v: CUDA tensors [n_tok, heads, head_dim]
    whose channels are contiguous (views of a packed projection output are fine)."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        if not (isinstance(t, torch.Tensor) and t.is_cuda):
            raise TypeError(f"{name} must be a tensor on the GPU")
        if t.stride(2) != 1 and t.shape[2] > 1:
            raise TypeError(f"the channels of {name} must be contiguous")
    st = (q.stride(0), q.stride(1))
    if (k.stride(0), k.stride(1)) != st or (v.stride(0), v.stride(1)) != st:
        raise TypeError("q, k and v must share their row and head strides")
    if q.is_contiguous():
        st = (0, 0)
    return q.data_ptr(), k.data_ptr(), v.data_ptr(), st


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


def _qkv(q, k, v):
    if q.dim() != 3 or k.shape != q.shape or v.shape != q.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v must share shape [n_tok, heads, head_dim] and dtype")
    return q.shape[0], q.shape[1], q.shape[2], _dtype_code(q)


def speed3r_workspace_bytes(n_tok, heads, head_dim, block, topk, dtype, n_forced=0) -> int:
    return int(load().speed3r_workspace_bytes(n_tok, heads, head_dim, block, topk, n_forced, dtype))


def _shape_params(n_tok, heads, head_dim, block, topk, dtype, n_forced, tokens_per_view, special_per_view, grid,
                  compress_queries=0):
    p = s3r_params()
    p.compress_queries = int(compress_queries)
    p.n_tok, p.heads, p.head_dim, p.block, p.topk, p.dtype = n_tok, heads, head_dim, block, topk, dtype
    p.n_forced, p.tokens_per_view, p.special_per_view = n_forced, tokens_per_view, special_per_view
    p.grid_h, p.grid_w, p.window = grid if grid else (0, 0, 0)
    return p


def speed3r_workspace_bytes_ex(n_tok, heads, head_dim, block, topk, dtype, n_forced=0, tokens_per_view=0,
                               special_per_view=0, grid=None, compress_queries=0) -> int:
    """grid = (grid_h, grid_w, window) for spatial pooling windows."""
    p = _shape_params(n_tok, heads, head_dim, block, topk, dtype, n_forced, tokens_per_view, special_per_view, grid,
                      compress_queries)
    return int(load().speed3r_workspace_bytes_ex(ctypes.byref(p)))


def speed3r_num_blocks(n_tok, heads, head_dim, block, topk, dtype, tokens_per_view=0, special_per_view=0,
                       grid=None) -> int:
    p = _shape_params(n_tok, heads, head_dim, block, topk, dtype, 0, tokens_per_view, special_per_view, grid)
    n = int(load().speed3r_num_blocks(ctypes.byref(p)))
    if n < 0:
        raise Speed3rError(S3R_ERR_INVALID_ARG, speed3r_last_error())
    return n


def speed3r_selected_per_row(n_tok, block, topk, n_forced=0) -> int:
    w = int(load().speed3r_selected_per_row(n_tok, block, topk, n_forced))
    if w < 0:
        raise ValueError("invalid arguments to speed3r_selected_per_row")
    return w


def speed3r_sparse_global_attn_ex(q, k, v, out, block, topk, *, gate_logits=None, softmax_scale=0.0,
                                  topk_idx=None, lse_sel=None, o_comp=None, o_sel=None,
                                  forced_blocks=None, tokens_per_view=0, special_per_view=0, grid=None,
                                  compress_queries=0, workspace=None, status=None, stream=None):
    """The whole path on caller-provided buffers.  `workspace` is a uint8 CUDA tensor of at least
    speed3r_workspace_bytes(...) bytes (allocated here when None).  `forced_blocks` is an int32
    CUDA tensor of ascending distinct block indices attended by every query block.  With
    special_per_view > 0 the first rows of every view of tokens_per_view rows are special tokens
    (dense attention over all rows); the other rows form the sequence of the sparse path.
    grid = (grid_h, grid_w, window) makes the blocks spatial windows of each view's patch grid.
    compress_queries = 1: every row's own query (instead of its block's pooled query) attends the
    pooled keys in the compression branch.  `status`: an int32 CUDA tensor of one element that receives
    0 or the S3R_DIAG_* bits for a forced_blocks list that is out of range or not strictly ascending.  q, k, v may be strided views with contiguous channels
    and common strides (slices of one packed tensor).  Returns the workspace used."""
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    n_forced = 0 if forced_blocks is None else int(forced_blocks.numel())
    if workspace is None:
        need = speed3r_workspace_bytes_ex(n_tok, heads, head_dim, block, topk, dt, n_forced, tokens_per_view,
                                          special_per_view, grid, compress_queries)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)   # 0: the call below says why
    p = s3r_params()
    p.q, p.k, p.v, (p.stride_tok, p.stride_head) = _strided_qkv(q, k, v)
    p.out = _dev(out, "out", q.dtype)
    p.gate_logits = _dev(gate_logits, "gate_logits", q.dtype)
    p.forced_blocks = _dev(forced_blocks, "forced_blocks", torch.int32) if n_forced else None
    p.n_forced = n_forced
    p.status = _dev(status, "status", torch.int32)
    p.tokens_per_view, p.special_per_view = int(tokens_per_view), int(special_per_view)
    p.grid_h, p.grid_w, p.window = grid if grid else (0, 0, 0)
    p.compress_queries = int(compress_queries)
    p.n_tok, p.heads, p.head_dim, p.block, p.topk, p.dtype = n_tok, heads, head_dim, block, topk, dt
    p.softmax_scale = float(softmax_scale)
    p.topk_idx = _dev(topk_idx, "topk_idx", torch.int32)
    p.lse_sel = _dev(lse_sel, "lse_sel", torch.float32)
    p.o_comp = _dev(o_comp, "o_comp", torch.float32)
    p.o_sel = _dev(o_sel, "o_sel", q.dtype)
    p.workspace = _dev(workspace, "workspace", torch.uint8)
    p.workspace_bytes = workspace.numel()
    p.stream = _stream(stream)
    _check(load().speed3r_sparse_global_attn_ex(ctypes.byref(p)))
    return workspace


def speed3r_sparse_global_attn(q, k, v, out, block, topk, stream=None):
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    if dt != S3R_BF16:
        raise TypeError("the short form is bf16 only; use speed3r_sparse_global_attn_ex")
    _check(load().speed3r_sparse_global_attn(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                             _dev(out, "out", q.dtype), n_tok, heads, head_dim,
                                             block, topk, _stream(stream)))


STATIC_SCRATCH_BYTES = 64 << 20


def speed3r_sparse_global_attn_noalloc(q, k, v, out, block, topk, stream=None):
    """The short form on the library's fixed device scratch: the call allocates nothing."""
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    if dt != S3R_BF16:
        raise TypeError("the short forms are bf16 only; use speed3r_sparse_global_attn_ex")
    _check(load().speed3r_sparse_global_attn_noalloc(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                                     _dev(out, "out", q.dtype), n_tok, heads, head_dim,
                                                     block, topk, _stream(stream)))


def speed3r_dense_attn(q, k, v, out, lse=None, softmax_scale=0.0, stream=None):
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    _check(load().speed3r_dense_attn(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                     _dev(out, "out", q.dtype), _dev(lse, "lse", torch.float32),
                                     n_tok, heads, head_dim, dt, float(softmax_scale), _stream(stream)))


def speed3r_pool_blocks(q, k, v, qc, kc, vc, block, stream=None):
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    f32 = torch.float32
    _check(load().speed3r_pool_blocks(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(qc, "qc", f32),
                                      _dev(kc, "kc", f32), _dev(vc, "vc", f32), n_tok, heads,
                                      head_dim, block, dt, _stream(stream)))


def speed3r_compress_attn_scores(qc, kc, vc, s_guide, o_comp, softmax_scale=0.0, accurate_pv=False,
                                 stream=None):
    heads, n_blk, head_dim = qc.shape
    if s_guide.dim() != 3 or s_guide.shape[0] != heads or s_guide.shape[1] != n_blk:
        raise ValueError("s_guide must be [heads, n_blk, ld_s]")
    f32 = torch.float32
    _check(load().speed3r_compress_attn_scores(_dev(qc, "qc", f32), _dev(kc, "kc", f32),
                                               _dev(vc, "vc", f32), _dev(s_guide, "s_guide", f32),
                                               s_guide.shape[2], _dev(o_comp, "o_comp", f32), n_blk,
                                               heads, head_dim, float(softmax_scale),
                                               int(bool(accurate_pv)), _stream(stream)))


def speed3r_compress_attn_topk(qc, kc, vc, o_comp, idx, topk, softmax_scale=0.0, accurate_pv=False, stream=None):
    heads, n_blk, head_dim = qc.shape
    f32 = torch.float32
    _check(load().speed3r_compress_attn_topk(_dev(qc, "qc", f32), _dev(kc, "kc", f32), _dev(vc, "vc", f32),
                                             _dev(o_comp, "o_comp", f32), _dev(idx, "idx", torch.int32), n_blk,
                                             heads, head_dim, int(topk), float(softmax_scale),
                                             int(bool(accurate_pv)), _stream(stream)))


def speed3r_topk_blocks(s_guide, idx, n_blk, topk, stream=None):
    heads, rows, ld_s = s_guide.shape
    if rows != n_blk:
        raise ValueError("s_guide must be [heads, n_blk, ld_s]")
    _check(load().speed3r_topk_blocks(_dev(s_guide, "s_guide", torch.float32), ld_s,
                                      _dev(idx, "idx", torch.int32), n_blk, heads, topk,
                                      _stream(stream)))


def speed3r_select_attn(q, k, v, idx, out, block, *, o_comp=None, gate_logits=None, o_sel=None,
                        lse=None, softmax_scale=0.0, stream=None):
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    if idx.dim() != 3 or idx.shape[0] != heads:
        raise ValueError("idx must be [heads, n_blk, kk]")
    _check(load().speed3r_select_attn(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                      _dev(idx, "idx", torch.int32),
                                      _dev(o_comp, "o_comp", torch.float32),
                                      _dev(gate_logits, "gate_logits", q.dtype),
                                      _dev(out, "out", q.dtype), _dev(o_sel, "o_sel", q.dtype),
                                      _dev(lse, "lse", torch.float32), n_tok, heads, head_dim, block,
                                      idx.shape[2], dt, float(softmax_scale), _stream(stream)))


# ---- cross attention and a cache in 4 bits ------------------------------------------------------------------
# Tensors may be on any GPU, all of a call on one; the launches go to that GPU's current stream.  A decoding step makes these
# calls for every layer and token: the checks are written to cost 3 to 4 us of a call's 8 (the launch itself takes 3.5).

def _gpu(t, name):
    """Index of the tensor's GPU."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name} must be a tensor on the GPU")
    return t.get_device()


def _arg(t, name, index, dtype, shape):
    """data_ptr of a contiguous tensor of that type and shape on GPU `index` (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        raise TypeError(f"{name} must be a tensor on GPU {index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows_arg(t, name, index, dtype, shape):
    """data_ptr and (row, head) strides of a tensor [rows, heads, head_dim] with contiguous channels.  A stride along an
    axis of one entry is not used and may be anything."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        raise TypeError(f"{name} must be a tensor on GPU {index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
    row, head = shape[1] * shape[2], shape[2]
    if not t.is_contiguous():
        if t.stride(2) != 1:
            raise TypeError(f"the channels of {name} must be contiguous")
        if shape[0] > 1:
            row = t.stride(0)
        if shape[1] > 1:
            head = t.stride(1)
        if row == 0 or head == 0:
            raise TypeError(f"{name} must not be broadcast along its rows or heads")
    return t.data_ptr(), row, head


def _kv_arg(k, v, index, dtype, shape):
    """data_ptrs of k and v and their common strides."""
    pk, row, head = _rows_arg(k, "k", index, dtype, shape)
    pv, v_row, v_head = _rows_arg(v, "v", index, dtype, shape)
    if (row, head) != (v_row, v_head):
        raise TypeError("k and v must share their row and head strides")
    return pk, pv, row, head


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _stream_of(stream, index):
    if isinstance(stream, torch.cuda.Stream) and stream.device_index != index:
        raise ValueError(f"stream belongs to GPU {stream.device_index}, the tensors to GPU {index}")
    return _raw_stream(index) if stream is None else _stream(stream)


def _empty_on(need, stream, index):
    """`need` bytes of the allocator's memory for the stream that uses them: it may be given to nothing else before that is done."""
    if stream is None:
        return torch.empty(need, dtype=torch.uint8, device=f"cuda:{index}")
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=index) if int(stream) else torch.cuda.default_stream(index)
    with torch.cuda.stream(stream):
        return torch.empty(need, dtype=torch.uint8, device=f"cuda:{index}")


def _call(fn, p, need, workspace, index, stream=None, *more):
    """The call with a workspace of `need` bytes (2^64 - 1: its arguments are wrong and the call says why), the caller's where there
    is one, and with `more` arguments behind p.  Returns the workspace."""
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor) or workspace.get_device() != index or workspace.dtype is not torch.uint8 \
                or not workspace.is_contiguous():
            raise TypeError(f"workspace must be a contiguous uint8 tensor on GPU {index}")
    elif 0 < need < 1 << 62:
        workspace = _empty_on(need, stream, index)
    if workspace is not None:
        p.workspace, p.workspace_bytes = workspace.data_ptr(), workspace.numel()
    if index == torch.cuda.current_device():
        status = fn(ctypes.byref(p), *more)
    else:
        with torch.cuda.device(index):
            status = fn(ctypes.byref(p), *more)
    if status != S3R_OK:
        raise Speed3rError(status, speed3r_last_error())
    return workspace


def _cross_params(q, k, v, out, lse, q_start, kv_start, key_mask, softmax_scale, accurate_pv, status, stream, index):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q must be [n_q, heads, head_dim], k and v [n_kv, kv_heads, head_dim]")
    n_q, heads, head_dim = shape = q.shape
    n_kv, kv_heads, _ = kv_shape = (k.shape[0], k.shape[1], head_dim)
    dtype = q.dtype
    pq, q_row, q_head = _rows_arg(q, "q", index, dtype, shape)
    pk, pv, kv_row, kv_head = _kv_arg(k, v, index, dtype, kv_shape)
    batch = 1 if q_start is None else q_start.numel() - 1
    if key_mask is not None and key_mask.dtype is torch.bool:
        key_mask = key_mask.view(torch.uint8)
    return s3r_cross_params(
        pq, pk, pv, _arg(out, "out", index, dtype, shape), _arg(lse, "lse", index, torch.float32, (heads, n_q)), None, None, None, None,
        _arg(q_start, "q_start", index, torch.int32, (batch + 1,)), _arg(kv_start, "kv_start", index, torch.int32, (batch + 1,)),
        _arg(key_mask, "key_mask", index, torch.uint8, (n_kv,)), _arg(status, "status", index, torch.int32, (1,)), n_q, n_kv,
        q_row, q_head, kv_row, kv_head, batch, heads, kv_heads, head_dim, _dtype_code(q), softmax_scale, None, 0, _stream_of(stream, index), int(bool(accurate_pv)))


def speed3r_cross_workspace_bytes(q, k, *, q_start=None, backward=False) -> int:
    """Bytes of workspace that speed3r_cross_attn, or its gradient, needs for these shapes (tensors, or anything
    with their `shape` and `dtype`)."""
    p = s3r_cross_params()
    p.n_q, p.heads, p.head_dim = q.shape
    p.n_kv, p.kv_heads = k.shape[0], k.shape[1]
    p.dtype = _dtype_code(q)
    p.batch = 1 if q_start is None else q_start.numel() - 1
    p.q_start = p.kv_start = None if q_start is None else 4          # only whether they are given counts here
    need = load().speed3r_cross_workspace_bytes(ctypes.byref(p), int(bool(backward)))
    if need >= 1 << 62:
        raise Speed3rError(S3R_ERR_INVALID_ARG, speed3r_last_error())
    return need


def speed3r_cross_attn(q, k, v, out, *, lse=None, q_start=None, kv_start=None, key_mask=None, softmax_scale=0.0,
                       accurate_pv=False, workspace=None, status=None, stream=None):
    """Attention of q [n_q, heads, 64] over k, v [n_kv, kv_heads, 64] into out (contiguous, like q); lse: fp32 [heads, n_q].
    q_start, kv_start: int32 [batch + 1], the sequences of a ragged batch; key_mask: bool or uint8 [n_kv], 0 leaves a key
    out; accurate_pv: bf16 probabilities enter their product in two parts, not one, also where there are many rows; status: int32 [1], receives 0 or
    S3R_DIAG_SPANS.  q, and k and v alike, may be strided views.  Returns the workspace used (None: none was needed)."""
    index, lib = _gpu(q, "q"), load()
    p = _cross_params(q, k, v, out, lse, q_start, kv_start, key_mask, softmax_scale, accurate_pv, status, stream, index)
    return _call(lib.speed3r_cross_attn, p, lib.speed3r_cross_workspace_bytes(ctypes.byref(p), 0), workspace, index, stream)


def speed3r_cross_attn_backward(q, k, v, out, lse, d_out, dq, dk, dv, *, q_start=None, kv_start=None, key_mask=None,
                                softmax_scale=0.0, accurate_pv=False, workspace=None, status=None, stream=None):
    """Gradients of speed3r_cross_attn into dq, dk, dv (contiguous, like q, k, v), from its out and lse and the gradient
    d_out of out.  The other arguments are those of the forward call (accurate_pv: of probabilities and dS here).  Returns the workspace used."""
    index, lib = _gpu(q, "q"), load()
    p = _cross_params(q, k, v, out, lse, q_start, kv_start, key_mask, softmax_scale, accurate_pv, status, stream, index)
    p.d_out, p.dq = _arg(d_out, "d_out", index, q.dtype, q.shape), _arg(dq, "dq", index, q.dtype, q.shape)
    p.dk, p.dv = _arg(dk, "dk", index, q.dtype, k.shape), _arg(dv, "dv", index, q.dtype, k.shape)
    return _call(lib.speed3r_cross_attn_backward, p, lib.speed3r_cross_workspace_bytes(ctypes.byref(p), 1), workspace, index, stream)


def _view_arg(tokens_per_view):
    # (one that 32 bits cannot hold is longer than every sequence; ctypes would cut it down)
    return max(-1, min(tokens_per_view, 2 ** 31 - 1))


def speed3r_causal_workspace_bytes(q, k, *, q_start=None, tokens_per_view=1, backward=False) -> int:
    """Bytes of workspace that speed3r_causal_attn, or its gradient, needs for these shapes (tensors, or anything
    with their `shape` and `dtype`)."""
    p = s3r_cross_params()
    p.n_q, p.heads, p.head_dim = q.shape
    p.n_kv, p.kv_heads = k.shape[0], k.shape[1]
    p.dtype = _dtype_code(q)
    p.batch = 1 if q_start is None else q_start.numel() - 1
    p.q_start = p.kv_start = None if q_start is None else 4          # only whether they are given counts here
    need = load().speed3r_causal_workspace_bytes(ctypes.byref(p), _view_arg(tokens_per_view), int(bool(backward)))
    if need >= 1 << 62:
        raise Speed3rError(S3R_ERR_INVALID_ARG, speed3r_last_error())
    return need


def speed3r_causal_attn(q, k, v, out, *, tokens_per_view=1, lse=None, q_start=None, kv_start=None, key_mask=None, softmax_scale=0.0,
                        accurate_pv=False, workspace=None, status=None, stream=None):
    """speed3r_cross_attn where the rows of a sequence are its last tokens, and each sees the tokens of its own view and of earlier ones
    (tokens_per_view 1: the tokens up to itself).  The other arguments are the same; q_start and kv_start are the same list where rows
    and keys are of the same tokens.  Returns the workspace used (None: none was needed)."""
    index, lib = _gpu(q, "q"), load()
    p = _cross_params(q, k, v, out, lse, q_start, kv_start, key_mask, softmax_scale, accurate_pv, status, stream, index)
    view = _view_arg(tokens_per_view)
    need = lib.speed3r_causal_workspace_bytes(ctypes.byref(p), view, 0)
    return _call(lib.speed3r_causal_attn, p, need, workspace, index, stream, view)


def speed3r_causal_attn_backward(q, k, v, out, lse, d_out, dq, dk, dv, *, tokens_per_view=1, q_start=None, kv_start=None, key_mask=None,
                                 softmax_scale=0.0, accurate_pv=False, workspace=None, status=None, stream=None):
    """Gradients of speed3r_causal_attn into dq, dk, dv (contiguous, like q, k, v), from its out and lse and the gradient
    d_out of out.  The other arguments are those of the forward call (accurate_pv: of probabilities and dS here).  Returns the workspace used."""
    index, lib = _gpu(q, "q"), load()
    p = _cross_params(q, k, v, out, lse, q_start, kv_start, key_mask, softmax_scale, accurate_pv, status, stream, index)
    p.d_out, p.dq = _arg(d_out, "d_out", index, q.dtype, q.shape), _arg(dq, "dq", index, q.dtype, q.shape)
    p.dk, p.dv = _arg(dk, "dk", index, q.dtype, k.shape), _arg(dv, "dv", index, q.dtype, k.shape)
    view = _view_arg(tokens_per_view)
    need = lib.speed3r_causal_workspace_bytes(ctypes.byref(p), view, 1)
    return _call(lib.speed3r_causal_attn_backward, p, need, workspace, index, stream, view)


class PagedCache(NamedTuple):
    """The four uint8 tensors of a cache in 4 bits: codes [n_pages, kv_heads, page, 32], scales [n_pages, kv_heads, page, 2]."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scales: torch.Tensor
    v_scales: torch.Tensor

    @classmethod
    def empty(cls, n_pages, kv_heads, page, device="cuda"):
        return cls(*(torch.zeros((n_pages, kv_heads, page, w), dtype=torch.uint8, device=device) for w in (32, 32, 2, 2)))


def _cache_params(cache, rows, page_table, kv_len, row_start, status, stream, index, *, q=None, out=None, k=None, v=None,
                  cos=None, sin=None, positions=None, pairs="halves", causal=0, softmax_scale=0.0, lse=None):
    """rows: the tensor [n_rows, heads, head_dim] whose heads count as the queries' and whose type as the rows'."""
    k_codes, v_codes, k_scales, v_scales = cache
    if k_codes.dim() != 4 or k_codes.shape[3] != 32:
        raise ValueError("codes must be [n_pages, kv_heads, page, 32]")
    if rows.dim() != 3:
        raise ValueError("rows must be [n_rows, heads, head_dim]")
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an int32 tensor [batch, max_pages]")
    u8, i32, dtype = torch.uint8, torch.int32, rows.dtype
    n_pages, kv_heads, page, _ = codes = k_codes.shape
    scales = (n_pages, kv_heads, page, 2)
    batch, max_pages = page_table.shape
    n_rows, heads, head_dim = rows.shape
    pq = pk = pv = None
    q_row = q_head = kv_row = kv_head = axes = places = 0
    if q is not None:
        pq, q_row, q_head = _rows_arg(q, "q", index, dtype, (n_rows, heads, head_dim))
    if k is not None:
        pk, pv, kv_row, kv_head = _kv_arg(k, v, index, dtype, (n_rows, kv_heads, head_dim))
    if cos is not None:
        if cos.dim() != 2 or cos.shape[1] not in (16, 32):
            raise ValueError("cos and sin must be [n_positions, 32], or [n_positions, 16] for two axes")
        axes, places = 32 // cos.shape[1], cos.shape[0]
        if positions is not None and axes == 1 and positions.dim() == 1:
            positions = positions[:, None]
    elif sin is not None or positions is not None:
        raise ValueError("sin and positions need cos")
    f32 = torch.float32
    return s3r_cache_params(
        _arg(k_codes, "k_codes", index, u8, codes), _arg(v_codes, "v_codes", index, u8, codes),
        _arg(k_scales, "k_scales", index, u8, scales), _arg(v_scales, "v_scales", index, u8, scales),
        _arg(page_table, "page_table", index, i32, page_table.shape), _arg(kv_len, "kv_len", index, i32, (batch,)),
        _arg(row_start, "row_start", index, i32, (batch + 1,)), n_pages, n_rows, page, max_pages, batch, heads, kv_heads, head_dim,
        _dtype_code(rows), pq, _arg(out, "out", index, dtype, (n_rows, heads, head_dim)), pk, pv, q_row, q_head, kv_row, kv_head,
        _arg(cos, "cos", index, f32, (places, 32 // max(axes, 1))), _arg(sin, "sin", index, f32, (places, 32 // max(axes, 1))),
        _arg(positions, "positions", index, i32, (n_rows, axes)), places, axes, int(pairs == "neighbours"), causal, softmax_scale,
        _arg(lse, "lse", index, f32, (heads, n_rows)), _arg(status, "status", index, i32, (1,)), None, 0, _stream_of(stream, index))


def speed3r_cache_append(cache, k, v, page_table, kv_len, row_start=None, *, q=None, q_out=None, cos=None, sin=None,
                         positions=None, pairs="halves", status=None, stream=None):
    """k, v [n_rows, kv_heads, 64] become the last tokens of their sequences in the cache (a PagedCache); kv_len int32 [batch]
    counts them.  page_table: int32 [batch, max_pages]; row_start: int32 [batch + 1] (None: one sequence).
    cos, sin: fp32 [n_positions, 32] rotate k by positions int32 [n_rows] (None: token numbers); of width 16 they rotate by
    two positions, int32 [n_rows, 2].  pairs: "halves" or "neighbours".  q [n_rows, heads, 64] is rotated into q_out."""
    index, lib = _gpu(cache[0], "the cache"), load()
    if pairs != "halves" and pairs != "neighbours":
        raise ValueError('pairs must be "halves" or "neighbours"')
    p = _cache_params(cache, k if q is None else q, page_table, kv_len, row_start, status, stream, index, q=q, out=q_out, k=k, v=v,
                      cos=cos, sin=sin, positions=positions, pairs=pairs)
    _call(lib.speed3r_cache_append, p, 0, None, index)


def speed3r_cache_read(cache, k, v, page_table, kv_len, row_start=None, *, status=None, stream=None):
    """The last tokens of the sequences, as many as k, v [n_rows, kv_heads, 64] have rows for them, as values into k and v."""
    index, lib = _gpu(cache[0], "the cache"), load()
    p = _cache_params(cache, k, page_table, kv_len, row_start, status, stream, index, k=k, v=v)
    _call(lib.speed3r_cache_read, p, 0, None, index)


def speed3r_cache_workspace_bytes(cache, n_rows, heads, dtype, batch, max_pages) -> int:
    """Bytes of workspace of speed3r_cache_attn; dtype: S3R_BF16 or S3R_F32."""
    p = s3r_cache_params()
    p.n_pages, p.kv_heads, p.page, _ = cache.k_codes.shape
    p.n_rows, p.heads, p.head_dim, p.dtype, p.batch, p.max_pages = n_rows, heads, HEAD_DIM, dtype, batch, max_pages
    p.row_start = 4                                                  # only whether it is given counts here
    need = load().speed3r_cache_workspace_bytes(ctypes.byref(p))
    if need >= 1 << 62:
        raise Speed3rError(S3R_ERR_INVALID_ARG, speed3r_last_error())
    return need


def speed3r_cache_attn(cache, q, out, page_table, kv_len, row_start=None, *, causal=True, lse=None, softmax_scale=0.0,
                       workspace=None, status=None, stream=None):
    """Attention of q [n_rows, heads, 64] (rotated already) over the cached tokens of their sequences into out.  The rows of a
    sequence are its last tokens; causal: each sees the tokens up to its own, otherwise all.  Returns the workspace used
    (None: none was needed)."""
    index, lib = _gpu(cache[0], "the cache"), load()
    p = _cache_params(cache, q, page_table, kv_len, row_start, status, stream, index, q=q, out=out, causal=int(bool(causal)),
                      softmax_scale=softmax_scale, lse=lse)
    return _call(lib.speed3r_cache_attn, p, lib.speed3r_cache_workspace_bytes(ctypes.byref(p)), workspace, index, stream)


# ---- rotary positions, and the residual stream with its norms ------------------------------------------------
_NORMS = {None: S3R_NORM_NONE, "rms": S3R_NORM_RMS, "layer": S3R_NORM_LAYER}
_PAIRS = {"halves": S3R_PAIRS_HALVES, "neighbours": S3R_PAIRS_NEIGHBOURS, "whole": S3R_PAIRS_WHOLE}


_ONE_AXIS = (32,)


_CODES = {torch.float32: S3R_F32, torch.bfloat16: S3R_BF16}


def _code(dtype, name):
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"{name} has unsupported dtype {dtype}")
    return code


def _weight_args(p, weights, dtype, index, shape):
    """Puts weights (by name) and the type that they have in common (none given: that of the rows) into p."""
    w_dtype = None
    for name, w in weights.items():
        if w is not None:
            if w_dtype is None:
                w_dtype = w.dtype
            setattr(p, name, _arg(w, name, index, w_dtype, shape))
    p.weight_dtype = _code(w_dtype or dtype, "a weight")


def _rotary_params(like_q, like_k, cos, sin, positions, axis_pairs, pairs, norm, eps, weights, status, stream, index):
    """weights: q_weight, q_bias, k_weight, k_bias and their gradients, by name."""
    like, heads, kv_heads = like_k if like_q is None else like_q, 0, 0
    if like.dim() != 3 or (like_k is not None and like_k.dim() != 3):
        raise ValueError("q and k must be [n_rows, heads, head_dim]")
    n_rows, heads, head_dim = like.shape
    dtype = like.dtype
    if like_q is None:
        heads, kv_heads = 0, heads
    elif like_k is not None:
        k_rows, kv_heads, k_dim = like_k.shape
        if k_rows != n_rows or k_dim != head_dim or like_k.dtype is not dtype:
            raise ValueError("q and k must share dtype, rows and head_dim")
    if pairs not in _PAIRS:
        raise ValueError(f"pairs must be one of {list(_PAIRS)}")
    if norm not in _NORMS:
        raise ValueError(f"norm must be one of {list(_NORMS)}")
    p = s3r_rotary_params()
    p.n_rows, p.heads, p.kv_heads, p.head_dim, p.dtype, p.pairs = n_rows, heads, kv_heads, head_dim, _code(dtype, "q or k"), _PAIRS[pairs]
    if cos is not None:
        if axis_pairs is None:
            axis_pairs = _ONE_AXIS
        if not 1 <= len(axis_pairs) <= 3:
            raise ValueError("axis_pairs must name 1 to 3 axes")
        p.axes, total, sizes = len(axis_pairs), 0, p.axis_pairs
        for i, n in enumerate(axis_pairs):
            sizes[i] = n
            total += n
        if cos.dim() != 2:
            raise ValueError("cos and sin must be [n_positions, pairs]")
        table = (cos.shape[0], total)
        p.n_positions, p.cos, p.sin = table[0], _arg(cos, "cos", index, torch.float32, table), _arg(sin, "sin", index, torch.float32, table)
        if positions is not None:
            if p.axes == 1 and positions.dim() == 1:
                positions = positions[:, None]
            p.positions = _arg(positions, "positions", index, torch.int32, (n_rows, p.axes))
    elif sin is not None or positions is not None or axis_pairs is not None:
        raise ValueError("sin, positions and axis_pairs need cos")
    if norm is not None:
        p.norm, p.eps = _NORMS[norm], eps
    _weight_args(p, weights, dtype, index, (head_dim,))
    if status is not None:
        p.status = _arg(status, "status", index, torch.int32, (1,))
    p.stream = _stream_of(stream, index)
    return p


def speed3r_rotary(q, k, q_out, k_out, cos=None, sin=None, positions=None, *, axis_pairs=None, pairs="halves", norm=None, eps=1e-6,
                   q_weight=None, q_bias=None, k_weight=None, k_bias=None, status=None, stream=None):
    """q [n_rows, heads, 64] and k [n_rows, kv_heads, 64] (either may be None), normed head by head (norm: None, "rms" or "layer";
    weights and biases: [64], all fp32 or all bf16) and rotated, into q_out and k_out (contiguous).  axis_pairs: channel pairs of each
    of up to three axes, by default (32,); cos, sin: fp32 [n_positions, pairs of all axes]; positions: int32 [n_rows, axes] (one axis: may be
    [n_rows], or None: row numbers); pairs: "halves" of an axis' channels, "neighbours", or "whole": halves of all axes' channels
    together.  Without cos nothing is rotated.  status: int32 [1], receives 0 or S3R_DIAG_POSITION.  q and k may be strided views."""
    index, lib = _gpu(k if q is None else q, "q" if k is None else "k"), load()
    p = _rotary_params(q, k, cos, sin, positions, axis_pairs, pairs, norm, eps,
                       {"q_weight": q_weight, "q_bias": q_bias, "k_weight": k_weight, "k_bias": k_bias}, status, stream, index)
    if q is not None:
        p.q, p.q_stride_tok, p.q_stride_head = _rows_arg(q, "q", index, q.dtype, q.shape)
        p.q_out = _arg(q_out, "q_out", index, q.dtype, q.shape)
    if k is not None:
        p.k, p.k_stride_tok, p.k_stride_head = _rows_arg(k, "k", index, k.dtype, k.shape)
        p.k_out = _arg(k_out, "k_out", index, k.dtype, k.shape)
    _call(lib.speed3r_rotary, p, 0, None, index)


def speed3r_rotary_workspace_bytes(weight_gradients=True) -> int:
    """Bytes of workspace of speed3r_rotary_backward, with gradients of weights or without (the same for all shapes)."""
    p = s3r_rotary_params()
    p.heads, p.head_dim, p.norm, p.eps, p.dtype = 1, HEAD_DIM, S3R_NORM_RMS, 1.0, S3R_BF16
    p.dq_weight = 16 if weight_gradients else None                   # only whether it is given counts here
    return load().speed3r_rotary_workspace_bytes(ctypes.byref(p))


def speed3r_rotary_backward(q, k, d_q_out, d_k_out, dq, dk, cos=None, sin=None, positions=None, *, axis_pairs=None, pairs="halves",
                            norm=None, eps=1e-6, q_weight=None, k_weight=None, dq_weight=None, dq_bias=None, dk_weight=None,
                            dk_bias=None, workspace=None, status=None, stream=None):
    """Gradients of speed3r_rotary from those of q_out and k_out (contiguous) into dq and dk (which may be strided views: parts of the
    gradient of a packed projection), and those of weights and biases that are given.  Without a norm q and k are not
    read and may be None.  The other arguments are those of the forward call.  Returns the workspace used (None: none was needed)."""
    like_q, like_k = d_q_out, d_k_out
    index, lib = _gpu(like_k if like_q is None else like_q, "d_q_out" if like_k is None else "d_k_out"), load()
    p = _rotary_params(like_q, like_k, cos, sin, positions, axis_pairs, pairs, norm, eps,
                       {"q_weight": q_weight, "k_weight": k_weight, "dq_weight": dq_weight, "dq_bias": dq_bias, "dk_weight": dk_weight,
                        "dk_bias": dk_bias}, status, stream, index)
    if like_q is not None:
        if q is not None:
            p.q, p.q_stride_tok, p.q_stride_head = _rows_arg(q, "q", index, like_q.dtype, like_q.shape)
        p.d_q_out = _arg(d_q_out, "d_q_out", index, like_q.dtype, like_q.shape)
        p.dq, p.dq_stride_tok, p.dq_stride_head = _rows_arg(dq, "dq", index, like_q.dtype, like_q.shape)
    if like_k is not None:
        if k is not None:
            p.k, p.k_stride_tok, p.k_stride_head = _rows_arg(k, "k", index, like_k.dtype, like_k.shape)
        p.d_k_out = _arg(d_k_out, "d_k_out", index, like_k.dtype, like_k.shape)
        p.dk, p.dk_stride_tok, p.dk_stride_head = _rows_arg(dk, "dk", index, like_k.dtype, like_k.shape)
    return _call(lib.speed3r_rotary_backward, p, lib.speed3r_rotary_workspace_bytes(ctypes.byref(p)), workspace, index, stream)


def _matrix_arg(t, name, index, dtype, shape):
    """data_ptr and row stride of a tensor [rows, width] with contiguous channels."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        raise TypeError(f"{name} must be a tensor on GPU {index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
    row = shape[1]
    if not t.is_contiguous():
        if t.stride(1) != 1:
            raise TypeError(f"the channels of {name} must be contiguous")
        if shape[0] > 1:
            row = t.stride(0)
        if row == 0:
            raise TypeError(f"{name} must not be broadcast along its rows")
    return t.data_ptr(), row


def _residual_params(x, like, f, norm, post_norm, eps, weights, gate, row_start, residual_scale, status, stream, index):
    """like: a tensor of the type that all but the stream have, or None: that of x."""
    if x.dim() != 2:
        raise ValueError("x must be [n_rows, width]")
    if norm not in _NORMS or post_norm not in _NORMS:
        raise ValueError(f"norm and post_norm must be among {list(_NORMS)}")
    if residual_scale == 0:
        raise ValueError("residual_scale must not be 0")
    shape = n_rows, width = x.shape
    dtype = x.dtype if like is None else like.dtype
    p = s3r_residual_params()
    p.n_rows, p.width, p.x_dtype, p.dtype = n_rows, width, _code(x.dtype, "x"), _code(dtype, "f or y")
    p.x, p.x_stride = _matrix_arg(x, "x", index, x.dtype, shape)
    if f is not None:
        p.f, p.f_stride = _matrix_arg(f, "f", index, dtype, shape)
    _weight_args(p, weights, dtype, index, (width,))
    p.batch = 1 if row_start is None else row_start.numel() - 1
    if gate is not None:
        p.gate, p.gate_stride = _matrix_arg(gate, "gate", index, dtype, (p.batch, width))
    if row_start is not None:
        p.row_start = _arg(row_start, "row_start", index, torch.int32, (p.batch + 1,))
    p.norm, p.post_norm, p.eps, p.residual_scale = _NORMS[norm], _NORMS[post_norm], eps, residual_scale
    if status is not None:
        p.status = _arg(status, "status", index, torch.int32, (1,))
    p.stream = _stream_of(stream, index)
    return p


def speed3r_residual_norm(x, y=None, *, f=None, r=None, norm=None, weight=None, bias=None, eps=1e-6, post_norm=None, post_weight=None,
                          post_bias=None, scale=None, gate=None, row_start=None, residual_scale=1.0, status=None, stream=None):
    """r = x + residual_scale * scale * gate * (f, normed by post_norm or not), and y = norm(r), for x and f [n_rows, width]; without f
    r is x.  r (of x's type; may be x itself) and y (of f's type) are contiguous, either may be None.  norm, post_norm: None, "rms" or
    "layer"; weights, biases and scale: [width], all fp32 or all bf16; gate: [batch, width], of f's type, for the sequences whose rows
    start at row_start (int32 [batch + 1]; None: one sequence).  x may be fp32 where f and y are bf16.  x, f and gate may have strides
    between rows.  status: int32 [1], receives 0 or S3R_DIAG_SPANS."""
    index, lib = _gpu(x, "x"), load()
    p = _residual_params(x, y if f is None else f, f, norm, post_norm, eps,
                         {"weight": weight, "bias": bias, "post_weight": post_weight, "post_bias": post_bias, "scale": scale},
                         gate, row_start, residual_scale, status, stream, index)
    if r is not None:
        p.r = _arg(r, "r", index, x.dtype, x.shape)
    if y is not None:
        p.y = _arg(y, "y", index, y.dtype if f is None else f.dtype, x.shape)
    _call(lib.speed3r_residual_norm, p, 0, None, index)


def speed3r_residual_workspace_bytes(n_rows, width, *, batch=1, weight_gradients=True, gate_gradients=False) -> int:
    """Bytes of workspace of speed3r_residual_norm_backward; weight_gradients: of any of weights, biases and scale."""
    p = s3r_residual_params()
    p.n_rows, p.width, p.batch, p.norm, p.eps = n_rows, width, batch, S3R_NORM_RMS, 1.0
    p.f = p.gate = p.row_start = 16                                  # only whether they are given counts here
    p.d_weight, p.d_gate = 16 if weight_gradients else None, 16 if gate_gradients else None
    need = load().speed3r_residual_workspace_bytes(ctypes.byref(p))
    if need >= 1 << 62:
        raise Speed3rError(S3R_ERR_INVALID_ARG, speed3r_last_error())
    return need


def speed3r_residual_norm_backward(x, d_y, dx, *, f=None, d_r=None, df=None, norm=None, weight=None, eps=1e-6, post_norm=None,
                                   post_weight=None, post_bias=None, scale=None, gate=None, row_start=None, residual_scale=1.0,
                                   d_weight=None, d_bias=None, d_post_weight=None, d_post_bias=None, d_scale=None, d_gate=None,
                                   workspace=None, status=None, stream=None):
    """Gradients of speed3r_residual_norm from those of y and r (d_y, d_r; contiguous, either may be None) into dx and df, and into
    those of weights, scale and gate that are given (each like its tensor).  The other arguments are those of the forward call.  Returns the
    workspace used (None: none was needed)."""
    index, lib = _gpu(x, "x"), load()
    p = _residual_params(x, d_y if f is None else f, f, norm, post_norm, eps,
                         {"weight": weight, "post_weight": post_weight, "post_bias": post_bias, "scale": scale, "d_weight": d_weight,
                          "d_bias": d_bias, "d_post_weight": d_post_weight, "d_post_bias": d_post_bias, "d_scale": d_scale},
                         gate, row_start, residual_scale, status, stream, index)
    dtype = x.dtype if d_y is None and f is None else (d_y if f is None else f).dtype
    p.d_y, p.d_r = _arg(d_y, "d_y", index, dtype, x.shape), _arg(d_r, "d_r", index, x.dtype, x.shape)
    p.dx, p.df = _arg(dx, "dx", index, x.dtype, x.shape), _arg(df, "df", index, dtype, x.shape)
    if d_gate is not None:
        p.d_gate = _arg(d_gate, "d_gate", index, dtype, (p.batch, x.shape[1]))
    return _call(lib.speed3r_residual_norm_backward, p, lib.speed3r_residual_workspace_bytes(ctypes.byref(p)), workspace, index, stream)


def speed3r_probe_select_loads(q, k, v, idx, out, block, ring_stages=0, wg_per_cu=0, stream=None):
    """The selection kernel's data movement without its arithmetic (measurement utility); out receives q.
    ring_stages 0/2..4 and wg_per_cu 0/1..5 vary the LDS ring depth and the workgroups per CU."""
    n_tok, heads, head_dim, dt = _qkv(q, k, v)
    if dt != S3R_BF16 or idx.dim() != 3 or idx.shape[0] != heads:
        raise ValueError("bf16 q, k, v and idx [heads, n_blk, kk] expected")
    _check(load().speed3r_probe_select_loads(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(idx, "idx", torch.int32),
                                             _dev(out, "out", q.dtype), n_tok, heads, head_dim, block, idx.shape[2],
                                             int(ring_stages), int(wg_per_cu), _stream(stream)))


def speed3r_set_profiling(enable: bool):
    _check(load().speed3r_set_profiling(int(bool(enable))))


def speed3r_get_stage_ms():
    """(ms, launches) dictionaries keyed by stage name, summed over the profiled calls since the
    previous read."""
    ms = (_flt * len(STAGES))()
    n = (_int * len(STAGES))()
    _check(load().speed3r_get_stage_ms(ms, n))
    return ({s: float(ms[i]) for i, s in enumerate(STAGES)},
            {s: int(n[i]) for i, s in enumerate(STAGES)})


def speed3r_set_kernel_choice(choice: int):
    _check(load().speed3r_set_kernel_choice(int(choice)))


def speed3r_release_scratch():
    _check(load().speed3r_release_scratch())
