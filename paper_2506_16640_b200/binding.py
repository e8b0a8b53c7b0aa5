"""Thin ctypes binding of ``libentmax_attn.so``: argument marshalling only.

Same entry-point names as ``include/entmax_attn.h``.  PyTorch supplies device memory and streams;
every step of the computation runs in the library's CUDA kernels.  There is no fallback: if the
library is missing or a call is rejected, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libentmax_attn.so")

DTYPE_BF16, DTYPE_FP32 = 0, 1
STATUS_WORDS = 8
STATUS_FLAGS, STATUS_DENSE_ROWS, STATUS_TILE_SWEEPS, STATUS_TILES = 0, 1, 2, 3
STATUS_SKIPPED_STEPS, STATUS_SCORED_STEPS = 4, 5
FLAG_WAIT_EXPIRED, FLAG_BAD_SCALE, FLAG_BAD_LENGTH, FLAG_BAD_PAGE, FLAG_NO_PAGES = 1, 2, 4, 8, 16
PAGED_MAX_KV = 1 << 24


class Params(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seq", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("n_mode", ctypes.c_int32), ("alpha", ctypes.c_float), ("sm_scale", ctypes.c_float),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


class DecodeParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("q_len", ctypes.c_int32),
                ("kv_capacity", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("alpha", ctypes.c_float),
                ("sm_scale", ctypes.c_float), ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64),
                ("kv_stride_n", ctypes.c_int64)]


class ProjParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seq", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("x_dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("n_mode", ctypes.c_int32),
                ("gamma_range", ctypes.c_float)]


class PagedCache(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("table_stride", ctypes.c_int64), ("stride_page", ctypes.c_int64), ("stride_token", ctypes.c_int64),
                ("stride_head", ctypes.c_int64)]


class PagedAppendParams(ctypes.Structure):
    _fields_ = [("total_q", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("rot_positions", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("q_stride_t", ctypes.c_int64),
                ("q_stride_h", ctypes.c_int64), ("k_stride_t", ctypes.c_int64), ("k_stride_h", ctypes.c_int64),
                ("v_stride_t", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("out_stride_t", ctypes.c_int64),
                ("out_stride_h", ctypes.c_int64)]


class PagedParams(ctypes.Structure):
    _fields_ = [("total_q", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("max_q_len", ctypes.c_int32),
                ("max_kv_len", ctypes.c_int32), ("alpha", ctypes.c_float), ("sm_scale", ctypes.c_float),
                ("q_stride_t", ctypes.c_int64), ("q_stride_h", ctypes.c_int64)]


class Strides(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("n", ctypes.c_int64)]


class SoftmaxParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("seq", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("softcap", ctypes.c_float), ("q", Strides), ("k", Strides), ("v", Strides), ("o", Strides)]


class SoftmaxTerms(ctypes.Structure):
    _fields_ = [("row_ranges", ctypes.c_void_p), ("beta", ctypes.c_void_p), ("gamma", ctypes.c_void_p), ("delta", ctypes.c_void_p),
                ("c_rows", ctypes.c_void_p), ("alibi_slopes", ctypes.c_void_p)]


class SoftmaxGrads(ctypes.Structure):
    _fields_ = [("d_o", Strides), ("dq", Strides), ("dk", Strides), ("dv", Strides), ("d_scale_rows", ctypes.c_void_p),
                ("dbeta", ctypes.c_void_p), ("dgamma", ctypes.c_void_p), ("ddelta", ctypes.c_void_p)]


class SoftmaxPagedParams(ctypes.Structure):
    _fields_ = [("total_q", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("max_q_len", ctypes.c_int32), ("max_kv_len", ctypes.c_int32),
                ("window", ctypes.c_int32), ("softcap", ctypes.c_float), ("sm_scale", ctypes.c_float), ("q_stride_t", ctypes.c_int64),
                ("q_stride_h", ctypes.c_int64)]


class PagedTablesParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("total_q", ctypes.c_int32), ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("free_capacity", ctypes.c_int32), ("table_stride", ctypes.c_int64)]


class WsLayout(ctypes.Structure):
    _fields_ = [("row_count_offset", ctypes.c_size_t), ("entries_offset", ctypes.c_size_t),
                ("scale_offset", ctypes.c_size_t), ("dense_count_offset", ctypes.c_size_t),
                ("capacity", ctypes.c_int32), ("keep_limit", ctypes.c_int32)]


class Extras(ctypes.Structure):
    _fields_ = [("c_rows", ctypes.c_void_p), ("alibi_slopes", ctypes.c_void_p), ("d_scale_rows", ctypes.c_void_p),
                ("dbeta", ctypes.c_void_p), ("dgamma", ctypes.c_void_p), ("ddelta", ctypes.c_void_p),
                ("fwd_workspace", ctypes.c_void_p), ("saved_supports", ctypes.c_void_p)]


class EntmaxAttnError(RuntimeError):
    pass


_lib = None


def load():
    """Loads the CUDA library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise EntmaxAttnError(
                "libentmax_attn.so is missing: build it with `python -m paper_2506_16640_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, fp, ip = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(Params)
        lib.entmax_attn_workspace_bytes.restype = ctypes.c_size_t
        lib.entmax_attn_workspace_bytes.argtypes = [pp, ctypes.c_int]
        lib.entmax_attn_workspace_layout.restype = ctypes.c_int
        lib.entmax_attn_workspace_layout.argtypes = [pp, ctypes.POINTER(WsLayout)]
        lib.entmax_attn_fwd.restype = ctypes.c_int
        lib.entmax_attn_fwd.argtypes = [pp, vp, vp, vp, fp, fp, fp, vp, fp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_bwd.restype = ctypes.c_int
        lib.entmax_attn_bwd.argtypes = [pp, vp, vp, vp, fp, fp, fp, fp, vp, vp, vp, vp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_bwd_scale.restype = ctypes.c_int
        lib.entmax_attn_bwd_scale.argtypes = [pp, vp, vp, vp, fp, fp, fp, fp, vp, vp, vp, vp, fp, fp, fp, fp, vp,
                                              ctypes.c_size_t, ip, vp]
        ep = ctypes.POINTER(Extras)
        lib.entmax_attn_fwd_ex.restype = ctypes.c_int
        lib.entmax_attn_fwd_ex.argtypes = [pp, vp, vp, vp, fp, fp, fp, ep, vp, fp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_bwd_ex.restype = ctypes.c_int
        lib.entmax_attn_bwd_ex.argtypes = [pp, vp, vp, vp, fp, fp, fp, ep, fp, vp, vp, vp, vp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_fwd_rowscale.restype = ctypes.c_int
        lib.entmax_attn_fwd_rowscale.argtypes = [pp, vp, vp, vp, fp, vp, fp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_bwd_rowscale.restype = ctypes.c_int
        lib.entmax_attn_bwd_rowscale.argtypes = [pp, vp, vp, vp, fp, fp, vp, vp, vp, vp, fp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_fwd_static.restype = ctypes.c_int
        lib.entmax_attn_fwd_static.argtypes = [pp, vp, vp, vp, fp, fp, fp, vp, fp, ip, vp]
        dp = ctypes.POINTER(DecodeParams)
        lib.entmax_attn_decode_workspace_bytes.restype = ctypes.c_size_t
        lib.entmax_attn_decode_workspace_bytes.argtypes = [dp]
        lib.entmax_attn_decode_fwd.restype = ctypes.c_int
        lib.entmax_attn_decode_fwd.argtypes = [dp, vp, vp, vp, ip, fp, fp, fp, fp, vp, fp, ip, vp, ctypes.c_size_t, ip, vp]
        cp, ap, gp = ctypes.POINTER(PagedCache), ctypes.POINTER(PagedAppendParams), ctypes.POINTER(PagedParams)
        lib.entmax_attn_paged_append.restype = ctypes.c_int
        lib.entmax_attn_paged_append.argtypes = [cp, ap, vp, vp, vp, fp, ip, ip, ip, vp, vp, vp, ip, vp]
        lib.entmax_attn_paged_workspace_bytes.restype = ctypes.c_size_t
        lib.entmax_attn_paged_workspace_bytes.argtypes = [cp, gp, ctypes.c_int]
        lib.entmax_attn_paged_fwd.restype = ctypes.c_int
        lib.entmax_attn_paged_fwd.argtypes = [cp, gp, vp, vp, vp, ip, ip, ip, fp, fp, fp, fp, vp, fp, ip, vp, ctypes.c_size_t,
                                              ip, vp]
        sp, tp, sg, kp = (ctypes.POINTER(t) for t in (SoftmaxParams, SoftmaxTerms, SoftmaxGrads, SoftmaxPagedParams))
        lib.entmax_attn_softmax_fwd.restype = ctypes.c_int
        lib.entmax_attn_softmax_fwd.argtypes = [sp, vp, vp, vp, tp, vp, fp, ip, vp]
        lib.entmax_attn_softmax_workspace_bytes.restype = ctypes.c_size_t
        lib.entmax_attn_softmax_workspace_bytes.argtypes = [sp]
        lib.entmax_attn_softmax_bwd.restype = ctypes.c_int
        lib.entmax_attn_softmax_bwd.argtypes = [sp, vp, vp, vp, tp, vp, fp, vp, sg, vp, vp, vp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_row_ranges.restype = ctypes.c_int
        lib.entmax_attn_row_ranges.argtypes = [ctypes.c_int32] * 5 + [ip, ip, ip, vp]
        lib.entmax_attn_softmax_paged_workspace_bytes.restype = ctypes.c_size_t
        lib.entmax_attn_softmax_paged_workspace_bytes.argtypes = [cp, kp, ctypes.c_int]
        lib.entmax_attn_softmax_paged_fwd.restype = ctypes.c_int
        lib.entmax_attn_softmax_paged_fwd.argtypes = [cp, kp, vp, vp, vp, ip, ip, ip, fp, fp, fp, fp, vp, fp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_paged_tables.restype = ctypes.c_int
        lib.entmax_attn_paged_tables.argtypes = [ctypes.POINTER(PagedTablesParams)] + [ip] * 11 + [vp]
        lib.entmax_attn_saved_bytes.restype = ctypes.c_size_t
        lib.entmax_attn_saved_bytes.argtypes = [pp]
        lib.entmax_attn_save_supports.restype = ctypes.c_int
        lib.entmax_attn_save_supports.argtypes = [pp, vp, vp, ctypes.c_size_t, vp]
        lib.entmax_attn_scores_debug.restype = ctypes.c_int
        lib.entmax_attn_scores_debug.argtypes = [pp, vp, vp, ctypes.c_int32, fp, vp, ctypes.c_size_t, ip, vp]
        lib.entmax_attn_profile_events.restype = ctypes.c_int
        lib.entmax_attn_profile_events.argtypes = [ctypes.c_int, vp, vp]
        jp = ctypes.POINTER(ProjParams)
        lib.entmax_attn_scale_proj_fwd.restype = ctypes.c_int
        lib.entmax_attn_scale_proj_fwd.argtypes = [jp, vp, fp, fp, fp, fp, vp]
        lib.entmax_attn_scale_proj_bwd.restype = ctypes.c_int
        lib.entmax_attn_scale_proj_bwd.argtypes = [jp, vp, fp, fp, fp, fp, fp, fp, vp, vp]
        lib.entmax_attn_selftest_wait_expiry.restype = ctypes.c_int
        lib.entmax_attn_selftest_wait_expiry.argtypes = [ctypes.c_uint64, ip, vp]
        lib.entmax_attn_strerror.restype = ctypes.c_char_p
        lib.entmax_attn_strerror.argtypes = [ctypes.c_int]
        lib.entmax_attn_last_cuda_error.restype = ctypes.c_int
        lib.entmax_attn_version.restype = ctypes.c_int
        _lib = lib
    return _lib


def _check(rc: int, what: str):
    if rc != 0:
        lib = load()
        msg = lib.entmax_attn_strerror(rc).decode()
        extra = ""
        if rc == -7:
            extra = " (cudaError %d)" % lib.entmax_attn_last_cuda_error()
        raise EntmaxAttnError("%s failed: %s%s" % (what, msg, extra))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()      # the argtypes say c_void_p: a plain int converts fastest


def make_params(q: torch.Tensor, alpha: float, causal: bool, sm_scale: float = 0.0, n_mode: int = 0) -> Params:
    if q.dim() != 4:
        raise EntmaxAttnError("expected [batch, heads, seq, head_dim] tensors")
    if q.dtype == torch.bfloat16:
        dt = DTYPE_BF16
    elif q.dtype == torch.float32:
        dt = DTYPE_FP32
    else:
        raise EntmaxAttnError("dtype must be bfloat16 or float32")
    sb, sh, sn, sd = q.stride()
    if sd != 1:
        raise EntmaxAttnError("head_dim must be the innermost, contiguous dimension")
    B, H, N, D = q.shape
    return Params(B, H, N, D, dt, int(bool(causal)), int(n_mode), float(alpha), float(sm_scale), sb, sh, sn)


def _same_layout(ref: torch.Tensor, *others):
    shape, stride, dtype, device = ref.shape, ref.stride(), ref.dtype, ref.device
    for t in others:
        if t.shape != shape or t.stride() != stride or t.dtype != dtype or t.device != device:
            raise EntmaxAttnError("all [B,H,N,D] tensors of a call must share shape, strides, dtype and device")


def entmax_attn_workspace_bytes(params: Params, is_bwd: bool) -> int:
    return int(load().entmax_attn_workspace_bytes(ctypes.byref(params), int(bool(is_bwd))))


def entmax_attn_workspace_layout(params: Params) -> WsLayout:
    out = WsLayout()
    _check(load().entmax_attn_workspace_layout(ctypes.byref(params), ctypes.byref(out)), "entmax_attn_workspace_layout")
    return out


def alloc_workspace(params: Params, is_bwd: bool, device) -> torch.Tensor:
    nbytes = entmax_attn_workspace_bytes(params, is_bwd)
    if nbytes == 0:
        raise EntmaxAttnError("invalid parameters (workspace size query returned 0)")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)   # torch's allocator aligns to >= 512 B


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    # the current stream's handle without a Stream object around it (5 us of the 21 a small call took)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def entmax_attn_fwd(q, k, v, alpha, causal, beta=None, gamma=None, delta=None, *, sm_scale=0.0, n_mode=0,
                    o=None, tau=None, workspace=None, status=None, stream=None):
    """Forward pass.  Returns (o, tau).  `workspace` (uint8 CUDA tensor) and `status` (int32[4] CUDA
    tensor) are allocated when not given; pass your own to inspect them afterwards."""
    _same_layout(q, k, v)
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    if o is None:
        o = torch.empty_like(q)
    else:
        _same_layout(q, o)
    B, H, N, _ = q.shape
    if tau is None:
        tau = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(params, False, q.device)
    rc = load().entmax_attn_fwd(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma), _ptr(delta),
                                _ptr(o), _ptr(tau), _ptr(workspace), workspace.numel(), _ptr(status),
                                _stream_ptr(stream))
    _check(rc, "entmax_attn_fwd")
    return o, tau


def entmax_attn_fwd_static(q, k, v, alpha, causal, beta=None, gamma=None, delta=None, *, sm_scale=0.0, n_mode=0,
                           o, tau, status=None, stream=None):
    """Forward pass without a workspace, for callers that cannot allocate device memory: the scratch is
    a fixed array inside the library.  `o` and `tau` must be passed in (this wrapper allocates nothing
    either).  Raises EntmaxAttnError when the problem exceeds the built-in scratch.  Calls that overlap
    on the GPU share that scratch and race; keep them on one stream."""
    _same_layout(q, k, v, o)
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    rc = load().entmax_attn_fwd_static(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma),
                                       _ptr(delta), _ptr(o), _ptr(tau), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_fwd_static")
    return o, tau


def entmax_attn_decode_fwd(q, k, v, alpha, kv_len=None, beta=None, gamma=None, delta=None, *, alibi_slopes=None,
                           sm_scale=0.0, o=None, tau=None, support_size=None, workspace=None, status=None,
                           stream=None):
    """Decode-shape forward: q [B,H,q_len,d] (contiguous) against the cache k, v [B,H,kv_capacity,d] (any
    strides with d innermost, e.g. a view of a [B,kv_capacity,H,d] cache), kv_len int32 [B] or None.
    Returns (o, tau, support_size)."""
    if q.dtype != torch.bfloat16 or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
        raise EntmaxAttnError("entmax_attn_decode_fwd: bf16 tensors only")
    if not q.is_contiguous() or k.stride() != v.stride() or k.shape != v.shape or k.stride(3) != 1:
        raise EntmaxAttnError("entmax_attn_decode_fwd: q contiguous; k and v the same shape and strides, d innermost")
    B, H, QL, D = q.shape
    if k.shape[0] != B or k.shape[1] != H or k.shape[3] != D:
        raise EntmaxAttnError("entmax_attn_decode_fwd: q and k/v disagree on batch, heads or head_dim")
    params = DecodeParams(B, H, QL, k.shape[2], D, float(alpha), float(sm_scale), k.stride(0), k.stride(1), k.stride(2))
    o = torch.empty_like(q) if o is None else o
    tau = torch.empty((B, H, QL), dtype=torch.float32, device=q.device) if tau is None else tau
    if support_size is None:
        support_size = torch.empty((B, H, QL), dtype=torch.int32, device=q.device)
    if workspace is None:
        nbytes = load().entmax_attn_decode_workspace_bytes(ctypes.byref(params))
        if nbytes == 0:
            raise EntmaxAttnError("entmax_attn_decode_workspace_bytes: invalid parameters")
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    rc = load().entmax_attn_decode_fwd(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(kv_len), _ptr(beta),
                                       _ptr(gamma), _ptr(delta), _ptr(alibi_slopes), _ptr(o), _ptr(tau),
                                       _ptr(support_size), _ptr(workspace), workspace.numel(), _ptr(status),
                                       _stream_ptr(stream))
    _check(rc, "entmax_attn_decode_fwd")
    return o, tau, support_size


def rotation_table(positions: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """float32 [positions, rot_dim] for entmax_attn_paged_append: cosines, then sines, of position * base^(-2i / rot_dim), computed in
    64 bits (in 32 the angle of a position near 10^6 is off by 0.03)."""
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-2.0 * i / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32).to(device)


# The paged calls sit in a serving loop, one of each per layer and step, where checking some forty shapes, strides and dtypes and filling in
# the parameter structures took 20 of the 30 us a small call needed.  All of that depends on the tensors' layouts alone, so it is done
# once per combination of layouts and looked up afterwards (nothing of the tensors themselves is kept).  Hashing the layouts costs as much as
# the checks did, so they are found under a few of their numbers and compared.
_layouts: dict = {}
_LAYOUTS_KEPT = 512


def _layout_of(*tensors):
    return tuple([None if t is None else (t.dtype, t.shape, t.stride(), t.get_device()) for t in tensors])


def _keep(where, key, value):
    if len(_layouts) >= _LAYOUTS_KEPT:
        _layouts.clear()
    _layouts[where] = key, value
    return value


def _row_strides(name, x, heads, d):
    """(token, head) strides of a bf16 [tokens, heads, d] tensor; a dimension of one element has no stride of its own."""
    if x.dim() != 3 or x.dtype != torch.bfloat16 or x.shape[1] != heads or x.shape[2] != d or x.stride(2) != 1:
        raise EntmaxAttnError("%s must be a bfloat16 [tokens, %d, %d] tensor with the last dimension contiguous" % (name, heads, d))
    return x.stride(0) if x.shape[0] > 1 else heads * d, x.stride(1) if heads > 1 else d


def _paged_cache(what, k_cache, v_cache, block_table, kv_len, cu_q, status, total_q, device):
    if k_cache.dim() != 4 or k_cache.dtype != torch.bfloat16 or k_cache.stride(3) != 1:
        raise EntmaxAttnError("%s: k_cache must be a bfloat16 [pages, page_size, kv_heads, head_dim] tensor, head_dim contiguous" % what)
    if v_cache.shape != k_cache.shape or v_cache.stride() != k_cache.stride() or v_cache.dtype != k_cache.dtype:
        raise EntmaxAttnError("%s: k_cache and v_cache must share shape, strides and dtype" % what)
    if block_table.dim() != 2 or block_table.dtype != torch.int32 or block_table.stride(1) != 1 and block_table.shape[1] > 1:
        raise EntmaxAttnError("%s: block_table must be an int32 [batch, max_pages] tensor with contiguous rows" % what)
    B, max_pages = block_table.shape
    if kv_len.shape != (B,) or kv_len.dtype != torch.int32 or not kv_len.is_contiguous():
        raise EntmaxAttnError("%s: kv_len must be a contiguous int32 [batch] tensor" % what)
    if cu_q is not None and (cu_q.shape != (B + 1,) or cu_q.dtype != torch.int32 or not cu_q.is_contiguous()):
        raise EntmaxAttnError("%s: cu_q must be a contiguous int32 [batch + 1] tensor" % what)
    if cu_q is None and B and total_q % B:
        raise EntmaxAttnError("%s: without cu_q the number of new tokens must be a multiple of the batch" % what)
    if status is not None and (status.dtype != torch.int32 or status.numel() < STATUS_WORDS or not status.is_contiguous()):
        raise EntmaxAttnError("%s: status must be a contiguous int32 tensor of %d words" % (what, STATUS_WORDS))
    for t in (k_cache, v_cache, block_table, kv_len, cu_q, status):
        if t is not None and t.device != device:
            raise EntmaxAttnError("%s: all tensors must be on one device" % what)
    P, ps, KH, D = k_cache.shape
    return PagedCache(B, KH, D, ps, P, max_pages, block_table.stride(0) if B > 1 else max_pages,
                      k_cache.stride(0) if P > 1 else ps * KH * D, k_cache.stride(1), k_cache.stride(2) if KH > 1 else D)


def _on_device(device):
    """The launches go to the current device's context: made the tensors' own for the call where it is another."""
    if device < 0:
        raise EntmaxAttnError("CUDA tensors only (there is no CPU fallback)")
    return torch.cuda.device(device) if device != torch._C._cuda_getDevice() else None


def _call_on(device, fn, *args):
    guard = _on_device(device)
    if guard is None:
        return fn(*args)
    with guard:
        return fn(*args)


def _new_on(stream, like, shape, dtype):
    """A tensor that the allocator gives away again in the order of the stream the call runs on."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _like_on(stream, like):
    """The same, contiguous with the shape and dtype of `like` (1 us less than by shape)."""
    if stream is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):
        return torch.empty_like(like, memory_format=torch.contiguous_format)


def _clear_status(status, stream):
    """What the library does at the start of a call, for a call that has nothing to launch."""
    if status is None:
        return
    if stream is None:
        status.zero_()
    else:
        with torch.cuda.stream(stream):
            status.zero_()


def _append_layout(what, q, k, v, k_cache, v_cache, block_table, kv_len, cu_q, rotation, interleaved, q_out, status):
    T, KH, D = k.shape if k.dim() == 3 else (0, 0, 0)
    ks, vs = _row_strides("k", k, KH, D), _row_strides("v", v, KH, D)
    cache = _paged_cache(what, k_cache, v_cache, block_table, kv_len, cu_q, status, T, k.device)
    if (cache.kv_heads, cache.head_dim) != (KH, D) or v.shape != k.shape or v.device != k.device:
        raise EntmaxAttnError("%s: k, v and the cache disagree on tokens, kv_heads, head_dim or device" % what)
    H, qs, os_ = 0, (D, D), (D, D)
    if q is not None:
        H = q.shape[1] if q.dim() == 3 else 0
        qs = _row_strides("q", q, H, D)
        os_ = (H * D, D) if q_out is None else _row_strides("q_out", q_out, H, D)
        if q.shape[0] != T or q.device != k.device or q_out is not None and (q_out.shape != q.shape or q_out.device != k.device):
            raise EntmaxAttnError("%s: q, q_out and k disagree on tokens or device" % what)
    elif q_out is not None:
        raise EntmaxAttnError("%s: q_out without q" % what)
    rot_pos, rot = 0, 0
    if rotation is not None:
        if rotation.dim() != 2 or rotation.dtype != torch.float32 or not rotation.is_contiguous() or rotation.device != k.device:
            raise EntmaxAttnError("%s: rotation must be a contiguous float32 [positions, rot_dim] tensor on the device of k" % what)
        rot_pos, rot = rotation.shape
    params = PagedAppendParams(T, H, rot, rot_pos, int(bool(interleaved)), *qs, *ks, *vs, *os_)
    return ctypes.byref(cache), ctypes.byref(params), T, H, D


def entmax_attn_paged_append(q, k, v, k_cache, v_cache, block_table, kv_len, cu_q=None, *, rotation=None, interleaved=False,
                             q_out=None, status=None, stream=None):
    """Rotates new queries and keys to their positions and appends keys and values to a paged cache, in one pass.

    q [T, H, d] (or None), k, v [T, kv_heads, d]: the new tokens' rows, bf16, any strides with d contiguous; k_cache, v_cache
    [pages, page_size, kv_heads, d], written in place (a [pages, kv_heads, page_size, d] pool as its transpose(1, 2));
    block_table int32 [B, max_pages]; kv_len int32 [B], new tokens included; cu_q int32 [B + 1]: rows cu_q[b] .. cu_q[b+1] - 1
    are sequence b's (None: T / B each).  rotation: float32 [positions, rot_dim] (rotation_table) or None; interleaved: pairs
    (2i, 2i + 1) instead of (i, i + rot_dim / 2).  Returns the rotated q (q_out; may be q itself)."""
    what = "entmax_attn_paged_append"
    where = (what, k.numel(), k_cache.numel(), block_table.numel())
    key = (interleaved, _layout_of(q, k, v, k_cache, v_cache, block_table, kv_len, cu_q, rotation, q_out, status))
    known = _layouts.get(where)
    cache, params, T, H, D = known[1] if known is not None and known[0] == key else _keep(where, key, _append_layout(
        what, q, k, v, k_cache, v_cache, block_table, kv_len, cu_q, rotation, interleaved, q_out, status))
    device = k.get_device()
    if q is not None and q_out is None:
        q_out = _new_on(stream, q, (T, H, D), torch.bfloat16)
    if T == 0:
        _clear_status(status, stream)
        return q_out
    rc = _call_on(device, lambda: load().entmax_attn_paged_append(
        cache, params, _ptr(q), k.data_ptr(), v.data_ptr(), _ptr(rotation), _ptr(cu_q), kv_len.data_ptr(), block_table.data_ptr(), _ptr(q_out),
        k_cache.data_ptr(), v_cache.data_ptr(), _ptr(status), _stream_ptr(stream)))
    _check(rc, what)
    return q_out


def entmax_attn_paged_workspace_bytes(cache: PagedCache, params: PagedParams, uniform: bool) -> int:
    return int(load().entmax_attn_paged_workspace_bytes(ctypes.byref(cache), ctypes.byref(params), int(bool(uniform))))


def _paged_layout(what, q, k_cache, v_cache, alpha, block_table, kv_len, cu_q, beta, gamma, delta, alibi_slopes, sm_scale, max_q_len,
                  max_kv_len, o, tau, support_size, status):
    T, H, D = q.shape if q.dim() == 3 else (0, 0, 0)
    params = PagedParams(T, H, int(max_q_len), int(max_kv_len), float(alpha), float(sm_scale), *_row_strides("q", q, H, D))
    device = q.device
    cache = _paged_cache(what, k_cache, v_cache, block_table, kv_len, cu_q, status, T, device)
    if cache.head_dim != D:
        raise EntmaxAttnError("%s: q and the cache disagree on head_dim" % what)
    for name, t in (("beta", beta), ("gamma", gamma), ("delta", delta), ("alibi_slopes", alibi_slopes)):
        if t is not None and (t.shape != (H,) or t.dtype != torch.float32 or not t.is_contiguous() or t.device != device):
            raise EntmaxAttnError("%s: %s must be a contiguous float32 [%d] tensor on the device of q" % (what, name, H))
    for name, t, shape, dtype in (("o", o, (T, H, D), torch.bfloat16), ("tau", tau, (T, H), torch.float32),
                                  ("support_size", support_size, (T, H), torch.int32)):
        if t is not None and (t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.device != device):
            raise EntmaxAttnError("%s: %s must be a contiguous %s %s tensor on the device of q" % (what, name, dtype, list(shape)))
    # (0 bytes: parameters that the call itself refuses, with the reason)
    return (ctypes.byref(cache), ctypes.byref(params), T, H, D, entmax_attn_paged_workspace_bytes(cache, params, cu_q is None) if T else 0)


def entmax_attn_paged_fwd(q, k_cache, v_cache, alpha, block_table, kv_len, cu_q=None, beta=None, gamma=None, delta=None, *,
                          alibi_slopes=None, sm_scale=0.0, max_q_len=0, max_kv_len=0, o=None, tau=None, support_size=None,
                          workspace=None, status=None, stream=None):
    """Attention of new tokens over a paged cache that already holds their keys and values: q [T, H, d] bf16, packed as in
    entmax_attn_paged_append, H a multiple of the cache's kv_heads (query heads h * H / kv_heads .. share K/V head h).  One new
    token per sequence, a chunk, or whole prompts, mixed as they come.  max_q_len, max_kv_len: the most new tokens and the
    longest kv_len of the call, where the caller knows them (they size the workspace and the launches).
    Returns (o [T, H, d], tau [T, H], support_size [T, H] or None where no tensor was given for it)."""
    what = "entmax_attn_paged_fwd"
    where = (what, q.numel(), k_cache.numel(), block_table.numel(), max_q_len, max_kv_len)
    key = (alpha, sm_scale, _layout_of(q, k_cache, v_cache, block_table, kv_len, cu_q, beta, gamma, delta, alibi_slopes, o, tau, support_size,
                                       status))
    known = _layouts.get(where)
    cache, params, T, H, D, nbytes = known[1] if known is not None and known[0] == key else _keep(where, key, _paged_layout(
        what, q, k_cache, v_cache, alpha, block_table, kv_len, cu_q, beta, gamma, delta, alibi_slopes, sm_scale, max_q_len, max_kv_len, o,
        tau, support_size, status))
    device = q.get_device()
    if o is None:
        o = _new_on(stream, q, (T, H, D), torch.bfloat16)
    if tau is None:
        tau = _new_on(stream, q, (T, H), torch.float32)
    if T == 0:
        _clear_status(status, stream)
        return o, tau, support_size
    if workspace is None:
        workspace = _new_on(stream, q, (nbytes,), torch.uint8)
    elif workspace.dtype != torch.uint8 or workspace.get_device() != device or not workspace.is_contiguous():
        raise EntmaxAttnError("%s: workspace must be a contiguous uint8 tensor on the device of q" % what)
    rc = _call_on(device, lambda: load().entmax_attn_paged_fwd(
        cache, params, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), _ptr(cu_q), kv_len.data_ptr(), block_table.data_ptr(), _ptr(beta),
        _ptr(gamma), _ptr(delta), _ptr(alibi_slopes), o.data_ptr(), tau.data_ptr(), _ptr(support_size), workspace.data_ptr(),
        workspace.numel(), _ptr(status), _stream_ptr(stream)))
    _check(rc, what)
    return o, tau, support_size


def _softmax_paged_layout(what, q, k_cache, v_cache, block_table, kv_len, cu_q, beta, gamma, delta, alibi_slopes, softcap, window, sm_scale,
                          max_q_len, max_kv_len, o, lse, status):
    T, H, D = q.shape if q.dim() == 3 else (0, 0, 0)
    params = SoftmaxPagedParams(T, H, int(max_q_len), int(max_kv_len), int(window), float(softcap), float(sm_scale), *_row_strides("q", q, H, D))
    device = q.device
    cache = _paged_cache(what, k_cache, v_cache, block_table, kv_len, cu_q, status, T, device)
    if cache.head_dim != D:
        raise EntmaxAttnError("%s: q and the cache disagree on head_dim" % what)
    _check_tensors(what, device, ("beta", beta, (H,), torch.float32), ("gamma", gamma, (H,), torch.float32), ("delta", delta, (H,), torch.float32),
                   ("alibi_slopes", alibi_slopes, (H,), torch.float32), ("o", o, (T, H, D), torch.bfloat16), ("lse", lse, (T, H), torch.float32))
    # (0 bytes: parameters that the call itself refuses, with the reason)
    nbytes = int(load().entmax_attn_softmax_paged_workspace_bytes(ctypes.byref(cache), ctypes.byref(params), int(cu_q is None))) if T else 0
    return ctypes.byref(cache), ctypes.byref(params), T, H, D, nbytes


def entmax_attn_softmax_paged_fwd(q, k_cache, v_cache, block_table, kv_len, cu_q=None, beta=None, gamma=None, delta=None, *,
                                  alibi_slopes=None, softcap=0.0, window=0, sm_scale=0.0, max_q_len=0, max_kv_len=0, o=None, lse=None,
                                  workspace=None, status=None, stream=None):
    """Softmax attention of new tokens over a paged cache that already holds their keys and values: tensors, packing and lengths as for
    entmax_attn_paged_fwd; softcap caps the scores by a tanh, window > 0 leaves a token its last `window` keys.
    Returns (o [T, H, d], lse [T, H])."""
    what = "entmax_attn_softmax_paged_fwd"
    where = (what, q.numel(), k_cache.numel(), block_table.numel(), max_q_len, max_kv_len)
    key = (softcap, window, sm_scale, _layout_of(q, k_cache, v_cache, block_table, kv_len, cu_q, beta, gamma, delta, alibi_slopes, o, lse, status))
    known = _layouts.get(where)
    cache, params, T, H, D, nbytes = known[1] if known is not None and known[0] == key else _keep(where, key, _softmax_paged_layout(
        what, q, k_cache, v_cache, block_table, kv_len, cu_q, beta, gamma, delta, alibi_slopes, softcap, window, sm_scale, max_q_len, max_kv_len,
        o, lse, status))
    device = q.get_device()
    if o is None:
        o = _like_on(stream, q)
    if lse is None:
        lse = _new_on(stream, q, (T, H), torch.float32)
    if T == 0:
        _clear_status(status, stream)
        return o, lse
    if workspace is None:
        workspace = _new_on(stream, q, (nbytes,), torch.uint8)
    elif workspace.dtype != torch.uint8 or workspace.get_device() != device or not workspace.is_contiguous():
        raise EntmaxAttnError("%s: workspace must be a contiguous uint8 tensor on the device of q" % what)
    rc = _call_on(device, lambda: load().entmax_attn_softmax_paged_fwd(
        cache, params, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), _ptr(cu_q), kv_len.data_ptr(), block_table.data_ptr(), _ptr(beta),
        _ptr(gamma), _ptr(delta), _ptr(alibi_slopes), o.data_ptr(), lse.data_ptr(), workspace.data_ptr(), workspace.numel(), _ptr(status),
        _stream_ptr(stream)))
    _check(rc, what)
    return o, lse


def _check_tensors(what, device, *named):
    for name, t, shape, dtype in named:
        if t is not None and (t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.device != device):
            raise EntmaxAttnError("%s: %s must be a contiguous %s %s tensor on %s" % (what, name, dtype, list(shape), device))


def _tables_layout(what, kv_len, new_len, block_table, free_pages, free_count, page_size, num_pages, total_q, kv_len_out, cu_q, positions, slots,
                   free_count_out, status):
    i32, device = torch.int32, kv_len.device
    if block_table.dim() != 2 or block_table.dtype != i32 or block_table.device != device or block_table.shape[1] > 1 and block_table.stride(1) != 1:
        raise EntmaxAttnError("%s: block_table must be an int32 [batch, max_pages] tensor with contiguous rows, on the device of kv_len" % what)
    B, max_pages = block_table.shape
    _check_tensors(what, device, ("kv_len", kv_len, (B,), i32), ("new_len", new_len, (B,), i32), ("free_pages", free_pages, (free_pages.numel(),), i32),
                   ("free_count", free_count, (1,), i32), ("kv_len_out", kv_len_out, (B,), i32), ("cu_q", cu_q, (B + 1,), i32),
                   ("positions", positions, (total_q,), i32), ("slots", slots, (total_q,), torch.int64), ("free_count_out", free_count_out, (1,), i32))
    if status is not None and (status.dtype != i32 or status.numel() < STATUS_WORDS or not status.is_contiguous() or status.device != device):
        raise EntmaxAttnError("%s: status must be a contiguous int32 tensor of %d words on the device of kv_len" % (what, STATUS_WORDS))
    return ctypes.byref(PagedTablesParams(B, int(total_q), int(page_size), int(num_pages), max_pages, free_pages.numel(),
                                          block_table.stride(0) if B > 1 else max_pages)), B


def entmax_attn_paged_tables(kv_len, new_len, block_table, free_pages, free_count, page_size, num_pages, total_q, *, kv_len_out=None, cu_q=None,
                             positions=None, slots=None, free_count_out=None, status=None, stream=None):
    """Tables of a serving step from the requests' lengths, on the GPU: kv_len int32 [B] tokens in the cache, new_len int32 [B] tokens to
    come (-1: the sequence has ended and gives its pages back), block_table int32 [B, max_pages] (completed in place), free_pages int32 [capacity]
    and free_count int32 [1], a stack of free pages, total_q the sum of the new tokens.  kv_len_out and free_count_out may be kv_len and free_count.
    Returns (kv_len_out [B], cu_q [B + 1], positions [total_q] int32, slots [total_q] int64, free_count_out [1])."""
    what = "entmax_attn_paged_tables"
    where = (what, kv_len.numel(), block_table.numel(), free_pages.numel(), total_q)
    key = (page_size, num_pages, _layout_of(kv_len, new_len, block_table, free_pages, free_count, kv_len_out, cu_q, positions, slots, free_count_out,
                                            status))
    known = _layouts.get(where)
    params, B = known[1] if known is not None and known[0] == key else _keep(where, key, _tables_layout(
        what, kv_len, new_len, block_table, free_pages, free_count, page_size, num_pages, total_q, kv_len_out, cu_q, positions, slots,
        free_count_out, status))
    kv_len_out = _like_on(stream, kv_len) if kv_len_out is None else kv_len_out
    cu_q = _new_on(stream, kv_len, (B + 1,), torch.int32) if cu_q is None else cu_q
    positions = _new_on(stream, kv_len, (total_q,), torch.int32) if positions is None else positions
    slots = _new_on(stream, kv_len, (total_q,), torch.int64) if slots is None else slots
    free_count_out = _like_on(stream, free_count) if free_count_out is None else free_count_out
    # (an empty tensor has no address, and without positions and slots the library does not hold the new tokens to total_q: any address stands
    # for no rows)
    rc = _call_on(kv_len.get_device(), lambda: load().entmax_attn_paged_tables(
        params, kv_len.data_ptr(), new_len.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(), kv_len_out.data_ptr(),
        cu_q.data_ptr(), positions.data_ptr() or cu_q.data_ptr(), slots.data_ptr(), free_count_out.data_ptr(), _ptr(status), _stream_ptr(stream)))
    _check(rc, what)
    return kv_len_out, cu_q, positions, slots, free_count_out


def entmax_attn_row_ranges(cu_docs, seq, causal, *, prefix_len=None, window=0, row_ranges=None, stream=None):
    """The keys each row sees when documents are packed into a batch row: cu_docs int32 [B, docs + 1] boundaries, prefix_len int32 [B, docs] or
    None (tokens every row of the document sees; causal only), window > 0: the last `window` keys.  Tokens in no document see nothing.
    Returns int32 [B, seq, 2] for entmax_attn_softmax_fwd and softmax_attention, which are then called with causal=False."""
    what = "entmax_attn_row_ranges"
    if cu_docs.dim() != 2 or cu_docs.shape[1] < 2 or cu_docs.dtype != torch.int32 or not cu_docs.is_contiguous():
        raise EntmaxAttnError("%s: cu_docs must be a contiguous int32 [batch, docs + 1] tensor" % what)
    B, docs = cu_docs.shape[0], cu_docs.shape[1] - 1
    _check_tensors(what, cu_docs.device, ("prefix_len", prefix_len, (B, docs), torch.int32), ("row_ranges", row_ranges, (B, seq, 2), torch.int32))
    if row_ranges is None:
        row_ranges = _new_on(stream, cu_docs, (B, seq, 2), torch.int32)
    rc = _call_on(cu_docs.get_device(), lambda: load().entmax_attn_row_ranges(
        B, int(seq), docs, int(bool(causal)), int(window), cu_docs.data_ptr(), _ptr(prefix_len), row_ranges.data_ptr(), _stream_ptr(stream)))
    _check(rc, what)
    return row_ranges


def _strides4(what, name, x, shape, dtype, device):
    if x.shape != shape or x.dtype != dtype or x.device != device or x.stride(3) != 1:
        raise EntmaxAttnError("%s: %s must be a %s %s tensor on %s with the last dimension contiguous" % (what, name, dtype, list(shape), device))
    # (a dimension of one entry may have any stride; 0 throughout would mean "contiguous")
    return Strides(x.stride(0), x.stride(1), max(x.stride(2), 1))


def _softmax_layout(what, q, k, v, causal, beta, gamma, delta, c_rows, alibi_slopes, row_ranges, softcap, sm_scale, o, lse, status, d_o, dq, dk,
                    dv, d_scale_rows, bwd):
    if q.dim() != 4 or k.dim() != 4:
        raise EntmaxAttnError("%s: expected [batch, heads, seq, head_dim] tensors" % what)
    if q.dtype not in (torch.bfloat16, torch.float32):
        raise EntmaxAttnError("%s: dtype must be bfloat16 or float32" % what)
    (B, H, N, D), G, dev, dt = q.shape, k.shape[1], q.device, q.dtype
    shape, kv = (B, H, N, D), (B, G, N, D)
    strides = lambda name, x, sh: _strides4(what, name, x, sh, dt, dev)  # noqa: E731
    none = Strides(0, 0, 0)
    params = SoftmaxParams(B, H, G, N, D, DTYPE_BF16 if dt == torch.bfloat16 else DTYPE_FP32, int(bool(causal)), float(sm_scale), float(softcap),
                           strides("q", q, shape), strides("k", k, kv), strides("v", v, kv), none if o is None else strides("o", o, shape))
    f32 = torch.float32
    _check_tensors(what, dev, ("beta", beta, (H,), f32), ("gamma", gamma, (H,), f32), ("delta", delta, (H,), f32), ("c_rows", c_rows, (B, H, N), f32),
                   ("alibi_slopes", alibi_slopes, (H,), f32), ("row_ranges", row_ranges, (B, N, 2), torch.int32), ("lse", lse, (B, H, N), f32),
                   ("d_scale_rows", d_scale_rows, (B, H, N), f32))
    if status is not None and (status.dtype != torch.int32 or status.numel() < STATUS_WORDS or not status.is_contiguous() or status.device != dev):
        raise EntmaxAttnError("%s: status must be a contiguous int32 tensor of %d words on the device of q" % (what, STATUS_WORDS))
    if not bwd:
        return params, None, 0
    grads = SoftmaxGrads(strides("d_o", d_o, shape), *(none if x is None else strides(name, x, sh) for name, x, sh in
                                                      (("dq", dq, shape), ("dk", dk, kv), ("dv", dv, kv))), None, None, None, None)
    return params, grads, int(load().entmax_attn_softmax_workspace_bytes(ctypes.byref(params)))


def entmax_attn_softmax_fwd(q, k, v, causal, beta=None, gamma=None, delta=None, *, c_rows=None, alibi_slopes=None, row_ranges=None, softcap=0.0,
                            sm_scale=0.0, o=None, lse=None, status=None, stream=None):
    """Softmax attention (alpha -> 1) of q [B,H,N,d], k, v [B,G,N,d] (H a multiple of G; bf16 or fp32, each with strides of its own, d contiguous):
    scores c (softcap tanh(z / softcap) - slope |i - j|), c from beta, gamma, delta [H] or c_rows [B,H,N]; row_ranges int32 [B,N,2]: the keys a row
    sees (entmax_attn_row_ranges).  Returns (o, lse)."""
    what = "entmax_attn_softmax_fwd"
    where = (what, q.numel(), k.numel())
    key = (causal, softcap, sm_scale, _layout_of(q, k, v, beta, gamma, delta, c_rows, alibi_slopes, row_ranges, o, lse, status))
    known = _layouts.get(where)
    params, _, _ = known[1] if known is not None and known[0] == key else _keep(where, key, _softmax_layout(
        what, q, k, v, causal, beta, gamma, delta, c_rows, alibi_slopes, row_ranges, softcap, sm_scale, o, lse, status, None, None, None, None, None,
        False))
    B, H, N, _ = shape = q.shape
    if o is None:
        o = _like_on(stream, q)
    if lse is None:
        lse = _new_on(stream, q, (B, H, N), torch.float32)
    terms = SoftmaxTerms(_ptr(row_ranges), _ptr(beta), _ptr(gamma), _ptr(delta), _ptr(c_rows), _ptr(alibi_slopes))
    rc = _call_on(q.get_device(), lambda: load().entmax_attn_softmax_fwd(
        ctypes.byref(params), q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(terms), o.data_ptr(), lse.data_ptr(), _ptr(status),
        _stream_ptr(stream)))
    _check(rc, what)
    return o, lse


def entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, causal, beta=None, gamma=None, delta=None, *, c_rows=None, alibi_slopes=None, row_ranges=None,
                            softcap=0.0, sm_scale=0.0, want_scale_rows=False, want_param_grads=False, dq=None, dk=None, dv=None,
                            d_scale_rows=None, workspace=None, status=None, stream=None):
    """Backward pass of entmax_attn_softmax_fwd, whose o and lse it takes.
    Returns (dq, dk, dv, d_scale_rows or None, (dbeta, dgamma, ddelta) or None)."""
    what = "entmax_attn_softmax_bwd"
    where = (what, q.numel(), k.numel())
    key = (causal, softcap, sm_scale, _layout_of(q, k, v, beta, gamma, delta, c_rows, alibi_slopes, row_ranges, o, lse, status, d_o, dq, dk, dv,
                                                 d_scale_rows))
    known = _layouts.get(where)
    params, strides, nbytes = known[1] if known is not None and known[0] == key else _keep(where, key, _softmax_layout(
        what, q, k, v, causal, beta, gamma, delta, c_rows, alibi_slopes, row_ranges, softcap, sm_scale, o, lse, status, d_o, dq, dk, dv, d_scale_rows,
        True))
    B, H, N, _ = q.shape
    dq = _like_on(stream, q) if dq is None else dq
    dk = _like_on(stream, k) if dk is None else dk
    dv = _like_on(stream, v) if dv is None else dv
    if d_scale_rows is None and want_scale_rows:
        d_scale_rows = _new_on(stream, q, (B, H, N), torch.float32)
    if want_param_grads and (beta is None or gamma is None or delta is None):
        raise EntmaxAttnError("%s: there are no scale parameters to take gradients of" % what)
    params_grads = tuple([_like_on(stream, x) for x in (beta, gamma, delta)]) if want_param_grads else None
    if workspace is None:
        workspace = _new_on(stream, q, (nbytes,), torch.uint8)
    elif workspace.dtype != torch.uint8 or workspace.get_device() != q.get_device() or not workspace.is_contiguous():
        raise EntmaxAttnError("%s: workspace must be a contiguous uint8 tensor on the device of q" % what)
    g = params_grads or (None, None, None)
    terms = SoftmaxTerms(_ptr(row_ranges), _ptr(beta), _ptr(gamma), _ptr(delta), _ptr(c_rows), _ptr(alibi_slopes))
    grads = SoftmaxGrads(strides.d_o, strides.dq, strides.dk, strides.dv, _ptr(d_scale_rows), _ptr(g[0]), _ptr(g[1]), _ptr(g[2]))
    rc = _call_on(q.get_device(), lambda: load().entmax_attn_softmax_bwd(
        ctypes.byref(params), q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(terms), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(),
        ctypes.byref(grads), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), workspace.numel(), _ptr(status),
        _stream_ptr(stream)))
    _check(rc, what)
    return dq, dk, dv, d_scale_rows, params_grads


def _param_grads(H: int, device):
    # three tensors, not views of one: the caller may change, free or save each by itself
    f32 = torch.float32
    return torch.empty(H, dtype=f32, device=device), torch.empty(H, dtype=f32, device=device), torch.empty(H, dtype=f32, device=device)


def entmax_attn_bwd(q, k, v, tau, d_o, alpha, causal, beta=None, gamma=None, delta=None, *, sm_scale=0.0, n_mode=0,
                    dq=None, dk=None, dv=None, workspace=None, status=None, stream=None):
    """Backward pass.  Returns (dq, dk, dv)."""
    _same_layout(q, k, v, d_o)
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    _same_layout(q, dq, dk, dv)
    if workspace is None:
        workspace = alloc_workspace(params, True, q.device)
    rc = load().entmax_attn_bwd(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma), _ptr(delta),
                                _ptr(tau), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                workspace.numel(), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_bwd")
    return dq, dk, dv


def entmax_attn_bwd_scale(q, k, v, tau, d_o, alpha, causal, beta, gamma, delta, *, sm_scale=0.0, n_mode=0,
                          dq=None, dk=None, dv=None, d_scale_rows=None, want_param_grads=True, workspace=None,
                          status=None, stream=None):
    """Backward pass with the gradients of the ASEntmax scale.
    Returns (dq, dk, dv, d_scale_rows, (dbeta, dgamma, ddelta) or None)."""
    _same_layout(q, k, v, d_o)
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    _same_layout(q, dq, dk, dv)
    B, H, N, _ = q.shape
    if d_scale_rows is None:
        d_scale_rows = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    grads = None
    if want_param_grads:
        grads = _param_grads(H, q.device)
    if workspace is None:
        workspace = alloc_workspace(params, True, q.device)
    g = grads if grads is not None else (None, None, None)
    rc = load().entmax_attn_bwd_scale(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma),
                                      _ptr(delta), _ptr(tau), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv),
                                      _ptr(d_scale_rows), _ptr(g[0]), _ptr(g[1]), _ptr(g[2]), _ptr(workspace),
                                      workspace.numel(), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_bwd_scale")
    return dq, dk, dv, d_scale_rows, grads


def entmax_attn_fwd_rowscale(q, k, v, c_rows, alpha, causal, *, sm_scale=0.0, o=None, tau=None, workspace=None,
                             status=None, stream=None):
    """Forward pass with a per-query scale table c_rows (float32 [B,H,N]).  Returns (o, tau)."""
    _same_layout(q, k, v)
    params = make_params(q, alpha, causal, sm_scale, 0)
    B, H, N, _ = q.shape
    if c_rows.shape != (B, H, N) or c_rows.dtype != torch.float32 or not c_rows.is_contiguous():
        raise EntmaxAttnError("c_rows must be a contiguous float32 [batch, heads, seq] tensor")
    o = torch.empty_like(q) if o is None else o
    if tau is None:
        tau = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(params, False, q.device)
    rc = load().entmax_attn_fwd_rowscale(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(c_rows), _ptr(o),
                                         _ptr(tau), _ptr(workspace), workspace.numel(), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_fwd_rowscale")
    return o, tau


def entmax_attn_bwd_rowscale(q, k, v, c_rows, tau, d_o, alpha, causal, *, sm_scale=0.0, dq=None, dk=None, dv=None,
                             d_scale_rows=None, workspace=None, status=None, stream=None):
    """Backward pass with a per-query scale table.  Returns (dq, dk, dv, d_scale_rows)."""
    _same_layout(q, k, v, d_o)
    params = make_params(q, alpha, causal, sm_scale, 0)
    B, H, N, _ = q.shape
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    if d_scale_rows is None:
        d_scale_rows = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(params, True, q.device)
    rc = load().entmax_attn_bwd_rowscale(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(c_rows), _ptr(tau),
                                         _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(d_scale_rows), _ptr(workspace),
                                         workspace.numel(), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_bwd_rowscale")
    return dq, dk, dv, d_scale_rows


def entmax_attn_fwd_ex(q, k, v, alpha, causal, beta=None, gamma=None, delta=None, *, c_rows=None, alibi_slopes=None,
                       sm_scale=0.0, n_mode=0, o=None, tau=None, workspace=None, status=None, stream=None):
    """Extended forward pass: optional per-query scale table and ALiBi slopes.  Returns (o, tau)."""
    _same_layout(q, k, v)
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    B, H, N, _ = q.shape
    o = torch.empty_like(q) if o is None else o
    if tau is None:
        tau = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(params, False, q.device)
    ex = Extras(_ptr(c_rows), _ptr(alibi_slopes), None, None, None, None, None)
    rc = load().entmax_attn_fwd_ex(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma), _ptr(delta),
                                   ctypes.byref(ex), _ptr(o), _ptr(tau), _ptr(workspace), workspace.numel(),
                                   _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_fwd_ex")
    return o, tau


def entmax_attn_save_supports(q, alpha, causal, fwd_workspace, *, sm_scale=0.0, n_mode=0, saved=None, stream=None):
    """Compact copy of a finished forward call's supports (uint8 CUDA tensor) for entmax_attn_bwd_ex(saved_supports=...)."""
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    nbytes = load().entmax_attn_saved_bytes(ctypes.byref(params))
    if nbytes == 0:
        raise EntmaxAttnError("entmax_attn_saved_bytes: invalid parameters (bf16 problems only)")
    if saved is None:
        saved = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    rc = load().entmax_attn_save_supports(ctypes.byref(params), _ptr(fwd_workspace), _ptr(saved), saved.numel(),
                                          _stream_ptr(stream))
    _check(rc, "entmax_attn_save_supports")
    return saved


def entmax_attn_bwd_ex(q, k, v, tau, d_o, alpha, causal, beta=None, gamma=None, delta=None, *, c_rows=None,
                       alibi_slopes=None, fwd_workspace=None, saved_supports=None, want_scale_rows=False,
                       want_param_grads=False,
                       sm_scale=0.0, n_mode=0, dq=None, dk=None, dv=None, workspace=None, status=None, stream=None):
    """Extended backward pass.  `fwd_workspace`: the forward call's workspace tensor, untouched since
    (the backward pass then reuses the supports it holds instead of sweeping Q K^T again).
    Returns (dq, dk, dv, d_scale_rows or None, (dbeta, dgamma, ddelta) or None)."""
    _same_layout(q, k, v, d_o)
    params = make_params(q, alpha, causal, sm_scale, n_mode)
    B, H, N, _ = q.shape
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    dc = torch.empty((B, H, N), dtype=torch.float32, device=q.device) if want_scale_rows else None
    grads = _param_grads(H, q.device) if want_param_grads else None
    g = grads if grads is not None else (None, None, None)
    if workspace is None:
        workspace = alloc_workspace(params, True, q.device)
    ex = Extras(_ptr(c_rows), _ptr(alibi_slopes), _ptr(dc), _ptr(g[0]), _ptr(g[1]), _ptr(g[2]), _ptr(fwd_workspace),
                _ptr(saved_supports))
    rc = load().entmax_attn_bwd_ex(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma), _ptr(delta),
                                   ctypes.byref(ex), _ptr(tau), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                   workspace.numel(), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_bwd_ex")
    return dq, dk, dv, dc, grads


def entmax_attn_scores_debug(q, k, bh, causal, *, workspace=None, status=None, stream=None):
    """Raw tensor-core accumulators <q_i, k_j> of one (batch, head) pair as a float32 [N, N] tensor
    (NaN where the mask removes the entry)."""
    _same_layout(q, k)
    params = make_params(q, 1.5, causal)
    N = q.shape[2]
    out = torch.full((N, N), float("nan"), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = alloc_workspace(params, False, q.device)
    rc = load().entmax_attn_scores_debug(ctypes.byref(params), _ptr(q), _ptr(k), int(bh), _ptr(out), _ptr(workspace),
                                         workspace.numel(), _ptr(status), _stream_ptr(stream))
    _check(rc, "entmax_attn_scores_debug")
    return out


def entmax_attn_profile_events(which: int, start: Optional[torch.cuda.Event], stop: Optional[torch.cuda.Event]):
    """Record `start`/`stop` around the score-sweep kernel of later forward (which=0) or backward (which=1)
    calls of this thread; None, None switches the hook off.  The events must have been created with
    enable_timing=True and recorded once (so that their CUDA handles exist)."""
    a = None if start is None else ctypes.c_void_p(start.cuda_event)
    b = None if stop is None else ctypes.c_void_p(stop.cuda_event)
    _check(load().entmax_attn_profile_events(int(which), a, b), "entmax_attn_profile_events")


def read_support(params: Params, workspace: torch.Tensor, rows):
    """Support lists a forward call left in its workspace, for global row ids `rows`
    (row id = (b*heads + h)*seq + i).  Returns a list of (indices int64 tensor or None, y float32 tensor or None)."""
    lay = entmax_attn_workspace_layout(params)
    total = params.batch * params.heads * params.seq
    cnt = workspace[lay.row_count_offset: lay.row_count_offset + 4 * total].view(torch.int32)
    ent = workspace[lay.entries_offset: lay.entries_offset + 8 * total * lay.capacity].view(torch.int32)
    ent = ent.view(total, lay.capacity, 2)
    rows_t = torch.as_tensor(rows, dtype=torch.long, device=workspace.device)
    cnt_h = cnt[rows_t].cpu()
    ent_h = ent[rows_t].cpu()
    out = []
    for r in range(len(rows)):
        c = int(cnt_h[r])
        if c < 0:
            out.append((None, None))
        else:
            out.append((ent_h[r, :c, 1].to(torch.int64), ent_h[r, :c, 0].contiguous().view(torch.float32)))
    return out


def read_dense_support_sizes(params: Params, workspace: torch.Tensor, rows):
    """Support sizes of rows the dense path computed (row_count == -2), for global row ids `rows`: int64 tensor,
    -1 where the row kept a list instead (use read_support there)."""
    lay = entmax_attn_workspace_layout(params)
    total = params.batch * params.heads * params.seq
    cnt = workspace[lay.row_count_offset: lay.row_count_offset + 4 * total].view(torch.int32)
    dense = workspace[lay.dense_count_offset: lay.dense_count_offset + 8 * total].view(torch.int32).view(total, 2)
    rows_t = torch.as_tensor(rows, dtype=torch.long, device=workspace.device)
    size = dense[rows_t].sum(dim=1).to(torch.int64)
    return torch.where(cnt[rows_t] == -2, size, torch.full_like(size, -1)).cpu()


def entmax_attn_selftest_wait_expiry(limit_ns: int, status: torch.Tensor, stream=None):
    """Runs the bounded-wait self-test: one CTA waits `limit_ns` for a barrier nothing arrives on, then returns with
    FLAG_WAIT_EXPIRED in status[0] and the microseconds it waited in status[1]."""
    _check(load().entmax_attn_selftest_wait_expiry(int(limit_ns), _ptr(status), _stream_ptr(stream)),
           "entmax_attn_selftest_wait_expiry")


def _proj_params(x, heads, causal, n_mode, gamma_range):
    if x.dim() != 3 or not x.is_contiguous():
        raise EntmaxAttnError("x must be a contiguous [batch, seq, d_model] tensor")
    if x.dtype == torch.bfloat16:
        dt = DTYPE_BF16
    elif x.dtype == torch.float32:
        dt = DTYPE_FP32
    else:
        raise EntmaxAttnError("x must be bfloat16 or float32")
    B, N, dm = x.shape
    return ProjParams(B, int(heads), N, dm, dt, int(bool(causal)), int(n_mode), float(gamma_range))


def entmax_attn_scale_proj_fwd(x, w_beta, w_gamma, delta, gamma_range, causal, *, n_mode=0, c_rows=None, stream=None):
    """c_rows [B, H, N] (float32) from the layer input x [B, N, d_model] and per-head weights [H, d_model]."""
    H = w_beta.shape[0]
    params = _proj_params(x, H, causal, n_mode, gamma_range)
    if c_rows is None:
        c_rows = torch.empty((x.shape[0], H, x.shape[1]), dtype=torch.float32, device=x.device)
    _check(load().entmax_attn_scale_proj_fwd(ctypes.byref(params), _ptr(x), _ptr(w_beta), _ptr(w_gamma), _ptr(delta),
                                             _ptr(c_rows), _stream_ptr(stream)), "entmax_attn_scale_proj_fwd")
    return c_rows


def entmax_attn_scale_proj_bwd(x, w_beta, w_gamma, d_scale_rows, gamma_range, causal, *, n_mode=0, want_dx=True,
                               stream=None):
    """Chain rule of the projection.  Returns (dw_beta, dw_gamma, ddelta, dx or None)."""
    H = w_beta.shape[0]
    params = _proj_params(x, H, causal, n_mode, gamma_range)
    dwb, dwg = torch.empty_like(w_beta), torch.empty_like(w_gamma)
    dd = torch.empty((H,), dtype=torch.float32, device=x.device)
    dx = torch.empty_like(x) if want_dx else None
    _check(load().entmax_attn_scale_proj_bwd(ctypes.byref(params), _ptr(x), _ptr(w_beta), _ptr(w_gamma), _ptr(d_scale_rows),
                                             _ptr(dwb), _ptr(dwg), _ptr(dd), _ptr(dx), _stream_ptr(stream)),
           "entmax_attn_scale_proj_bwd")
    return dwb, dwg, dd, dx
