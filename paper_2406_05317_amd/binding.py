"""Thin ctypes binding of liblococo.so (the C ABI in include/lococo.h).

Argument marshalling only: torch tensors supply device memory and the current
HIP stream; every step of the path runs inside the library's kernels.  There
is no fallback: if the shared library is missing, importing this module's
functions raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblococo.so")

LOCOCO_OK, LOCOCO_EINVAL, LOCOCO_EUNSUPPORTED, LOCOCO_ESTATE, LOCOCO_EHIP, LOCOCO_EWORKSPACE = range(6)
LOCOCO_F32, LOCOCO_BF16 = 0, 1
LOCOCO_IMPL_AUTO, LOCOCO_IMPL_GENERIC, LOCOCO_IMPL_MFMA = 0, 1, 2
LOCOCO_FLAG_FILTERS_PREPARED = 1
LOCOCO_PAIRS_HALVES, LOCOCO_PAIRS_ADJACENT = 0, 1
(LOCOCO_OPT_RESET, LOCOCO_OPT_SPIN_LIMIT, LOCOCO_OPT_SCAN_PER_STEP, LOCOCO_OPT_CHAIN_SYNC_DEVICE,
 LOCOCO_OPT_LOGITS_TILES, LOCOCO_OPT_MAX_RESIDENT, LOCOCO_OPT_UNFUSED_KV, LOCOCO_OPT_NO_STEP_PIPELINE) = range(8)

EXPORTS = ["lococo_plan", "lococo_workspace_bytes", "lococo_attn_only", "lococo_segment_step",
           "lococo_sequence_forward", "lococo_mix_from_logits", "lococo_last_error",
           "lococo_version", "lococo_timing_begin", "lococo_timing_end", "lococo_scan_status",
           "lococo_prepare_filters", "lococo_backward_workspace_bytes", "lococo_segment_step_backward",
           "lococo_measure_peaks", "lococo_debug_option", "lococo_describe_path",
           "lococo_segment_step_noalloc", "lococo_sequence_backward_workspace_bytes",
           "lococo_sequence_backward",
           "lococo_pages_plan", "lococo_pages_store", "lococo_pages_load", "lococo_pages_workspace_bytes",
           "lococo_pages_attn",
           "lococo_rows_rotate", "lococo_rows_rotate_backward_workspace_bytes", "lococo_rows_rotate_backward", "lococo_pages_append",
           "lococo_pages_tree", "lococo_pages_attn_tree_workspace_bytes", "lococo_pages_attn_tree", "lococo_pages_keep", "lococo_pages_move"]


class lococo_config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("M", C.c_int32), ("conv_width", C.c_int32), ("conv_in", C.c_int32),
                ("norm", C.c_int32), ("impl", C.c_int32), ("flags", C.c_int32),
                ("w_head_stride", C.c_int64), ("b_head_stride", C.c_int64),
                ("attn_scale", C.c_float), ("norm_eps", C.c_float)]


class lococo_cache(C.Structure):
    _fields_ = [("k", C.c_void_p * 2), ("v", C.c_void_p * 2), ("cur", C.c_int32),
                ("len", C.c_int32), ("protect", C.c_void_p), ("protect_chain_stride", C.c_int64),
                ("attn_colsum", C.c_void_p)]


class lococo_tensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64),
                ("stride_t", C.c_int64)]


class lococo_qkvo(C.Structure):
    _fields_ = [("q", lococo_tensor), ("k", lococo_tensor), ("v", lococo_tensor),
                ("o", lococo_tensor)]


class lococo_seg(C.Structure):
    _fields_ = [("start", C.c_int64), ("len", C.c_int32), ("branch", C.c_int32),
                ("len_before", C.c_int32), ("len_after", C.c_int32), ("buf_after", C.c_int32),
                ("reserved", C.c_int32)]


class lococo_kernel_time(C.Structure):
    _fields_ = [("name", C.c_char_p), ("launches", C.c_int64), ("total_ms", C.c_double)]


class lococo_path_info(C.Structure):
    _fields_ = [("path", C.c_int32), ("compute_units", C.c_int32), ("tile_slots", C.c_int32),
                ("scan_groups", C.c_int32), ("scan_resident_limit", C.c_int32), ("position_split", C.c_int32),
                ("step_pipeline", C.c_int32), ("reserved", C.c_int32)]


class lococo_pages(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_rows", C.c_int32), ("n_pages", C.c_int32), ("attn_scale", C.c_float),
                ("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p)]


class lococo_requests(C.Structure):
    _fields_ = [("n", C.c_int32), ("tokens", C.c_int32), ("table_pages", C.c_int32), ("max_new", C.c_int32),
                ("max_held", C.c_int32), ("tables", C.c_void_p), ("starts", C.c_void_p), ("held", C.c_void_p)]


class lococo_rotation(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("pairing", C.c_int32), ("norm", C.c_int32),
                ("norm_eps", C.c_float), ("freqs", C.c_void_p), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p),
                ("q_weight_stride", C.c_int64), ("k_weight_stride", C.c_int64)]


class LococoError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"lococo status {status}: {message}")
        self.status = status


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2406_05317_amd.build` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        cfgp, qp, cap = C.POINTER(lococo_config), C.POINTER(lococo_qkvo), C.POINTER(lococo_cache)
        L.lococo_plan.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                  C.POINTER(lococo_seg), C.POINTER(C.c_int64)]
        L.lococo_workspace_bytes.argtypes = [cfgp, C.c_int64, C.c_int32, C.c_int32,
                                             C.POINTER(C.c_size_t)]
        L.lococo_attn_only.argtypes = [cfgp, qp, C.c_int32, cap, C.c_void_p]
        L.lococo_segment_step.argtypes = [cfgp, qp, C.c_int32, C.c_void_p, C.c_void_p, cap,
                                          C.c_void_p, C.c_size_t, C.c_void_p]
        L.lococo_segment_step_noalloc.argtypes = [cfgp, qp, C.c_int32, C.c_void_p, C.c_void_p, cap, C.c_void_p]
        L.lococo_sequence_forward.argtypes = [cfgp, qp, C.c_int64, C.c_int32, C.c_void_p,
                                              C.c_void_p, cap, C.c_void_p, C.c_size_t, C.c_void_p]
        L.lococo_mix_from_logits.argtypes = [cfgp, qp, C.c_int32, C.c_void_p, cap, C.c_void_p]
        L.lococo_scan_status.argtypes = [cfgp, C.c_void_p, C.POINTER(C.c_int32)]
        L.lococo_prepare_filters.argtypes = [cfgp, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        fp = C.c_void_p
        L.lococo_backward_workspace_bytes.argtypes = [cfgp, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.lococo_segment_step_backward.argtypes = [cfgp, qp, C.c_int32, C.c_void_p, C.c_void_p, cap] + [fp] * 10 + [
            C.c_void_p, C.c_size_t, C.c_void_p]
        L.lococo_sequence_backward_workspace_bytes.argtypes = [cfgp, C.c_int64, C.c_int32, C.POINTER(C.c_size_t)]
        L.lococo_sequence_backward.argtypes = [cfgp, qp, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, cap] + [
            fp] * 10 + [C.c_void_p, C.c_size_t, C.c_void_p]
        L.lococo_measure_peaks.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_double),
                                           C.POINTER(C.c_double)]
        L.lococo_debug_option.argtypes = [C.c_int32, C.c_int64]
        L.lococo_describe_path.argtypes = [cfgp, C.c_int32, C.POINTER(lococo_path_info)]
        pgp, rqp, tp, i32 = C.POINTER(lococo_pages), C.POINTER(lococo_requests), C.POINTER(lococo_tensor), C.c_int32
        L.lococo_pages_plan.argtypes = [pgp, i32, i32, i32] + [C.c_void_p] * 12
        L.lococo_pages_store.argtypes = [pgp, tp, tp, i32, i32, C.c_void_p, C.c_void_p]
        L.lococo_pages_load.argtypes = [pgp, C.c_void_p, i32, i32, tp, tp, C.c_void_p]
        L.lococo_pages_workspace_bytes.argtypes = [pgp, rqp, C.POINTER(C.c_size_t)]
        L.lococo_pages_attn.argtypes = [pgp, rqp, tp, tp, i32, C.c_void_p, C.c_size_t, C.c_void_p]
        rtp, vp = C.POINTER(lococo_rotation), C.c_void_p
        L.lococo_rows_rotate.argtypes = [rtp, tp, tp, tp, tp, i32, i32, vp, vp]
        L.lococo_rows_rotate_backward_workspace_bytes.argtypes = [rtp, i32, C.POINTER(C.c_size_t)]
        L.lococo_rows_rotate_backward.argtypes = [rtp, tp, tp, i32, i32] + [vp] * 8 + [C.c_size_t, vp]
        L.lococo_pages_append.argtypes = [pgp, rtp, tp, tp, tp, tp, i32, i32, vp, vp, vp]
        L.lococo_pages_tree.argtypes = [i32, i32, vp, vp, vp, vp, i32, vp, vp, vp]
        L.lococo_pages_attn_tree_workspace_bytes.argtypes = [pgp, rqp, C.POINTER(C.c_size_t)]
        L.lococo_pages_attn_tree.argtypes = [pgp, rqp, tp, tp, i32, vp, i32, vp, C.c_size_t, vp]
        L.lococo_pages_keep.argtypes = [pgp, i32, i32, i32] + [vp] * 13
        L.lococo_pages_move.argtypes = [pgp, i32, i32] + [vp] * 4
        L.lococo_timing_begin.argtypes = []
        L.lococo_timing_end.argtypes = [C.POINTER(lococo_kernel_time), C.POINTER(C.c_int32)]
        for n in EXPORTS[:6] + EXPORTS[8:]:
            getattr(L, n).restype = C.c_int
        L.lococo_last_error.restype = C.c_char_p
        L.lococo_version.restype = C.c_char_p
        _lib = L
    return _lib


def _check(status: int):
    if status != LOCOCO_OK:
        raise LococoError(status, lib().lococo_last_error().decode())


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return LOCOCO_F32
    if dt == torch.bfloat16:
        return LOCOCO_BF16
    raise TypeError(f"unsupported storage dtype {dt}")


def make_config(*, dtype: torch.dtype, batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                M: int, conv_width: int, conv_in: int = 0, norm: int = 0, impl: int = 0,
                w_head_stride: int = 0, b_head_stride: int = 0, attn_scale: float = 0.0,
                norm_eps: float = 0.0, flags: int = 0) -> lococo_config:
    return lococo_config(C.sizeof(lococo_config), _dtype_code(dtype), batch, n_q_heads, n_kv_heads,
                         head_dim, M, conv_width, conv_in, norm, impl, flags, w_head_stride,
                         b_head_stride, attn_scale, norm_eps)


def _tensor(t: torch.Tensor | None) -> lococo_tensor:
    """View of a [b, h, tokens, d] torch tensor (d contiguous)."""
    if t is None:
        return lococo_tensor(None, 0, 0, 0)
    assert t.dim() == 4 and t.stride(3) == 1, "expected [b, h, t, d] with d contiguous"
    return lococo_tensor(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def _qkvo(q, k, v, o) -> lococo_qkvo:
    return lococo_qkvo(_tensor(q), _tensor(k), _tensor(v), _tensor(o))


def _ptr(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class Cache:
    """Device buffers of the double-buffered KV cache plus the host-side state."""

    def __init__(self, cfg: lococo_config, device="cuda", dtype: torch.dtype | None = None):
        dt = dtype or (torch.float32 if cfg.dtype == LOCOCO_F32 else torch.bfloat16)
        shape = (cfg.batch, cfg.n_kv_heads, cfg.M, cfg.head_dim)
        self.kbuf = [torch.zeros(shape, dtype=dt, device=device) for _ in range(2)]
        self.vbuf = [torch.zeros(shape, dtype=dt, device=device) for _ in range(2)]
        self.c = lococo_cache((C.c_void_p * 2)(self.kbuf[0].data_ptr(), self.kbuf[1].data_ptr()),
                              (C.c_void_p * 2)(self.vbuf[0].data_ptr(), self.vbuf[1].data_ptr()),
                              0, 0, None, 0, None)
        self.M, self.device = cfg.M, device
        self._protect = None
        self.attn_colsum = None
        self._chains = (cfg.batch, cfg.n_kv_heads, cfg.M)

    @property
    def len(self) -> int:
        return self.c.len

    @property
    def cur(self) -> int:
        return self.c.cur

    @property
    def k(self) -> torch.Tensor:
        return self.kbuf[self.c.cur]

    @property
    def v(self) -> torch.Tensor:
        return self.vbuf[self.c.cur]

    def set_protect(self, mask):
        """mask: None, or a bool array/tensor [M] (one mask for every chain) or [batch, n_kv_heads, M]:
        True = the slot is protected (see lococo_cache.protect in lococo.h)."""
        if mask is None:
            self._protect, self.c.protect, self.c.protect_chain_stride = None, None, 0
            return
        m = torch.as_tensor(mask).to(torch.bool).cpu()
        words = (self.M + 31) // 32
        flat = m.reshape(-1, self.M)
        bits = torch.zeros(flat.shape[0], words * 32, dtype=torch.int64)
        bits[:, :self.M] = flat.to(torch.int64)
        w = (bits.reshape(flat.shape[0], words, 32) << torch.arange(32, dtype=torch.int64)).sum(-1)
        w = torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)
        self._protect = w.to(self.device).contiguous()
        self.c.protect = self._protect.data_ptr()
        self.c.protect_chain_stride = 0 if m.dim() == 1 else words

    def track_attention(self, on: bool = True):
        """Allocate (zeroed) or drop the fp32 [batch, n_kv_heads, M] accumulator of attention scores
        per cache slot (see lococo_cache.attn_colsum in lococo.h); read it as `self.attn_colsum`."""
        self.attn_colsum = torch.zeros(self._chains, dtype=torch.float32, device=self.device) if on else None
        self.c.attn_colsum = _ptr(self.attn_colsum)

    def load(self, k: torch.Tensor, v: torch.Tensor, length: int):
        self.kbuf[self.c.cur].copy_(k)
        self.vbuf[self.c.cur].copy_(v)
        self.c.len = length


class Pages:
    """Device arrays of paged 4-bit rows and their description (lococo_pages in lococo.h): `n_pages` pages of `page_rows` rows
    of every kv head.  Nobody owns a page at first: see fresh_ring."""

    def __init__(self, *, dtype: torch.dtype, n_q_heads: int, n_kv_heads: int, head_dim: int, page_rows: int, n_pages: int,
                 attn_scale: float = 0.0, device="cuda"):
        codes, scales = (n_pages, n_kv_heads, page_rows, head_dim // 2), (n_pages, n_kv_heads, head_dim // 32, page_rows)
        self.k_codes, self.v_codes = (torch.zeros(codes, dtype=torch.uint8, device=device) for _ in range(2))
        self.k_scales, self.v_scales = (torch.zeros(scales, dtype=torch.uint8, device=device) for _ in range(2))
        self.c = lococo_pages(C.sizeof(lococo_pages), _dtype_code(dtype), n_q_heads, n_kv_heads, head_dim, page_rows, n_pages,
                              attn_scale, self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(),
                              self.v_scales.data_ptr())
        self.ref, self.dtype, self.device = C.byref(self.c), dtype, device

    def fresh_ring(self):
        """(ring, ends) with every page free, as lococo_pages_plan takes them."""
        return (torch.arange(self.c.n_pages, dtype=torch.int32, device=self.device),
                torch.tensor([0, self.c.n_pages], dtype=torch.int64, device=self.device))


class Rotation:
    """Norm and position rotation of a layer's query and key rows (lococo_rotation in lococo.h): `freqs` fp32 [rotary_dim / 2] in radians
    a position (None: no rotation), weights [head_dim] for all heads or [heads, head_dim], of the rows' type."""

    def __init__(self, *, dtype: torch.dtype, n_q_heads: int, n_kv_heads: int, head_dim: int, freqs: torch.Tensor | None = None,
                 adjacent: bool = False, norm: bool = False, norm_eps: float = 0.0, q_weight: torch.Tensor | None = None,
                 k_weight: torch.Tensor | None = None):
        self.dtype, self.freqs, self.weights = dtype, freqs, (q_weight, k_weight)
        if freqs is not None and (freqs.dtype is not torch.float32 or not freqs.is_cuda or not freqs.is_contiguous() or freqs.dim() != 1):
            raise TypeError(f"expected frequencies [rotary_dim / 2] in fp32 on the device, got {tuple(freqs.shape)} of {freqs.dtype}, {freqs.device}")
        strides = []
        for w, heads in ((q_weight, n_q_heads), (k_weight, n_kv_heads)):
            if w is not None and (w.dtype is not dtype or not w.is_cuda or not w.is_contiguous() or
                                  tuple(w.shape) not in ((head_dim,), (heads, head_dim))):
                raise TypeError(f"expected contiguous weights [{head_dim}] or [{heads}, {head_dim}] of {dtype} on the device, got "
                                f"{tuple(w.shape)} of {w.dtype}, {w.device}")
            strides.append(head_dim if w is not None and w.dim() == 2 else 0)
        self.device = next((t.device.index for t in (freqs, q_weight, k_weight) if t is not None), None)
        if any(t is not None and t.device.index != self.device for t in (freqs, q_weight, k_weight)):
            raise TypeError("frequencies and weights are on different devices")
        self.c = lococo_rotation(C.sizeof(lococo_rotation), _dtype_code(dtype), n_q_heads, n_kv_heads, head_dim,
                                 0 if freqs is None else 2 * freqs.numel(), LOCOCO_PAIRS_ADJACENT if adjacent else LOCOCO_PAIRS_HALVES,
                                 int(norm), norm_eps, _ptr(freqs), _ptr(q_weight), _ptr(k_weight), *strides)
        self.ref = C.byref(self.c)
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim


def lococo_version() -> str:
    return lib().lococo_version().decode()


def lococo_plan(L: int, B: int, M: int, len0: int = 0, cur0: int = 0):
    """List of (start, len, branch, len_before, len_after, buf_after) tuples."""
    n = C.c_int64(0)
    _check(lib().lococo_plan(L, B, M, len0, cur0, None, C.byref(n)))
    rows = (lococo_seg * max(n.value, 1))()
    cap = C.c_int64(n.value)
    _check(lib().lococo_plan(L, B, M, len0, cur0, rows, C.byref(cap)))
    return [(r.start, r.len, r.branch, r.len_before, r.len_after, r.buf_after)
            for r in rows[:n.value]]


def lococo_workspace_bytes(cfg: lococo_config, L: int, B: int, history: bool = False) -> int:
    out = C.c_size_t(0)
    _check(lib().lococo_workspace_bytes(C.byref(cfg), L, B, int(history), C.byref(out)))
    return out.value


def lococo_attn_only(cfg, q, k, v, o, cache: Cache):
    B = q.shape[2]
    x = _qkvo(q, k, v, o)
    _check(lib().lococo_attn_only(C.byref(cfg), C.byref(x), B, C.byref(cache.c), _stream()))


def lococo_segment_step(cfg, q, k, v, o, conv_w, conv_b, cache: Cache, workspace=None):
    B = q.shape[2]
    x = _qkvo(q, k, v, o)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().lococo_segment_step(C.byref(cfg), C.byref(x), B, _ptr(conv_w), _ptr(conv_b),
                                     C.byref(cache.c), _ptr(workspace), ws_bytes, _stream()))


def lococo_segment_step_noalloc(cfg, q, k, v, o, conv_w, conv_b, cache: Cache):
    """lococo_segment_step on the library's own scratch array (allocates nothing)."""
    B = q.shape[2]
    x = _qkvo(q, k, v, o)
    _check(lib().lococo_segment_step_noalloc(C.byref(cfg), C.byref(x), B, _ptr(conv_w), _ptr(conv_b),
                                             C.byref(cache.c), _stream()))


def lococo_sequence_forward(cfg, q, k, v, o, conv_w, conv_b, cache: Cache, B: int, workspace=None):
    L = q.shape[2]
    x = _qkvo(q, k, v, o)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().lococo_sequence_forward(C.byref(cfg), C.byref(x), L, B, _ptr(conv_w),
                                         _ptr(conv_b), C.byref(cache.c), _ptr(workspace), ws_bytes,
                                         _stream()))


def lococo_mix_from_logits(cfg, k, v, logits, cache: Cache):
    B = k.shape[2]
    assert logits.dtype == torch.float32 and logits.is_contiguous()
    x = _qkvo(None, k, v, None)
    _check(lib().lococo_mix_from_logits(C.byref(cfg), C.byref(x), B, logits.data_ptr(),
                                        C.byref(cache.c), _stream()))


def lococo_prepare_filters(cfg, conv_w, workspace):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().lococo_prepare_filters(C.byref(cfg), _ptr(conv_w), _ptr(workspace), ws_bytes, _stream()))


def lococo_backward_workspace_bytes(cfg, B: int, length: int) -> int:
    out = C.c_size_t(0)
    _check(lib().lococo_backward_workspace_bytes(C.byref(cfg), B, length, C.byref(out)))
    return out.value


def lococo_segment_step_backward(cfg, q, k, v, conv_w, conv_b, cache: Cache, d_o, d_new_k, d_new_v, d_q, d_k,
                                 d_v, d_cache_k, d_cache_v, d_conv_w, d_conv_b, workspace):
    """Gradients of one block step; `cache` is the state BEFORE the step.  All gradient tensors are
    fp32, contiguous, on the device; d_conv_w / d_conv_b are added to."""
    for t in (d_o, d_new_k, d_new_v, d_q, d_k, d_v, d_cache_k, d_cache_v, d_conv_w, d_conv_b):
        assert t is None or (t.dtype == torch.float32 and t.is_contiguous() and t.is_cuda)
    B = q.shape[2]
    x = _qkvo(q, k, v, None)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().lococo_segment_step_backward(
        C.byref(cfg), C.byref(x), B, _ptr(conv_w), _ptr(conv_b), C.byref(cache.c), _ptr(d_o), _ptr(d_new_k),
        _ptr(d_new_v), _ptr(d_q), _ptr(d_k), _ptr(d_v), _ptr(d_cache_k), _ptr(d_cache_v), _ptr(d_conv_w),
        _ptr(d_conv_b), _ptr(workspace), ws_bytes, _stream()))


def lococo_sequence_backward_workspace_bytes(cfg, L: int, B: int) -> int:
    out = C.c_size_t(0)
    _check(lib().lococo_sequence_backward_workspace_bytes(C.byref(cfg), L, B, C.byref(out)))
    return out.value


def lococo_sequence_backward(cfg, q, k, v, B: int, conv_w, conv_b, cache: Cache, d_o, d_final_k, d_final_v, d_q,
                             d_k, d_v, d_cache0_k, d_cache0_v, d_conv_w, d_conv_b, workspace):
    """Gradients of a whole scan started from `cache` (left as it is).  All gradient tensors are fp32,
    contiguous, on the device; d_final_k / d_final_v may be None (zero); d_conv_w / d_conv_b are added to."""
    for t in (d_o, d_final_k, d_final_v, d_q, d_k, d_v, d_cache0_k, d_cache0_v, d_conv_w, d_conv_b):
        assert t is None or (t.dtype == torch.float32 and t.is_contiguous() and t.is_cuda)
    L = q.shape[2]
    x = _qkvo(q, k, v, None)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().lococo_sequence_backward(
        C.byref(cfg), C.byref(x), L, B, _ptr(conv_w), _ptr(conv_b), C.byref(cache.c), _ptr(d_o), _ptr(d_final_k),
        _ptr(d_final_v), _ptr(d_q), _ptr(d_k), _ptr(d_v), _ptr(d_cache0_k), _ptr(d_cache0_v), _ptr(d_conv_w),
        _ptr(d_conv_b), _ptr(workspace), ws_bytes, _stream()))


# The calls on pages are short enough for the marshalling to count: their checks and addresses are taken in one go.
_I32, _I64 = torch.int32, torch.int64


def _numbers(dtype, *arrays):
    """Addresses of contiguous device arrays of whole numbers."""
    for t in arrays:
        if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
            raise TypeError(f"expected a contiguous {dtype} array on the device, got {t.dtype}, {t.device}, strides {t.stride()}")
    return [t.data_ptr() for t in arrays]


def _rows(pages: Pages, t: torch.Tensor, heads: int) -> lococo_tensor:
    """View of a [b, heads, t, d] tensor of the pages' type."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not pages.dtype or not t.is_cuda or len(shape) != 4 or shape[1] != heads or shape[3] != pages.c.head_dim or stride[3] != 1:
        raise TypeError(f"expected [b, {heads}, t, {pages.c.head_dim}] of {pages.dtype} on the device with the last axis contiguous, got "
                        f"{tuple(shape)} of {t.dtype}, {t.device}, strides {stride}")
    return lococo_tensor(t.data_ptr(), stride[0], stride[1], stride[2])


def _stream_now() -> int:
    """The current device's current stream: as _stream(), without an object for it."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def lococo_pages_plan(pages: Pages, new_rows, held, tables, ring, ends, held_after, ends_after, starts, slots, positions, totals):
    """Pages, slots and positions of a turn from its requests' lengths (all arrays on the device: int32, ends int64)."""
    new_p, held_p, tables_p, ring_p, after_p, starts_p, slots_p, positions_p, totals_p = _numbers(
        _I32, new_rows, held, tables, ring, held_after, starts, slots, positions, totals)
    ends_p, ends_after_p = _numbers(_I64, ends, ends_after)
    n, width = tables.shape
    tokens = slots.numel()
    if not (new_rows.numel() == held.numel() == held_after.numel() == starts.numel() - 1 == n and positions.numel() == tokens and
            ring.numel() == pages.c.n_pages and ends.numel() == ends_after.numel() == 2 and totals.numel() == 4):
        raise ValueError("arrays of the plan do not fit each other")
    _check(lib().lococo_pages_plan(pages.ref, n, tokens, width, new_p, held_p, tables_p, ring_p, ends_p, after_p, ends_after_p, starts_p,
                                   slots_p, positions_p, totals_p, _stream_now()))


def _slots_of(slots, k, v):
    if k.shape != v.shape or slots.numel() != k.shape[0] * k.shape[2]:
        raise ValueError(f"{slots.numel()} slots for k, v of {tuple(k.shape)}, {tuple(v.shape)}")
    return _numbers(_I32, slots)[0]


def lococo_pages_store(pages: Pages, k, v, slots):
    """k, v [b, n_kv_heads, t, d] to 4 bits, row (b, t) at slots[b * T + t]."""
    x, y = _rows(pages, k, pages.c.n_kv_heads), _rows(pages, v, pages.c.n_kv_heads)
    at = _slots_of(slots, k, v)
    _check(lib().lococo_pages_store(pages.ref, C.byref(x), C.byref(y), max(k.shape[2], 1), slots.numel(), at, _stream_now()))


def lococo_pages_load(pages: Pages, slots, k, v):
    """The rows at `slots` into k, v [b, n_kv_heads, t, d]."""
    x, y = _rows(pages, k, pages.c.n_kv_heads), _rows(pages, v, pages.c.n_kv_heads)
    at = _slots_of(slots, k, v)
    _check(lib().lococo_pages_load(pages.ref, at, max(k.shape[2], 1), slots.numel(), C.byref(x), C.byref(y), _stream_now()))


def lococo_pages_workspace_bytes(pages: Pages, n: int, tokens: int, max_new: int, max_held: int, table_pages: int = 1) -> int:
    r, out = lococo_requests(n, tokens, table_pages, max_new, max_held, None, None, None), C.c_size_t(0)
    _check(lib().lococo_pages_workspace_bytes(pages.ref, C.byref(r), C.byref(out)))
    return out.value


def lococo_pages_attn(pages: Pages, q, o, tables, starts, held, max_new: int, max_held: int, workspace=None):
    """Attention of the requests' new rows q [b, n_q_heads, t, d] over all rows of their request, into o."""
    x, y = _rows(pages, q, pages.c.n_q_heads), _rows(pages, o, pages.c.n_q_heads)
    n, width = tables.shape
    b, _, t, _ = q.shape
    if q.shape != o.shape or starts.numel() != n + 1 or held.numel() != n:
        raise ValueError("o, starts or held do not fit q and the tables")
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError(f"expected a contiguous workspace on the device, got {workspace.device}, strides {workspace.stride()}")
    r = lococo_requests(n, b * t, width, max_new, max_held, *_numbers(_I32, tables, starts, held))
    ws, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check(lib().lococo_pages_attn(pages.ref, C.byref(r), C.byref(x), C.byref(y), max(t, 1), ws, ws_bytes, _stream_now()))


# The calls below also see to it that what they are given is on the current device, whose current stream they run on.
def _here(*tensors):
    """Device arrays on the current device; returns their addresses (None for None)."""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise TypeError(f"expected arrays on the current device, {dev}, got one on {t.device}")
    return [None if t is None else t.data_ptr() for t in tensors]


def _whole(dtype, *arrays):
    """Addresses of contiguous arrays of whole numbers on the current device (None for None)."""
    for t in arrays:
        if t is not None and (t.dtype is not dtype or not t.is_contiguous()):
            raise TypeError(f"expected a contiguous {dtype} array on the device, got {t.dtype}, {t.device}, strides {t.stride()}")
    return _here(*arrays)


def _rotated(rot: Rotation, t: torch.Tensor, heads: int, dev: int) -> lococo_tensor:
    """View of a [b, heads, t, d] tensor of the rotation's type on the current device, `dev`."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not rot.dtype or len(shape) != 4 or shape[1] != heads or shape[3] != rot.head_dim or stride[3] != 1 or t.get_device() != dev:
        raise TypeError(f"expected [b, {heads}, t, {rot.head_dim}] of {rot.dtype} on the current device, {dev}, with the last axis contiguous, got "
                        f"{tuple(shape)} of {t.dtype}, {t.device}, strides {stride}")
    return lococo_tensor(t.data_ptr(), stride[0], stride[1], stride[2])


def _rotation_here(rot: Rotation) -> int:
    """The current device, which the rotation's arrays have to be on (-2 where there is none: no array is there)."""
    try:
        dev = torch._C._cuda_getDevice()
    except RuntimeError:
        dev = -2
    if rot.device is not None and rot.device != dev:
        raise TypeError(f"the rotation's frequencies and weights are on device {rot.device}, not on the current one, {dev}")
    return dev


def _rotated_pair(rot: Rotation, q, k, dev: int):
    """(views of q and k, batch entries, rows of one)"""
    if q is None:
        if k is None:
            raise ValueError("neither q nor k is given")
        return None, _rotated(rot, k, rot.n_kv_heads, dev), k.shape[0], k.shape[2]
    x = _rotated(rot, q, rot.n_q_heads, dev)
    b, _, t, _ = q.shape
    if k is None:
        return x, None, b, t
    if k.shape[0] != b or k.shape[2] != t:
        raise ValueError(f"q and k of {tuple(q.shape)} and {tuple(k.shape)} are not of the same tokens")
    return x, _rotated(rot, k, rot.n_kv_heads, dev), b, t


def _positions_of(positions, tokens):
    if positions is None:
        return None
    if positions.numel() != tokens:
        raise ValueError(f"{positions.numel()} positions for {tokens} rows")
    return _whole(_I32, positions)[0]


def lococo_rows_rotate(rot: Rotation, q, k, q_out, k_out, positions=None):
    """q, k [b, heads, t, d] normed and turned by their rows' positions (None: 0 .. t - 1) into q_out, k_out; either may be None."""
    dev = _rotation_here(rot)
    x, y, b, t = _rotated_pair(rot, q, k, dev)
    xo, yo, bo, to = _rotated_pair(rot, q_out, k_out, dev)
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (b, t) != (bo, to):
        raise ValueError("q_out, k_out do not fit q, k")
    _check(lib().lococo_rows_rotate(rot.ref, x, y, xo, yo, max(t, 1), b * t, _positions_of(positions, b * t), _stream_now()))


def lococo_rows_rotate_backward_workspace_bytes(rot: Rotation, tokens: int) -> int:
    out = C.c_size_t(0)
    _check(lib().lococo_rows_rotate_backward_workspace_bytes(rot.ref, tokens, C.byref(out)))
    return out.value


def lococo_rows_rotate_backward(rot: Rotation, q, k, positions, d_q_out, d_k_out, d_q, d_k, d_q_weight=None, d_k_weight=None, workspace=None):
    """Gradients of lococo_rows_rotate: fp32, contiguous; d_q, d_k overwritten (they may be d_q_out, d_k_out), the weights' added to."""
    x, y, b, t = _rotated_pair(rot, q, k, _rotation_here(rot))
    for rows, grads in ((q, (d_q_out, d_q)), (k, (d_k_out, d_k))):
        for g in grads:
            if (g is None) != (rows is None) or (g is not None and (g.dtype is not torch.float32 or not g.is_contiguous() or g.shape != rows.shape)):
                raise TypeError("expected contiguous fp32 gradients of the shapes of q and k")
    for w, g in zip(rot.weights, (d_q_weight, d_k_weight)):
        if g is not None and (w is None or g.dtype is not torch.float32 or not g.is_contiguous() or g.shape != w.shape):
            raise TypeError("expected contiguous fp32 gradients of the shapes of the weights")
    if workspace is not None and not workspace.is_contiguous():
        raise TypeError(f"expected a contiguous workspace, got strides {workspace.stride()}")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    *grads, ws = _here(d_q_out, d_k_out, d_q, d_k, d_q_weight, d_k_weight, workspace)
    _check(lib().lococo_rows_rotate_backward(rot.ref, x, y, max(t, 1), b * t, _positions_of(positions, b * t), *grads, ws, ws_bytes, _stream_now()))


def lococo_pages_append(pages: Pages, rot: Rotation, q, k, v, q_out, slots, positions):
    """New rows as a projection leaves them: q [b, n_q_heads, t, d] normed and turned into q_out, k so and v as it is to 4 bits at `slots`."""
    _rotation_here(rot)
    Hq, Hkv = pages.c.n_q_heads, pages.c.n_kv_heads
    views = [C.byref(_rows(pages, x, h)) for x, h in ((q, Hq), (k, Hkv), (v, Hkv), (q_out, Hq))]
    b, _, t, _ = q.shape
    if q_out.shape != q.shape or k.shape != v.shape or k.shape[0] != b or k.shape[2] != t or slots.numel() != b * t:
        raise ValueError("q, k, v, q_out or slots do not fit each other")
    _here(pages.k_codes, q, k, v, q_out)
    _check(lib().lococo_pages_append(pages.ref, rot.ref, *views, max(t, 1), b * t, _whole(_I32, slots)[0], _positions_of(positions, b * t),
                                     _stream_now()))


def lococo_pages_tree(starts, held, parents, masks, positions, bases=None):
    """masks [tokens, words] (int32, words of bits) and positions [tokens] of the requests' trees from their rows' parents [tokens]."""
    n = held.numel()
    if starts.numel() != n + 1 or (bases is not None and bases.numel() != n):
        raise ValueError("starts or bases do not fit held")
    if masks.dim() != 2 or not masks.shape[0] == parents.numel() == positions.numel():
        raise ValueError("masks, parents and positions do not fit each other")
    s, h, b, p, m, x = _whole(_I32, starts, held, bases, parents, masks, positions)
    _check(lib().lococo_pages_tree(n, parents.numel(), s, h, b, p, masks.shape[1], m, x, _stream_now()))


def lococo_pages_attn_tree_workspace_bytes(pages: Pages, n: int, tokens: int, max_new: int, max_held: int, table_pages: int = 1) -> int:
    r, out = lococo_requests(n, tokens, table_pages, max_new, max_held, None, None, None), C.c_size_t(0)
    _check(lib().lococo_pages_attn_tree_workspace_bytes(pages.ref, C.byref(r), C.byref(out)))
    return out.value


def lococo_pages_attn_tree(pages: Pages, q, o, tables, starts, held, masks, max_new: int, max_held: int, workspace=None):
    """lococo_pages_attn with the new rows that a row sees named by its mask, masks [tokens, words] (int32, words of bits)."""
    x, y = _rows(pages, q, pages.c.n_q_heads), _rows(pages, o, pages.c.n_q_heads)
    n, width = tables.shape
    b, _, t, _ = q.shape
    if q.shape != o.shape or starts.numel() != n + 1 or held.numel() != n or masks.dim() != 2 or masks.shape[0] != b * t:
        raise ValueError("o, starts, held or masks do not fit q and the tables")
    if workspace is not None and not workspace.is_contiguous():
        raise TypeError(f"expected a contiguous workspace on the device, got {workspace.device}, strides {workspace.stride()}")
    ws = _here(workspace, pages.k_codes, q, o)[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    *numbers, m = _whole(_I32, tables, starts, held, masks)
    r = lococo_requests(n, b * t, width, max_new, max_held, *numbers)
    _check(lib().lococo_pages_attn_tree(pages.ref, C.byref(r), C.byref(x), C.byref(y), max(t, 1), m, masks.shape[1], ws, ws_bytes, _stream_now()))


def lococo_pages_keep(pages: Pages, tables, starts, held, slots, kept, ring, ends, held_after, ends_after, sources, targets, totals):
    """What becomes of a turn's rows and pages once the rows that `kept` marks stay (all arrays on the device: int32, ends int64)."""
    n, width = tables.shape
    tokens = slots.numel()
    if not (starts.numel() - 1 == held.numel() == held_after.numel() == n and kept.numel() == sources.numel() == targets.numel() == tokens and
            ring.numel() == pages.c.n_pages and ends.numel() == ends_after.numel() == 2 and totals.numel() == 2):
        raise ValueError("arrays of the kept rows do not fit each other")
    t, s, h, sl, k, r, ha, so, ta, to = _whole(_I32, tables, starts, held, slots, kept, ring, held_after, sources, targets, totals)
    e, ea = _whole(_I64, ends, ends_after)
    _check(lib().lococo_pages_keep(pages.ref, n, tokens, width, t, s, h, sl, k, r, e, ha, ea, so, ta, to, _stream_now()))


def lococo_pages_move(pages: Pages, starts, sources, targets):
    """The rows at sources to targets, as lococo_pages_keep leaves them, in one layer's pages."""
    if sources.numel() != targets.numel() or starts.numel() < 2:
        raise ValueError("sources and targets do not fit each other")
    _here(pages.k_codes)
    s, a, b = _whole(_I32, starts, sources, targets)
    _check(lib().lococo_pages_move(pages.ref, starts.numel() - 1, sources.numel(), s, a, b, _stream_now()))


def lococo_scan_status(cfg, workspace) -> int:
    """Synchronises; 0 = fine, 1 = a chain wait inside the one-launch scan of the lococo_sequence_forward or
    lococo_sequence_backward call that had this workspace gave up: its results are invalid."""
    out = C.c_int32(0)
    _check(lib().lococo_scan_status(C.byref(cfg), _ptr(workspace), C.byref(out)))
    return out.value


def lococo_measure_peaks(scratch: torch.Tensor) -> tuple:
    """(bf16 MFMA TFLOP/s of a bare loop, GB/s of a plain copy inside `scratch`) on the current GPU."""
    tf, gbs = C.c_double(0.0), C.c_double(0.0)
    _check(lib().lococo_measure_peaks(_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(),
                                      C.byref(tf), C.byref(gbs)))
    return tf.value, gbs.value


def lococo_debug_option(option: int, value: int = 0):
    """Process-wide test / measurement hook (see LOCOCO_OPT_* in lococo.h)."""
    _check(lib().lococo_debug_option(option, value))


def lococo_describe_path(cfg, B: int) -> dict:
    """Which kernels the configuration runs on, on the current device."""
    out = lococo_path_info()
    _check(lib().lococo_describe_path(C.byref(cfg), B, C.byref(out)))
    return {"path": out.path, "compute_units": out.compute_units, "tile_slots": out.tile_slots,
            "scan_groups": out.scan_groups, "scan_resident_limit": out.scan_resident_limit,
            "position_split": out.position_split, "step_pipeline": out.step_pipeline}


def lococo_timing_begin():
    _check(lib().lococo_timing_begin())


def lococo_timing_end() -> dict:
    """{kernel name: (launches, total_ms)} for the kernels launched since lococo_timing_begin."""
    rows = (lococo_kernel_time * 32)()
    n = C.c_int32(32)
    _check(lib().lococo_timing_end(rows, C.byref(n)))
    return {rows[i].name.decode(): (rows[i].launches, rows[i].total_ms) for i in range(n.value)}


def workspace(cfg, L: int, B: int, history: bool = False, device="cuda") -> torch.Tensor | None:
    """Allocate (through torch) the workspace a call with these sizes needs."""
    n = lococo_workspace_bytes(cfg, L, B, history)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device) if n else None


def pages_workspace(pages: Pages, n: int, tokens: int, max_new: int, max_held: int, trees: bool = True) -> torch.Tensor | None:
    """Allocate (through torch) the workspace of lococo_pages_attn calls of these sizes (max_held may be larger than theirs) and, unless
    `trees` is False, of lococo_pages_attn_tree calls, which may take 17 MB and 48 bytes a tile of rows where the others take nothing."""
    need = lococo_pages_workspace_bytes(pages, n, tokens, max_new, max_held)
    if trees:
        need = max(need, lococo_pages_attn_tree_workspace_bytes(pages, n, tokens, max_new, max_held))
    return torch.empty(need, dtype=torch.uint8, device=pages.device) if need else None


def rotate_workspace(rot: Rotation, tokens: int, device="cuda") -> torch.Tensor | None:
    """Allocate (through torch) the workspace of lococo_rows_rotate_backward calls of `tokens` rows with gradients of weights."""
    need = lococo_rows_rotate_backward_workspace_bytes(rot, tokens)
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


def config_for(w, impl: int = 0, **over) -> lococo_config:
    """lococo_config of an inputs.Workload."""
    Cc = w.C
    kw = dict(dtype=w.torch_dtype, batch=w.batch, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads,
              head_dim=w.head_dim, M=w.M, conv_width=w.conv_width, conv_in=w.conv_in, norm=w.norm,
              impl=impl,
              w_head_stride=w.M * Cc * w.conv_width if w.per_head_filters else 0,
              b_head_stride=w.M if w.per_head_filters else 0)
    kw.update(over)
    return make_config(**kw)
