"""ctypes binding of libspr: one Python function per C entry point, same
name without the ``spr_`` prefix, same argument order.  Argument
marshalling only (tensor -> device pointer, stream -> hipStream_t, status ->
exception); every step of the computation runs in the HIP library.

Tensors must be contiguous GPU tensors; ``None`` passes a NULL pointer.
The library must be built (``python -m paper_2606_01143_amd.build``);
loading fails loudly otherwise -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libspr.so")

SPR_F32 = 0
SPR_BF16 = 1
SPR_DETERMINISTIC = 1
SPR_ATOMIC_DQ = 2

OP_PREFIX_FWD = 0
OP_SUFFIX_FWD = 1
OP_SUFFIX_BWD = 2
OP_PREFIX_BWD = 3
OP_DENSE_BASELINE = 4
OP_SUFFIX_FWD_PADDED = 5
OP_SUFFIX_BWD_PADDED = 6

STATUS = {0: "SPR_OK", 1: "SPR_ERR_INVALID_ARG", 2: "SPR_ERR_UNSUPPORTED",
          3: "SPR_ERR_MISALIGNED", 4: "SPR_ERR_ALIASING", 5: "SPR_ERR_WORKSPACE",
          6: "SPR_ERR_HIP"}

# C symbol -> (argtypes, restype)
_P = c_void_p
_SIGNATURES = {
    "spr_prefix_fwd": ([_P, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_suffix_attn_fwd": ([_P, _P, _P, _P, _P, _P, _P, c_int32, c_int32, c_int32, _P, _P, _P,
                             c_size_t, _P], c_int32),
    "spr_suffix_attn_fwd_noalloc": ([_P, _P, _P, _P, _P, _P, _P, c_int32, c_int32, c_int32, _P, _P,
                                     _P], c_int32),
    "spr_suffix_attn_bwd_accum": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, c_int32, c_int32, c_int32,
                                   _P, _P, _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_prefix_bwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_suffix_attn_fwd_padded": ([_P, _P, _P, _P, _P, _P, _P, c_int32, c_int32, _P, _P, _P, c_size_t, _P],
                                   c_int32),
    "spr_suffix_attn_bwd_accum_padded": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, c_int32, c_int32, _P, _P,
                                          _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_prefix_bwd_dq": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_prefix_bwd_dkv": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_dense_recompute_baseline": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, c_int32, c_int32,
                                      c_int32, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                      c_size_t, _P], c_int32),
    "spr_workspace_size": ([c_int32, _P, c_int32, c_int32, c_int32, POINTER(c_size_t)], c_int32),
    "spr_check_cu_seqlens": ([POINTER(c_int32), c_int32, c_int32, c_int32], c_int32),
    "spr_gkv_cache_zero": ([_P, _P, _P, _P], c_int32),
    "spr_gkv_accumulate": ([_P, _P, _P, _P, _P, _P], c_int32),
    "spr_rmsnorm_fwd": ([c_int32, c_int32, c_float, _P, _P, _P, _P], c_int32),
    "spr_rmsnorm_bwd": ([c_int32, c_int32, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_rope_fwd": ([c_int32, c_int32, c_int32, c_int32, c_double, _P, _P, _P], c_int32),
    "spr_rope_bwd": ([c_int32, c_int32, c_int32, c_int32, c_double, _P, _P, _P], c_int32),
    "spr_head_norm_rope_fwd": ([c_int32, c_int32, c_int32, c_int32, c_int32, c_float, c_int32, _P, c_double, _P,
                                c_int64, _P, c_int64, _P, _P, _P, _P, _P], c_int32),
    "spr_head_norm_rope_bwd": ([c_int32, c_int32, c_int32, c_int32, c_int32, c_float, c_int32, _P, c_double, _P,
                                c_int64, _P, c_int64, _P, _P, _P, _P, _P, c_int64, _P, c_int64, _P, _P, c_int32, _P,
                                c_size_t, _P], c_int32),
    "spr_head_norm_rope_bwd_workspace_size": ([c_int32, c_int32, c_int32, c_int32, POINTER(c_size_t)], c_int32),
    "spr_embed_fwd": ([c_int32, c_int32, c_int32, c_int32, c_float, _P, _P, _P, _P], c_int32),
    "spr_embed_bwd": ([c_int32, c_int32, c_int32, c_int32, c_float, _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_embed_bwd_workspace_size": ([c_int32, c_int32, c_int32, POINTER(c_size_t)], c_int32),
    "spr_swiglu_fwd": ([c_int64, _P, _P, _P, _P], c_int32),
    "spr_swiglu_bwd": ([c_int64, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_grad_accumulate": ([c_int64, _P, _P, c_int32, _P], c_int32),
    "spr_experts_plan": ([c_int32, c_int32, c_int32, _P, _P, _P, _P, _P, c_size_t, _P], c_int32),
    "spr_experts_plan_workspace_size": ([c_int32, c_int32, c_int32, POINTER(c_size_t)], c_int32),
    "spr_experts_fwd": ([c_int32, c_int32, c_int32, c_int32, _P, _P, c_int32, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_experts_bwd_x": ([c_int32, c_int32, c_int32, c_int32, _P, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_experts_bwd_w": ([c_int32, c_int32, c_int32, c_int32, _P, _P, c_int32, _P, _P, _P, _P, _P, c_int32, _P],
                          c_int32),
    "spr_experts_combine_fwd": ([c_int32, c_int32, c_int32, c_int32, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_experts_combine_bwd": ([c_int32, c_int32, c_int32, c_int32, _P, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_act8_pack": ([c_int32, c_int32, c_int32, _P, _P, _P, _P], c_int32),
    "spr_act8_unpack": ([c_int32, c_int32, c_int32, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_block_norm_fwd": ([c_int32, c_int32, c_int32, c_float, c_float, c_float, _P, _P, _P, _P, c_int32, _P, _P, _P,
                            _P, _P, _P, _P, _P, _P, _P], c_int32),
    "spr_block_norm_bwd": ([c_int32, c_int32, c_int32, c_float, c_float, _P, _P, _P, _P, _P, _P, _P, _P, c_int32, _P,
                            _P, _P, _P, _P, _P, _P, _P, c_int32, _P, c_size_t, _P], c_int32),
    "spr_block_norm_bwd_workspace_size": ([c_int32, c_int32, POINTER(c_size_t)], c_int32),
    "spr_glu_fwd": ([c_int32, c_int32, c_int32, c_int32, c_int32, _P, _P, c_int32, _P, _P, _P, _P, _P, _P, _P, _P,
                     _P], c_int32),
    "spr_glu_bwd": ([c_int32, c_int32, c_int32, c_int32, c_int32, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P],
                    c_int32),
    "spr_moe_stats_bytes": ([c_int32, POINTER(c_size_t)], c_int32),
    "spr_moe_stats_zero": ([c_int32, _P, _P], c_int32),
    "spr_moe_aux_workspace_size": ([c_int32, c_int32, POINTER(c_size_t)], c_int32),
    "spr_moe_aux_accumulate": ([c_int32, c_int32, c_int32, _P, _P, c_int32, _P, _P, _P, c_size_t, _P],
                               c_int32),
    "spr_moe_aux_loss": ([c_int32, c_int32, c_double, _P, _P, _P, _P, _P], c_int32),
    "spr_moe_aux_grad": ([c_int32, c_int32, c_double, c_double, _P, c_int32, c_int32, _P, _P, _P],
                         c_int32),
    "spr_profile_enable": ([c_int32, c_char_p], c_int32),
    "spr_profile_reset": ([], c_int32),
    "spr_profile_query": ([c_char_p, POINTER(c_double), POINTER(c_int32)], c_int32),
    "spr_profile_num_kernels": ([], c_int32),
    "spr_profile_kernel_name": ([c_int32], c_char_p),
    "spr_status_string": ([c_int32], c_char_p),
    "spr_last_error": ([], c_char_p),
    "spr_version": ([], c_char_p),
}


class SprDims(ctypes.Structure):
    """Mirror of ``spr_dims`` in include/spr.h."""
    _fields_ = [("num_q_heads", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32),
                ("prefix_len", c_int32), ("softmax_scale", c_float), ("dtype", c_int32),
                ("flags", c_uint32)]


class SprError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        self.status_name = STATUS.get(status, f"status {status}")
        super().__init__(f"{self.status_name}: {message}")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libspr.so (once) and declare every entry point's signature."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"libspr.so is not built ({LIB_PATH}); build it with "
                "`python -m paper_2606_01143_amd.build` -- there is no fallback path")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (argtypes, restype) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.argtypes = argtypes
            fn.restype = restype
        _lib = handle
    return _lib


def make_dims(num_q_heads: int, num_kv_heads: int, head_dim: int, prefix_len: int,
              dtype: str = "bf16", softmax_scale: float = 0.0,
              deterministic: bool = False, atomic_dq: bool = False) -> SprDims:
    code = {"f32": SPR_F32, "bf16": SPR_BF16}[dtype]
    flags = (SPR_DETERMINISTIC if deterministic else 0) | (SPR_ATOMIC_DQ if atomic_dq else 0)
    return SprDims(num_q_heads, num_kv_heads, head_dim, prefix_len, softmax_scale, code, flags)


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_cuda:
        raise ValueError("libspr takes GPU tensors only")
    if not x.is_contiguous():
        raise ValueError("libspr takes contiguous tensors only")
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        # the current stream's handle without building a Stream object, which
        # takes 2.6 us, as long as the launch itself
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


class _Sizes:
    """Required sizes of one call's tensors, from the dims and the row counts.

    The C ABI takes plain pointers and cannot see a buffer's size; a tensor
    that is too small, or of another element type than the dims say, would
    be read or written past its end on the GPU.  Every attention wrapper
    therefore checks its tensors here first (None is a NULL pointer and is
    left to the library's own checks)."""

    def __init__(self, dims, rows_s: int = 0):
        self.P, self.hq, self.hkv, self.d = (int(dims.prefix_len), int(dims.num_q_heads),
                                             int(dims.num_kv_heads), int(dims.head_dim))
        self.eb = 4 if dims.dtype == SPR_F32 else 2
        self.T = int(rows_s)

    def _need(self, name, x, elems, esize):
        if x is None or isinstance(x, int):
            return
        if x.element_size() != esize:
            raise ValueError(f"{name}: elements of {x.element_size()} bytes, the call needs {esize}")
        if x.numel() < elems:
            raise ValueError(f"{name}: {x.numel()} elements, the call needs {elems}")

    def q(self, rows, **kw):   # [rows, Hq, d] storage dtype
        for k, v in kw.items():
            self._need(k, v, rows * self.hq * self.d, self.eb)

    def kv(self, rows, **kw):  # [rows, Hkv, d] storage dtype
        for k, v in kw.items():
            self._need(k, v, rows * self.hkv * self.d, self.eb)

    def lse(self, rows, **kw):  # [rows, Hq] fp32
        for k, v in kw.items():
            self._need(k, v, rows * self.hq, 4)

    def cache(self, **kw):     # [P, Hkv, d] fp32
        for k, v in kw.items():
            self._need(k, v, self.P * self.hkv * self.d, 4)

    def i32(self, n, **kw):
        for k, v in kw.items():
            self._need(k, v, n, 4)


def _check(status: int) -> None:
    if status != 0:
        raise SprError(status, lib().spr_last_error().decode())


def check_cu_seqlens(cu_host, n_mb, max_len, total_len) -> None:
    """Host-side check of a microbatch's suffix offsets (the values uploaded
    as cu_seqlens): raises SprError(SPR_ERR_INVALID_ARG) on a zero-length
    suffix or offsets inconsistent with n_mb / max_len / total_len."""
    vals = [int(x) for x in cu_host]
    if len(vals) != int(n_mb) + 1:
        raise SprError(1, f"cu_seqlens has {len(vals)} entries, n_mb + 1 = {int(n_mb) + 1} expected")
    arr = (c_int32 * len(vals))(*vals)
    _check(lib().spr_check_cu_seqlens(arr, n_mb, max_len, total_len))


def _nbytes(ws) -> int:
    return 0 if ws is None else ws.numel() * ws.element_size()


# ------------------------------------------------------------ entry points
def prefix_fwd(dims, q_p, k_p, v_p, o_p, lse_p, stream=None):
    z = _Sizes(dims)
    z.q(z.P, q_p=q_p, o_p=o_p)
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.lse(z.P, lse_p=lse_p)
    _check(lib().spr_prefix_fwd(byref(dims), _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p),
                                _ptr(lse_p), _stream(stream)))


def suffix_attn_fwd(dims, k_p, v_p, q_s, k_s, v_s, cu_seqlens, n_mb, max_len, total_len, o_s,
                    lse_s, ws=None, stream=None, cu_host=None):
    """``cu_host``: the host copy of cu_seqlens, checked first when given."""
    if cu_host is not None:
        check_cu_seqlens(cu_host, n_mb, max_len, total_len)
    z = _Sizes(dims, total_len)
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.q(z.T, q_s=q_s, o_s=o_s)
    z.kv(z.T, k_s=k_s, v_s=v_s)
    z.lse(z.T, lse_s=lse_s)
    z.i32(int(n_mb) + 1, cu_seqlens=cu_seqlens)
    _check(lib().spr_suffix_attn_fwd(byref(dims), _ptr(k_p), _ptr(v_p), _ptr(q_s), _ptr(k_s),
                                     _ptr(v_s), _ptr(cu_seqlens), n_mb, max_len, total_len,
                                     _ptr(o_s), _ptr(lse_s), _ptr(ws), _nbytes(ws),
                                     _stream(stream)))


# bytes of the static device scratch behind suffix_attn_fwd_noalloc
STATIC_SCRATCH_BYTES = 64 << 20


def suffix_attn_fwd_noalloc(dims, k_p, v_p, q_s, k_s, v_s, cu_seqlens, n_mb, max_len, total_len,
                            o_s, lse_s, stream=None, cu_host=None):
    """suffix_attn_fwd with the library's static scratch as its workspace:
    no device allocation anywhere (callers under graph capture, serving
    loops).  Calls that overlap on one GPU race on the scratch."""
    if cu_host is not None:
        check_cu_seqlens(cu_host, n_mb, max_len, total_len)
    z = _Sizes(dims, total_len)
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.q(z.T, q_s=q_s, o_s=o_s)
    z.kv(z.T, k_s=k_s, v_s=v_s)
    z.lse(z.T, lse_s=lse_s)
    z.i32(int(n_mb) + 1, cu_seqlens=cu_seqlens)
    _check(lib().spr_suffix_attn_fwd_noalloc(byref(dims), _ptr(k_p), _ptr(v_p), _ptr(q_s), _ptr(k_s),
                                             _ptr(v_s), _ptr(cu_seqlens), n_mb, max_len, total_len,
                                             _ptr(o_s), _ptr(lse_s), _stream(stream)))


def suffix_attn_bwd_accum(dims, k_p, v_p, q_s, k_s, v_s, o_s, lse_s, do_s, cu_seqlens, n_mb,
                          max_len, total_len, dq_s, dk_s, dv_s, gk_cache, gv_cache, ws=None,
                          stream=None, cu_host=None):
    """``cu_host``: the host copy of cu_seqlens, checked first when given."""
    if cu_host is not None:
        check_cu_seqlens(cu_host, n_mb, max_len, total_len)
    z = _Sizes(dims, total_len)
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.q(z.T, q_s=q_s, o_s=o_s, do_s=do_s, dq_s=dq_s)
    z.kv(z.T, k_s=k_s, v_s=v_s, dk_s=dk_s, dv_s=dv_s)
    z.lse(z.T, lse_s=lse_s)
    z.cache(gk_cache=gk_cache, gv_cache=gv_cache)
    z.i32(int(n_mb) + 1, cu_seqlens=cu_seqlens)
    _check(lib().spr_suffix_attn_bwd_accum(
        byref(dims), _ptr(k_p), _ptr(v_p), _ptr(q_s), _ptr(k_s), _ptr(v_s), _ptr(o_s),
        _ptr(lse_s), _ptr(do_s), _ptr(cu_seqlens), n_mb, max_len, total_len, _ptr(dq_s),
        _ptr(dk_s), _ptr(dv_s), _ptr(gk_cache), _ptr(gv_cache), _ptr(ws), _nbytes(ws),
        _stream(stream)))


def prefix_bwd(dims, q_p, k_p, v_p, o_p, lse_p, do_p, gk_cache, gv_cache, dq_p, dk_p, dv_p,
               ws=None, stream=None):
    z = _Sizes(dims)
    z.q(z.P, q_p=q_p, o_p=o_p, do_p=do_p, dq_p=dq_p)
    z.kv(z.P, k_p=k_p, v_p=v_p, dk_p=dk_p, dv_p=dv_p)
    z.lse(z.P, lse_p=lse_p)
    z.cache(gk_cache=gk_cache, gv_cache=gv_cache)
    _check(lib().spr_prefix_bwd(byref(dims), _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p),
                                _ptr(lse_p), _ptr(do_p), _ptr(gk_cache), _ptr(gv_cache),
                                _ptr(dq_p), _ptr(dk_p), _ptr(dv_p), _ptr(ws), _nbytes(ws),
                                _stream(stream)))


def suffix_attn_fwd_padded(dims, k_p, v_p, q_s, k_s, v_s, seq_lens, n, s_max, o_s, lse_s, ws=None,
                           stream=None):
    z = _Sizes(dims, int(n) * int(s_max))
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.q(z.T, q_s=q_s, o_s=o_s)
    z.kv(z.T, k_s=k_s, v_s=v_s)
    z.lse(z.T, lse_s=lse_s)
    z.i32(int(n), seq_lens=seq_lens)
    _check(lib().spr_suffix_attn_fwd_padded(byref(dims), _ptr(k_p), _ptr(v_p), _ptr(q_s), _ptr(k_s),
                                            _ptr(v_s), _ptr(seq_lens), n, s_max, _ptr(o_s), _ptr(lse_s),
                                            _ptr(ws), _nbytes(ws), _stream(stream)))


def suffix_attn_bwd_accum_padded(dims, k_p, v_p, q_s, k_s, v_s, o_s, lse_s, do_s, seq_lens, n, s_max,
                                 dq_s, dk_s, dv_s, gk_cache, gv_cache, ws=None, stream=None):
    z = _Sizes(dims, int(n) * int(s_max))
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.q(z.T, q_s=q_s, o_s=o_s, do_s=do_s, dq_s=dq_s)
    z.kv(z.T, k_s=k_s, v_s=v_s, dk_s=dk_s, dv_s=dv_s)
    z.lse(z.T, lse_s=lse_s)
    z.cache(gk_cache=gk_cache, gv_cache=gv_cache)
    z.i32(int(n), seq_lens=seq_lens)
    _check(lib().spr_suffix_attn_bwd_accum_padded(
        byref(dims), _ptr(k_p), _ptr(v_p), _ptr(q_s), _ptr(k_s), _ptr(v_s), _ptr(o_s), _ptr(lse_s),
        _ptr(do_s), _ptr(seq_lens), n, s_max, _ptr(dq_s), _ptr(dk_s), _ptr(dv_s), _ptr(gk_cache),
        _ptr(gv_cache), _ptr(ws), _nbytes(ws), _stream(stream)))


def prefix_bwd_dq(dims, q_p, k_p, v_p, o_p, lse_p, do_p, dq_p, ws=None, stream=None):
    z = _Sizes(dims)
    z.q(z.P, q_p=q_p, o_p=o_p, do_p=do_p, dq_p=dq_p)
    z.kv(z.P, k_p=k_p, v_p=v_p)
    z.lse(z.P, lse_p=lse_p)
    _check(lib().spr_prefix_bwd_dq(byref(dims), _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p),
                                   _ptr(lse_p), _ptr(do_p), _ptr(dq_p), _ptr(ws), _nbytes(ws),
                                   _stream(stream)))


def prefix_bwd_dkv(dims, q_p, k_p, v_p, o_p, lse_p, do_p, gk_cache, gv_cache, dk_p, dv_p,
                   ws=None, stream=None):
    z = _Sizes(dims)
    z.q(z.P, q_p=q_p, o_p=o_p, do_p=do_p)
    z.kv(z.P, k_p=k_p, v_p=v_p, dk_p=dk_p, dv_p=dv_p)
    z.lse(z.P, lse_p=lse_p)
    z.cache(gk_cache=gk_cache, gv_cache=gv_cache)
    _check(lib().spr_prefix_bwd_dkv(byref(dims), _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p),
                                    _ptr(lse_p), _ptr(do_p), _ptr(gk_cache), _ptr(gv_cache),
                                    _ptr(dk_p), _ptr(dv_p), _ptr(ws), _nbytes(ws),
                                    _stream(stream)))


def dense_recompute_baseline(dims, q_p, k_p, v_p, do_p_seq, q_s, k_s, v_s, do_s, cu_seqlens, n,
                             max_len, total_len, o_p, lse_p, o_s, lse_s, dq_s, dk_s, dv_s, dq_p,
                             dk_p, dv_p, ws=None, stream=None, cu_host=None):
    """``cu_host``: the host copy of cu_seqlens, checked first when given."""
    if cu_host is not None:
        check_cu_seqlens(cu_host, n, max_len, total_len)
    z = _Sizes(dims, total_len)
    z.q(z.P, q_p=q_p, o_p=o_p, dq_p=dq_p)
    z.q(int(n) * z.P, do_p_seq=do_p_seq)
    z.kv(z.P, k_p=k_p, v_p=v_p, dk_p=dk_p, dv_p=dv_p)
    z.lse(z.P, lse_p=lse_p)
    z.q(z.T, q_s=q_s, o_s=o_s, do_s=do_s, dq_s=dq_s)
    z.kv(z.T, k_s=k_s, v_s=v_s, dk_s=dk_s, dv_s=dv_s)
    z.lse(z.T, lse_s=lse_s)
    z.i32(int(n) + 1, cu_seqlens=cu_seqlens)
    _check(lib().spr_dense_recompute_baseline(
        byref(dims), _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(do_p_seq), _ptr(q_s), _ptr(k_s),
        _ptr(v_s), _ptr(do_s), _ptr(cu_seqlens), n, max_len, total_len, _ptr(o_p), _ptr(lse_p),
        _ptr(o_s), _ptr(lse_s), _ptr(dq_s), _ptr(dk_s), _ptr(dv_s), _ptr(dq_p), _ptr(dk_p),
        _ptr(dv_p), _ptr(ws), _nbytes(ws), _stream(stream)))


def _need_all(elems, esize, **tensors):
    """Every named tensor holds at least `elems` elements of `esize` bytes
    (None: a NULL pointer, left to the library)."""
    for name, x in tensors.items():
        if x is None:
            continue
        if x.element_size() != esize:
            raise ValueError(f"{name}: elements of {x.element_size()} bytes, the call needs {esize}")
        if x.numel() < elems:
            raise ValueError(f"{name}: {x.numel()} elements, the call needs {elems}")


def rmsnorm_fwd(x, y, rstd, eps=1e-5, stream=None):
    rows, width = int(x.shape[0]), int(x.shape[-1])
    _need_all(rows * width, 2, x=x, y=y)
    _need_all(rows, 4, rstd=rstd)
    _check(lib().spr_rmsnorm_fwd(rows, width, eps, _ptr(x), _ptr(y), _ptr(rstd), _stream(stream)))


def rmsnorm_bwd(x, rstd, dy, dx, add=None, stream=None):
    rows, width = int(x.shape[0]), int(x.shape[-1])
    _need_all(rows * width, 2, x=x, dy=dy, dx=dx, add=add)
    _need_all(rows, 4, rstd=rstd)
    _check(lib().spr_rmsnorm_bwd(rows, width, _ptr(x), _ptr(rstd), _ptr(dy), _ptr(add), _ptr(dx),
                                 _stream(stream)))


def rope_fwd(x, y, pos0, theta, stream=None):
    t, h, d = (int(v) for v in x.shape)
    _need_all(t * h * d, 2, x=x, y=y)
    _check(lib().spr_rope_fwd(t, h, d, pos0, float(theta), _ptr(x), _ptr(y), _stream(stream)))


def rope_bwd(dy, dx, pos0, theta, stream=None):
    t, h, d = (int(v) for v in dy.shape)
    _need_all(t * h * d, 2, dy=dy, dx=dx)
    _check(lib().spr_rope_bwd(t, h, d, pos0, float(theta), _ptr(dy), _ptr(dx), _stream(stream)))


def _fits(*sizes):
    """The C calls take 32-bit sizes, of which ctypes would pass the low bits.
    Callers test the sizes' common bits first, a third of this call's time."""
    if max(sizes) > 0x7FFFFFFF:
        raise ValueError(f"a size of {max(sizes)}: the call takes at most 2^31 - 1")


def _refuse(name, x, dtype, shape, dev):
    """Why _arg turned a tensor away."""
    if x.dtype is not dtype:
        raise ValueError(f"{name}: {x.dtype}, the call needs {dtype}")
    if shape is not None and x.shape != shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, the call needs {tuple(shape)}")
    if not x.is_cuda:
        raise ValueError("libspr takes GPU tensors only")
    if x.get_device() != dev:
        raise ValueError(f"{name} is on cuda:{x.get_device()}, not on the call's device cuda:{dev}")
    raise ValueError("libspr takes contiguous tensors only")


def _arg(name, x, dtype, shape, dev):
    """Pointer of a contiguous tensor of that type and shape on device ``dev``
    (the type exactly: fp16 has bf16's size); None is left to the library."""
    if x is None:
        return None
    if x.dtype is dtype and x.shape == shape and x.get_device() == dev and x.is_contiguous():
        return x.data_ptr()
    _refuse(name, x, dtype, shape, dev)


def _rows_arg(name, x, dtype, shape, dev):
    """Pointer and token stride of [tokens, heads, d] whose heads and values
    are contiguous (a view of a fused projection)."""
    if x.dtype is not dtype or x.shape != shape or x.get_device() != dev:
        _refuse(name, x, dtype, shape, dev)
    t, h, d = shape
    s0, s1, s2 = x.stride()
    if (d > 1 and s2 != 1) or (h > 1 and s1 != d):
        raise ValueError(f"{name}: a token's heads are not contiguous")
    if t <= 1:
        return x.data_ptr(), h * d
    if s0 < h * d:
        raise ValueError(f"{name}: tokens overlap (stride {s0}, a token has {h * d} elements)")
    return x.data_ptr(), s0


def _ws(ws, dev):
    """Pointer and bytes of a workspace (None: a NULL pointer)."""
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        _refuse("ws", ws, ws.dtype, None, dev)
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _storage(name, x):
    """The library's dtype code of a tensor that may be bf16 or fp32."""
    import torch
    if x.dtype is torch.bfloat16:
        return SPR_BF16
    if x.dtype is torch.float32:
        return SPR_F32
    raise ValueError(f"{name}: {x.dtype}, the call takes bfloat16 or float32")


def _on(dev, stream):
    """The stream of a call whose tensors lie on ``dev``: it has to be the
    current device, whose stream is taken where none is given."""
    import torch
    if dev < 0:
        raise ValueError("libspr takes GPU tensors only")
    if dev != torch.cuda.current_device():
        raise ValueError(f"the tensors are on cuda:{dev}, not on the current device "
                         f"cuda:{torch.cuda.current_device()}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    return stream if isinstance(stream, int) else stream.cuda_stream


def head_norm_rope_bwd_workspace_size(tokens, q_heads, kv_heads, head_dim) -> int:
    out = c_size_t(0)
    if (tokens | q_heads | kv_heads | head_dim) >> 31:
        _fits(tokens, q_heads, kv_heads, head_dim)
    _check(lib().spr_head_norm_rope_bwd_workspace_size(tokens, q_heads, kv_heads, head_dim, byref(out)))
    return int(out.value)


def head_norm_rope_fwd(q, k, gain_q, gain_k, yq, yk, pos0, theta, positions=None, eps=1e-6, stream=None):
    """RMS norm of every head of q [T, Hq, d] and k [T, Hkv, d] with gains [d],
    then the rotary embedding, in one pass; q and k may be views of one fused
    projection (heads contiguous).  ``positions``: int32 [T], added to pos0 in
    place of 0 .. T - 1."""
    import torch
    sq, (t, hkv, d), dt, dev = q.shape, k.shape, q.dtype, q.get_device()
    code, hq, sk = _storage("q", q), sq[1], (sq[0], hkv, sq[2])
    if (t | pos0) >> 31:
        _fits(t, pos0)
    pq, stride_q = _rows_arg("q", q, dt, sq, dev)
    pk, stride_k = _rows_arg("k", k, dt, sk, dev)
    args = (_arg("gain_q", gain_q, dt, (d,), dev), _arg("gain_k", gain_k, dt, (d,), dev), _arg("yq", yq, dt, sq, dev),
            _arg("yk", yk, dt, sk, dev))
    _check(lib().spr_head_norm_rope_fwd(code, t, hq, hkv, d, float(eps), pos0,
                                        _arg("positions", positions, torch.int32, (t,), dev), float(theta), pq, stride_q, pk,
                                        stride_k, *args, _on(dev, stream)))


def head_norm_rope_bwd(q, k, gain_q, gain_k, dyq, dyk, dq, dk, dgain_q, dgain_k, pos0, theta, positions=None,
                       eps=1e-6, overwrite=False, ws=None, stream=None):
    """Backward of head_norm_rope_fwd from its inputs: dq and dk (also views of
    one fused gradient) are written, dgain_q and dgain_k [d] fp32 added to, or
    written where ``overwrite``."""
    import torch
    sq, (t, hkv, d), dt, dev = q.shape, k.shape, q.dtype, q.get_device()
    code, hq, sk, f32 = _storage("q", q), sq[1], (sq[0], hkv, sq[2]), torch.float32
    if (t | pos0) >> 31:
        _fits(t, pos0)
    pq, stride_q = _rows_arg("q", q, dt, sq, dev)
    pk, stride_k = _rows_arg("k", k, dt, sk, dev)
    ins = (_arg("gain_q", gain_q, dt, (d,), dev), _arg("gain_k", gain_k, dt, (d,), dev),
           _arg("dyq", dyq, dt, sq, dev), _arg("dyk", dyk, dt, sk, dev))
    outs = (*_rows_arg("dq", dq, dt, sq, dev), *_rows_arg("dk", dk, dt, sk, dev),
            _arg("dgain_q", dgain_q, f32, (d,), dev), _arg("dgain_k", dgain_k, f32, (d,), dev))
    _check(lib().spr_head_norm_rope_bwd(code, t, hq, hkv, d, float(eps), pos0,
                                        _arg("positions", positions, torch.int32, (t,), dev), float(theta), pq, stride_q, pk,
                                        stride_k, *ins, *outs, 1 if overwrite else 0, *_ws(ws, dev),
                                        _on(dev, stream)))


def embed_fwd(ids, table, y, scale=1.0, stream=None):
    """y[t] = scale * table[ids[t]]; an id outside the table gives zeros."""
    import torch
    (t,), (v, w), dt, dev = ids.shape, table.shape, table.dtype, table.get_device()
    code = _storage("table", table)
    if (t | v | w) >> 31:
        _fits(t, v, w)
    _check(lib().spr_embed_fwd(code, t, v, w, float(scale), _arg("ids", ids, torch.int32, (t,), dev),
                               _arg("table", table, dt, (v, w), dev), _arg("y", y, dt, (t, w), dev),
                               _on(dev, stream)))


def embed_bwd_workspace_size(tokens, vocab, width) -> int:
    out = c_size_t(0)
    if (tokens | vocab | width) >> 31:
        _fits(tokens, vocab, width)
    _check(lib().spr_embed_bwd_workspace_size(tokens, vocab, width, byref(out)))
    return int(out.value)


def embed_bwd(ids, dy, dtable, scale=1.0, ws=None, stream=None):
    """dtable[v] += scale * the sum of dy over v's tokens, fp32, in token order."""
    import torch
    (t,), (v, w), dev = ids.shape, dtable.shape, dtable.get_device()
    code = _storage("dy", dy)
    if (t | v | w) >> 31:
        _fits(t, v, w)
    _check(lib().spr_embed_bwd(code, t, v, w, float(scale), _arg("ids", ids, torch.int32, (t,), dev),
                               _arg("dy", dy, dy.dtype, (t, w), dev),
                               _arg("dtable", dtable, torch.float32, (v, w), dev), *_ws(ws, dev),
                               _on(dev, stream)))


def swiglu_fwd(g, u, m, stream=None):
    n = int(g.numel())
    _need_all(n, 2, g=g, u=u, m=m)
    _check(lib().spr_swiglu_fwd(n, _ptr(g), _ptr(u), _ptr(m), _stream(stream)))


def swiglu_bwd(g, u, dm, dg, du, stream=None):
    n = int(g.numel())
    _need_all(n, 2, g=g, u=u, dm=dm, dg=dg, du=du)
    _check(lib().spr_swiglu_bwd(n, _ptr(g), _ptr(u), _ptr(dm), _ptr(dg), _ptr(du),
                                _stream(stream)))


def grad_accumulate(dst, src, overwrite=False, stream=None):
    n = int(dst.numel())
    _need_all(n, 4, dst=dst)
    _need_all(n, 2, src=src)
    _check(lib().spr_grad_accumulate(n, _ptr(src), _ptr(dst), 1 if overwrite else 0, _stream(stream)))


def experts_plan_workspace_size(n_experts, top_k, n_tokens) -> int:
    out = c_size_t(0)
    if (n_experts | top_k | n_tokens) >> 31:
        _fits(n_experts, top_k, n_tokens)
    _check(lib().spr_experts_plan_workspace_size(n_experts, top_k, n_tokens, byref(out)))
    return int(out.value)


def experts_plan(n_experts, experts, offsets, row_token, pos, ws=None, stream=None):
    """Stable sort of experts [T, k] by expert: offsets [E + 1], row_token
    [T k] and pos [T, k], all int32; ids outside [0, E) are dropped."""
    import torch
    (t, k), i32, dev = experts.shape, torch.int32, experts.get_device()
    if (n_experts | t | k) >> 31:
        _fits(n_experts, t, k)
    _check(lib().spr_experts_plan(n_experts, k, t, _arg("experts", experts, i32, (t, k), dev),
                                  _arg("offsets", offsets, i32, (n_experts + 1,), dev),
                                  _arg("row_token", row_token, i32, (t * k,), dev), _arg("pos", pos, i32, (t, k), dev),
                                  *_ws(ws, dev), _on(dev, stream)))


def _groups(offsets, w, name="w"):
    """(E, in, out) of a weight [E, in, out], or with E = 1 of one dense block's
    [in, out], which goes without offsets."""
    if w.dim() == 2:
        if offsets is not None:
            raise ValueError(f"{name} [in, out] is one dense block's: no offsets")
        return (1, *w.shape)
    e, i, o = w.shape
    if offsets is None and e != 1:
        raise ValueError(f"{name} holds {e} experts: offsets say which rows are whose")
    return e, i, o


def experts_fwd(offsets, x, w, y, w2=None, y2=None, row_token=None, stream=None):
    """y[r] = x[row_token[r]] w[e] (x[r] without row_token) for the rows r of
    every expert e, w [E, in, out]; w2, y2: a second product of the same rows.
    offsets None: all rows are one expert's, w [1, in, out] or [in, out]."""
    import torch
    (e, i, o), rows, n, dev, bf, i32 = _groups(offsets, w), y.shape[0], x.shape[0], w.get_device(), torch.bfloat16, torch.int32
    if (e | rows | n | i | o) >> 31:
        _fits(e, rows, n, i, o)
    _check(lib().spr_experts_fwd(e, rows, i, o, _arg("offsets", offsets, i32, (e + 1,), dev),
                                 _arg("x", x, bf, (n, i), dev), n, _arg("row_token", row_token, i32, (rows,), dev),
                                 _arg("w", w, bf, w.shape, dev), _arg("y", y, bf, (rows, o), dev),
                                 _arg("w2", w2, bf, w.shape, dev), _arg("y2", y2, bf, (rows, o), dev),
                                 _on(dev, stream)))


def experts_bwd_x(offsets, dy, w, dx, dy2=None, w2=None, stream=None):
    """dx[r] = dy[r] w[e]^T (+ dy2[r] w2[e]^T) for the rows r of every expert
    (offsets None: of one, as experts_fwd)."""
    import torch
    (e, i, o), rows, dev, bf = _groups(offsets, w), dy.shape[0], w.get_device(), torch.bfloat16
    if (e | rows | i | o) >> 31:
        _fits(e, rows, i, o)
    _check(lib().spr_experts_bwd_x(e, rows, i, o, _arg("offsets", offsets, torch.int32, (e + 1,), dev),
                                   _arg("dy", dy, bf, (rows, o), dev), _arg("w", w, bf, w.shape, dev),
                                   _arg("dy2", dy2, bf, (rows, o), dev), _arg("w2", w2, bf, w.shape, dev),
                                   _arg("dx", dx, bf, (rows, i), dev), _on(dev, stream)))


def experts_bwd_w(offsets, x, dy, dw, dy2=None, dw2=None, row_token=None, overwrite=False, stream=None):
    """dw[e] += the sum over e's rows of x[row_token[r]]^T dy[r], fp32 (written
    where ``overwrite``); dy2, dw2: a second pair of the same rows; offsets
    None: one expert, as experts_fwd."""
    import torch
    (e, i, o), rows, n, dev, bf, i32 = _groups(offsets, dw, "dw"), dy.shape[0], x.shape[0], dw.get_device(), torch.bfloat16, torch.int32
    if (e | rows | n | i | o) >> 31:
        _fits(e, rows, n, i, o)
    _check(lib().spr_experts_bwd_w(e, rows, i, o, _arg("offsets", offsets, i32, (e + 1,), dev),
                                   _arg("x", x, bf, (n, i), dev), n, _arg("row_token", row_token, i32, (rows,), dev),
                                   _arg("dy", dy, bf, (rows, o), dev), _arg("dw", dw, torch.float32, dw.shape, dev),
                                   _arg("dy2", dy2, bf, (rows, o), dev),
                                   _arg("dw2", dw2, torch.float32, dw.shape, dev), 1 if overwrite else 0,
                                   _on(dev, stream)))


def experts_combine_fwd(y, pos, weights, out, add=None, stream=None):
    """out[t] = add[t] + the sum over j of weights[t, j] y[pos[t, j]]; weights
    None: ones.  A pos outside y's rows is skipped."""
    import torch
    (t, k), (rows, width), dev, bf = pos.shape, y.shape, y.get_device(), torch.bfloat16
    if (t | k | rows | width) >> 31:
        _fits(t, k, rows, width)
    _check(lib().spr_experts_combine_fwd(t, k, rows, width, _arg("y", y, bf, (rows, width), dev),
                                         _arg("pos", pos, torch.int32, (t, k), dev),
                                         _arg("weights", weights, torch.float32, (t, k), dev),
                                         _arg("add", add, bf, (t, width), dev), _arg("out", out, bf, (t, width), dev),
                                         _on(dev, stream)))


def experts_combine_bwd(dout, y, pos, weights, dy, dweights, stream=None):
    """dy[pos[t, j]] = weights[t, j] dout[t], dweights[t, j] = <y[pos[t, j]],
    dout[t]>; y and dweights may both be None, weights None means ones."""
    import torch
    (t, k), (rows, width), dev, bf, f32 = pos.shape, dy.shape, dy.get_device(), torch.bfloat16, torch.float32
    if (t | k | rows | width) >> 31:
        _fits(t, k, rows, width)
    _check(lib().spr_experts_combine_bwd(t, k, rows, width, _arg("dout", dout, bf, (t, width), dev),
                                         _arg("y", y, bf, (rows, width), dev),
                                         _arg("pos", pos, torch.int32, (t, k), dev),
                                         _arg("weights", weights, f32, (t, k), dev),
                                         _arg("dy", dy, bf, (rows, width), dev),
                                         _arg("dweights", dweights, f32, (t, k), dev), _on(dev, stream)))


ACTS = {"silu": 0, "gelu": 1}  # gelu: the tanh form


def act8_empty(rows, width, device):
    """Room for [rows, width] values in 8 bits: q int8 and the blocks' exponents
    e uint8 [rows, ceil(width / 32)]."""
    import torch
    return (torch.empty(rows, width, dtype=torch.int8, device=device),
            torch.empty(rows, (width + 31) // 32, dtype=torch.uint8, device=device))


def _kept(name, x, dtype, shape, dev):
    """Pointers of a tensor that is kept whole (and no exponents), or of a pair
    (q, e) in 8 bits; None is two NULL pointers."""
    if x is None:
        return None, None
    if not isinstance(x, (tuple, list)):
        return _arg(name, x, dtype, shape, dev), None
    import torch
    q, e = x
    return (_arg(name + " (q)", q, torch.int8, shape, dev),
            _arg(name + " (e)", e, torch.uint8, (shape[0], (shape[1] + 31) // 32), dev))


def act8_pack(x, q, e, stream=None):
    """x [rows, width], bf16 or fp32, to 8 bits: q int8, e the exponents of 32
    values each (``act8_empty`` makes room for both)."""
    (rows, width), dev = x.shape, x.get_device()
    code = _storage("x", x)
    if (rows | width) >> 31:
        _fits(rows, width)
    pq, pe = _kept("q", (q, e), None, x.shape, dev)
    _check(lib().spr_act8_pack(code, rows, width, _arg("x", x, x.dtype, x.shape, dev), pq, pe, _on(dev, stream)))


def act8_unpack(q, e, y, rstd=None, gain=None, stream=None):
    """y = the values of (q, e) (* rstd[row]) (* gain[column]), bf16 or fp32."""
    import torch
    (rows, width), dev = y.shape, y.get_device()
    code = _storage("y", y)
    if (rows | width) >> 31:
        _fits(rows, width)
    pq, pe = _kept("q", (q, e), None, y.shape, dev)
    _check(lib().spr_act8_unpack(code, rows, width, pq, pe, _arg("rstd", rstd, torch.float32, (rows,), dev),
                                 _arg("gain", gain, y.dtype, (width,), dev), _arg("y", y, y.dtype, y.shape, dev),
                                 _on(dev, stream)))


def _gate(gate, dt, rows, width, dev):
    """Pointer of a gate [width] or [rows, width], and whether it is per row."""
    if gate is None:
        return None, 0
    per_row = 0 if gate.dim() == 1 else 1
    return _arg("gate", gate, dt, (rows, width) if per_row else (width,), dev), per_row


def block_norm_fwd(x, f, h, n, rstd_f=None, rstd_h=None, gain_post=None, gate=None, gain_pre=None,
                   residual_scale=1.0, branch_scale=1.0, eps=1e-5, h8=None, f8=None, stream=None):
    """h = residual_scale x + branch_scale gate (f r_f gain_post) and n = h r_h
    gain_pre, [rows, width] bf16 or fp32; r the rows' 1 / sqrt(mean square + eps),
    written to rstd_f and rstd_h (None: no norm on that side).  f None (and h
    None): n of x alone.  gate [width] or [rows, width]; h8, f8: (q, e) pairs
    that take h and f in 8 bits as well."""
    import torch
    s, dt, dev, f32 = x.shape, x.dtype, x.get_device(), torch.float32
    (rows, width), code = s, _storage("x", x)
    if (rows | width) >> 31:
        _fits(rows, width)
    pg, per_row = _gate(gate, dt, rows, width, dev)
    _check(lib().spr_block_norm_fwd(
        code, rows, width, float(eps), float(residual_scale), float(branch_scale), _arg("x", x, dt, s, dev),
        _arg("f", f, dt, s, dev), _arg("gain_post", gain_post, dt, (width,), dev), pg, per_row,
        _arg("gain_pre", gain_pre, dt, (width,), dev), _arg("h", h, dt, s, dev), _arg("n", n, dt, s, dev),
        _arg("rstd_f", rstd_f, f32, (rows,), dev), _arg("rstd_h", rstd_h, f32, (rows,), dev),
        *_kept("h8", h8, None, s, dev), *_kept("f8", f8, None, s, dev), _on(dev, stream)))


def block_norm_bwd_workspace_size(rows, width) -> int:
    out = c_size_t(0)
    if (rows | width) >> 31:
        _fits(rows, width)
    _check(lib().spr_block_norm_bwd_workspace_size(rows, width, byref(out)))
    return int(out.value)


def block_norm_bwd(h, f, dh, dn, dx, df=None, rstd_f=None, rstd_h=None, gain_post=None, gate=None, gain_pre=None,
                   dgain_post=None, dgate=None, dgain_pre=None, residual_scale=1.0, branch_scale=1.0,
                   overwrite=False, ws=None, stream=None):
    """Backward of block_norm_fwd from the kept h and f, each a tensor or an
    8-bit pair (q, e), and the gradients dh and dn of its outputs (either may be
    None).  dx and df are written; dgain_post, dgain_pre and the dgate of a
    shared gate, fp32 [width], added to, or written where ``overwrite``; the
    dgate of gates per row is written."""
    import torch
    s, dt, dev, f32 = dx.shape, dx.dtype, dx.get_device(), torch.float32
    (rows, width), code = s, _storage("dx", dx)
    if (rows | width) >> 31:
        _fits(rows, width)
    pg, per_row = _gate(gate, dt, rows, width, dev)
    pd = _arg("dgate", dgate, dt, s, dev) if per_row else _arg("dgate", dgate, f32, (width,), dev)
    _check(lib().spr_block_norm_bwd(
        code, rows, width, float(residual_scale), float(branch_scale), *_kept("h", h, dt, s, dev),
        *_kept("f", f, dt, s, dev), _arg("rstd_f", rstd_f, f32, (rows,), dev),
        _arg("rstd_h", rstd_h, f32, (rows,), dev), _arg("gain_post", gain_post, dt, (width,), dev), pg, per_row,
        _arg("gain_pre", gain_pre, dt, (width,), dev), _arg("dh", dh, dt, s, dev), _arg("dn", dn, dt, s, dev),
        _arg("dx", dx, dt, s, dev), _arg("df", df, dt, s, dev), _arg("dgain_post", dgain_post, f32, (width,), dev), pd,
        _arg("dgain_pre", dgain_pre, f32, (width,), dev), 1 if overwrite else 0, *_ws(ws, dev), _on(dev, stream)))


def _act_code(act):
    if act not in ACTS:
        raise ValueError(f"act {act!r}: the call takes {' or '.join(ACTS)}")
    return ACTS[act]


def glu_fwd(x, wg, wu, m, act="silu", offsets=None, row_token=None, g=None, u=None, stream=None):
    """m = act(x wg) * (x wu), bf16, in one kernel: wg, wu [in, mid] of a dense
    block, or [E, in, mid] with the experts' offsets [E + 1] (and row_token
    [rows], the rows of x that the sorted rows are).  g and u take x wg and x wu
    for the backward: tensors, or 8-bit pairs (q, e)."""
    import torch
    (e, i, o), rows, n, dev, bf, i32 = _groups(offsets, wg, "wg"), m.shape[0], x.shape[0], wg.get_device(), torch.bfloat16, torch.int32
    if (e | rows | n | i | o) >> 31:
        _fits(e, rows, n, i, o)
    s = (rows, o)
    _check(lib().spr_glu_fwd(_act_code(act), e, rows, i, o, _arg("offsets", offsets, i32, (e + 1,), dev),
                             _arg("x", x, bf, (n, i), dev), n, _arg("row_token", row_token, i32, (rows,), dev),
                             _arg("wg", wg, bf, wg.shape, dev), _arg("wu", wu, bf, wg.shape, dev),
                             _arg("m", m, bf, s, dev), *_kept("g", g, bf, s, dev), *_kept("u", u, bf, s, dev),
                             _on(dev, stream)))


def glu_bwd(dy, wd, g, u, dg, du, m=None, act="silu", offsets=None, stream=None):
    """Backward through y = m wd and m = act(g) * u: dm = dy wd^T, dg = dm u
    act'(g), du = dm act(g), and m again for wd's gradient (or None); wd [mid,
    out] or [E, mid, out]; g and u as glu_fwd kept them."""
    import torch
    (e, i, o), rows, dev, bf = _groups(offsets, wd, "wd"), dy.shape[0], wd.get_device(), torch.bfloat16
    if (e | rows | i | o) >> 31:
        _fits(e, rows, i, o)
    s = (rows, i)
    _check(lib().spr_glu_bwd(_act_code(act), e, rows, i, o, _arg("offsets", offsets, torch.int32, (e + 1,), dev),
                             _arg("dy", dy, bf, (rows, o), dev), _arg("wd", wd, bf, wd.shape, dev),
                             *_kept("g", g, bf, s, dev), *_kept("u", u, bf, s, dev), _arg("dg", dg, bf, s, dev),
                             _arg("du", du, bf, s, dev), _arg("m", m, bf, s, dev), _on(dev, stream)))


def moe_stats_bytes(n_experts: int) -> int:
    out = c_size_t(0)
    _check(lib().spr_moe_stats_bytes(n_experts, byref(out)))
    return int(out.value)


def moe_stats_zero(n_experts, stats, stream=None):
    _check(lib().spr_moe_stats_zero(n_experts, _ptr(stats), _stream(stream)))


def moe_aux_workspace_size(n_experts: int, n_tokens: int) -> int:
    out = c_size_t(0)
    _check(lib().spr_moe_aux_workspace_size(n_experts, n_tokens, byref(out)))
    return int(out.value)


def moe_aux_accumulate(n_experts, top_k, probs, experts, stats, multiplicity=1,
                       token_multiplicity=None, ws=None, stream=None):
    n = int(probs.shape[0]) if probs is not None else 0
    _check(lib().spr_moe_aux_accumulate(n_experts, top_k, n, _ptr(probs), _ptr(experts),
                                        multiplicity, _ptr(token_multiplicity), _ptr(stats),
                                        _ptr(ws), _nbytes(ws), _stream(stream)))


def moe_aux_loss(n_experts, top_k, aux_coef, stats, f, p, loss, stream=None):
    _check(lib().spr_moe_aux_loss(n_experts, top_k, float(aux_coef), _ptr(stats), _ptr(f), _ptr(p),
                                  _ptr(loss), _stream(stream)))


def moe_aux_grad(n_experts, top_k, aux_coef, upstream, stats, dprobs, multiplicity=1,
                 token_multiplicity=None, stream=None):
    n = int(dprobs.shape[0])
    _check(lib().spr_moe_aux_grad(n_experts, top_k, float(aux_coef), float(upstream), _ptr(stats), n,
                                  multiplicity, _ptr(token_multiplicity), _ptr(dprobs),
                                  _stream(stream)))


def workspace_size(op, dims, n_mb=0, max_len=0, total_len=0) -> int:
    out = c_size_t(0)
    _check(lib().spr_workspace_size(op, byref(dims), n_mb, max_len, total_len, byref(out)))
    return int(out.value)


def gkv_cache_zero(dims, gk_cache, gv_cache, stream=None):
    _Sizes(dims).cache(gk_cache=gk_cache, gv_cache=gv_cache)
    _check(lib().spr_gkv_cache_zero(byref(dims), _ptr(gk_cache), _ptr(gv_cache), _stream(stream)))


def gkv_accumulate(dims, gk_cache, gv_cache, dgk, dgv, stream=None):
    _Sizes(dims).cache(gk_cache=gk_cache, gv_cache=gv_cache, dgk=dgk, dgv=dgv)
    _check(lib().spr_gkv_accumulate(byref(dims), _ptr(gk_cache), _ptr(gv_cache), _ptr(dgk),
                                    _ptr(dgv), _stream(stream)))


def profile_enable(on: bool = True, only_kernel: str = None):
    _check(lib().spr_profile_enable(1 if on else 0,
                                    only_kernel.encode() if only_kernel else None))


def profile_reset():
    _check(lib().spr_profile_reset())


def profile_query(kernel: str):
    ms, cnt = c_double(0.0), c_int32(0)
    _check(lib().spr_profile_query(kernel.encode(), byref(ms), byref(cnt)))
    return float(ms.value), int(cnt.value)


def profile_kernels():
    n = lib().spr_profile_num_kernels()
    return [lib().spr_profile_kernel_name(i).decode() for i in range(n)]


def status_string(status: int) -> str:
    return lib().spr_status_string(status).decode()


def last_error() -> str:
    return lib().spr_last_error().decode()


def version() -> str:
    return lib().spr_version().decode()
