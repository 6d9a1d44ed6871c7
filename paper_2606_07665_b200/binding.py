"""ctypes binding of libac.so: the same entry points as include/ac.h, argument marshalling only.

Tensor arguments are torch CUDA tensors (their ``data_ptr()`` is passed through) or plain integer
addresses; ``stream`` is a ``torch.cuda.Stream``, a raw ``cudaStream_t`` integer, or None for torch's
current stream.  A non-zero status raises ``AcError``.  Nothing here computes anything: if the shared
library has not been built, loading it raises.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import c_char_p, c_double, c_float, c_int, c_int64, c_size_t, c_void_p, POINTER

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libac.so")
_lib = None

STATUS_NAMES = {0: "AC_OK", 1: "AC_ERR_NULL", 2: "AC_ERR_SHAPE", 3: "AC_ERR_UNSUPPORTED",
                4: "AC_ERR_ALIGN", 5: "AC_ERR_WORKSPACE", 6: "AC_ERR_CUDA", 7: "AC_ERR_NOT_INIT",
                8: "AC_ERR_SCRATCH_LIMIT"}
AC_FLAG_PAGE_OOB = 1
AC_FLAG_POSITION_OOB = 2
AC_FLAG_WAIT_TIMEOUT = 4
AC_FLAG_POOL_EXHAUSTED = 8
AC_FLAG_REF_COUNT = 16
AC_FLAG_ROW_OOB = 32
AC_MAX_PAGE_POOLS = 128
AC_PAGE_WHOLE = -1
AC_Q8_INT8, AC_Q8_E4M3 = 0, 1
AC_ROPE_NONE, AC_ROPE_LINEAR, AC_ROPE_BASE, AC_ROPE_RAMP = range(4)

EXPORTS = ("ac_init", "ac_status_string", "ac_last_cuda_error", "ac_sm_count", "ac_decode_plan",
           "ac_decode_plan_for_lengths",
           "ac_split_tokens", "ac_window_span", "ac_workspace_bytes", "ac_rope_kv_append", "ac_paged_decode_attn",
           "ac_splitkv_merge", "ac_decode_step_host", "ac_paged_decode_attn_static_scratch",
           "ac_fused_workspace_bytes", "ac_fused_workspace_reset", "ac_paged_decode_attn_fused_merge",
           "ac_decode_step_fused", "ac_paged_decode_attn_ex", "ac_decode_step_fused_ex",
           "ac_rope_kv_append_ex", "ac_qkv_rope_kv_append", "ac_oproj_residual_rmsnorm",
           "ac_hbm_read_probe", "ac_qkv_rope_kv_append_ex", "ac_rope_kv_append_q4", "ac_kv_store_q4",
           "ac_kv_load_q4", "ac_decode_plan_q4", "ac_paged_decode_attn_q4", "ac_rope_kv_append_q8",
           "ac_kv_store_q8", "ac_kv_load_q8", "ac_decode_plan_q8", "ac_paged_decode_attn_q8", "ac_rope_tables",
           "ac_rope_rows", "ac_cache_copy_pages",
           "ac_cache_workspace_bytes", "ac_cache_reserve", "ac_cache_fork", "ac_cache_release",
           "ac_cache_trim", "ac_cache_compact")
AC_STATIC_SCRATCH_BYTES = 8 << 20


class AcAttnOptions(ctypes.Structure):
    """Mirror of ac_attn_options."""
    _fields_ = [("window", c_int), ("fused_merge", c_int), ("row_order", c_void_p), ("rope", c_void_p),
                ("sinks", c_int), ("reserved", c_int * 1)]


class AcRopeOptions(ctypes.Structure):
    """Mirror of ac_rope_options."""
    _fields_ = [("rotary_dim", c_int), ("interleaved", c_int), ("q_norm_weight", c_void_p),
                ("k_norm_weight", c_void_p), ("norm_eps", c_float), ("reserved", c_int * 4)]


class AcQ4Cache(ctypes.Structure):
    """Mirror of ac_q4_cache (strides in bytes)."""
    _fields_ = [("k_codes", c_void_p), ("v_codes", c_void_p), ("params", c_void_p), ("stride_page", c_int64),
                ("stride_token", c_int64), ("stride_head", c_int64), ("group", c_int), ("reserved", c_int * 3)]


class AcQ8Cache(ctypes.Structure):
    """Mirror of ac_q8_cache (strides of the codes in bytes, of the scales in floats)."""
    _fields_ = [("k_codes", c_void_p), ("v_codes", c_void_p), ("scales", c_void_p), ("stride_page", c_int64),
                ("stride_token", c_int64), ("stride_head", c_int64), ("stride_scales", c_int64), ("block", c_int),
                ("format", c_int), ("reserved", c_int * 2)]


class AcRopeScaling(ctypes.Structure):
    """Mirror of ac_rope_scaling."""
    _fields_ = [("kind", c_int), ("reserved", c_int), ("base", c_double), ("factor", c_double),
                ("original", c_double), ("low", c_double), ("high", c_double), ("magnitude", c_double)]


class AcPagePool(ctypes.Structure):
    """Mirror of ac_page_pool."""
    _fields_ = [("base", c_void_p), ("page_bytes", c_int64), ("segments", c_int), ("reserved", c_int)]


class AcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().ac_status_string(status).decode()
        extra = f" (cuda error {lib().ac_last_cuda_error()})" if status == 6 else ""
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {msg}{extra}")


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded shared library; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2606_07665_b200.build`")
        L = ctypes.CDLL(_LIB_PATH)
        L.ac_init.argtypes = [c_int]
        L.ac_init.restype = c_int
        L.ac_status_string.argtypes = [c_int]
        L.ac_status_string.restype = c_char_p
        L.ac_last_cuda_error.argtypes = []
        L.ac_last_cuda_error.restype = c_int
        L.ac_sm_count.argtypes = []
        L.ac_sm_count.restype = c_int
        L.ac_decode_plan.argtypes = [c_int] * 7 + [POINTER(c_int), POINTER(c_int), POINTER(c_size_t)]
        L.ac_decode_plan.restype = c_int
        L.ac_decode_plan_for_lengths.argtypes = ([c_void_p] + [c_int] * 7 +
                                                 [POINTER(c_int), POINTER(c_int), POINTER(c_size_t)])
        L.ac_decode_plan_for_lengths.restype = c_int
        L.ac_split_tokens.argtypes = [c_int, c_int]
        L.ac_split_tokens.restype = c_int
        L.ac_window_span.argtypes = [c_int, c_int]
        L.ac_window_span.restype = c_int
        L.ac_workspace_bytes.argtypes = [c_int] * 4
        L.ac_workspace_bytes.restype = c_size_t
        L.ac_rope_kv_append.argtypes = ([c_void_p] * 6 + [c_int64] * 3 + [c_void_p, c_int, c_void_p,
                                        c_void_p, c_void_p, c_int] + [c_int] * 6 + [c_void_p, c_void_p])
        L.ac_rope_kv_append.restype = c_int
        L.ac_rope_kv_append_ex.argtypes = L.ac_rope_kv_append.argtypes + [POINTER(AcRopeOptions)]
        L.ac_rope_kv_append_ex.restype = c_int
        L.ac_qkv_rope_kv_append.argtypes = ([c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p] +
                                            [c_int64] * 3 + [c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                            c_int] + [c_int] * 6 + [c_void_p, c_void_p])
        L.ac_qkv_rope_kv_append.restype = c_int
        L.ac_qkv_rope_kv_append_ex.argtypes = L.ac_qkv_rope_kv_append.argtypes + [POINTER(AcRopeOptions)]
        L.ac_qkv_rope_kv_append_ex.restype = c_int
        L.ac_oproj_residual_rmsnorm.argtypes = [c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p, c_void_p,
                                                c_float, c_void_p, c_int, c_void_p]
        L.ac_oproj_residual_rmsnorm.restype = c_int
        L.ac_paged_decode_attn.argtypes = ([c_void_p] * 3 + [c_int64] * 3 + [c_void_p, c_int, c_void_p,
                                           c_int, c_float, c_int, c_void_p, c_size_t, c_void_p] +
                                           [c_int] * 7 + [c_void_p, c_void_p])
        L.ac_paged_decode_attn.restype = c_int
        L.ac_paged_decode_attn_fused_merge.argtypes = L.ac_paged_decode_attn.argtypes
        L.ac_paged_decode_attn_fused_merge.restype = c_int
        L.ac_fused_workspace_bytes.argtypes = [c_int] * 5
        L.ac_fused_workspace_bytes.restype = c_size_t
        L.ac_fused_workspace_reset.argtypes = [c_void_p, c_size_t] + [c_int] * 5 + [c_void_p]
        L.ac_fused_workspace_reset.restype = c_int
        L.ac_decode_step_fused.argtypes = ([c_void_p] * 6 + [c_int64] * 3 + [c_void_p, c_int, c_void_p,
                                           c_void_p, c_void_p, c_int, c_float, c_int, c_void_p, c_size_t,
                                           c_void_p] + [c_int] * 7 + [c_void_p, c_void_p])
        L.ac_decode_step_fused.restype = c_int
        L.ac_paged_decode_attn_ex.argtypes = L.ac_paged_decode_attn.argtypes + [POINTER(AcAttnOptions)]
        L.ac_paged_decode_attn_ex.restype = c_int
        L.ac_decode_step_fused_ex.argtypes = L.ac_decode_step_fused.argtypes + [POINTER(AcAttnOptions)]
        L.ac_decode_step_fused_ex.restype = c_int
        L.ac_splitkv_merge.argtypes = [c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]
        L.ac_splitkv_merge.restype = c_int
        L.ac_decode_step_host.argtypes = ([c_void_p] * 6 + [c_void_p] * 6 + [c_void_p] * 2 + [c_int64] * 3 +
                                          [c_int, c_void_p, c_void_p, c_int, c_float, c_int, c_void_p,
                                           c_size_t] + [c_int] * 7 + [c_void_p, c_void_p])
        L.ac_decode_step_host.restype = c_int
        L.ac_paged_decode_attn_static_scratch.argtypes = ([c_void_p] * 3 + [c_int64] * 3 + [c_void_p, c_int,
                                                          c_void_p, c_int, c_float, c_int, c_void_p] +
                                                          [c_int] * 7 + [c_void_p, c_void_p])
        L.ac_paged_decode_attn_static_scratch.restype = c_int
        L.ac_hbm_read_probe.argtypes = [c_void_p, c_size_t, c_void_p, c_void_p]
        L.ac_hbm_read_probe.restype = c_int
        L.ac_rope_kv_append_q4.argtypes = ([c_void_p] * 4 + [POINTER(AcQ4Cache), c_void_p, c_int, c_void_p,
                                           c_void_p, c_void_p, c_int] + [c_int] * 6 +
                                           [c_void_p, c_void_p, POINTER(AcRopeOptions)])
        L.ac_rope_kv_append_q4.restype = c_int
        L.ac_kv_store_q4.argtypes = ([c_void_p] * 2 + [POINTER(AcQ4Cache), c_void_p, c_int, c_void_p, c_void_p,
                                     c_int] + [c_int] * 5 + [c_void_p, c_void_p])
        L.ac_kv_store_q4.restype = c_int
        L.ac_kv_load_q4.argtypes = L.ac_kv_store_q4.argtypes
        L.ac_kv_load_q4.restype = c_int
        L.ac_decode_plan_q4.argtypes = L.ac_decode_plan_for_lengths.argtypes
        L.ac_decode_plan_q4.restype = c_int
        L.ac_paged_decode_attn_q4.argtypes = ([c_void_p, POINTER(AcQ4Cache), c_void_p, c_int, c_void_p, c_int,
                                              c_float, c_int, c_void_p, c_size_t, c_void_p] + [c_int] * 7 +
                                              [c_void_p, c_void_p, POINTER(AcAttnOptions)])
        L.ac_paged_decode_attn_q4.restype = c_int
        q8 = {POINTER(AcQ4Cache): POINTER(AcQ8Cache)}
        for name in ("ac_rope_kv_append", "ac_kv_store", "ac_kv_load", "ac_decode_plan", "ac_paged_decode_attn"):
            fn = getattr(L, name + "_q8")                  # the calls of the 4-bit cache with the other descriptor
            fn.argtypes = [q8.get(t, t) for t in getattr(L, name + "_q4").argtypes]
            fn.restype = c_int
        L.ac_rope_tables.argtypes = [c_void_p, c_void_p, c_int64, c_int, c_int, POINTER(AcRopeScaling), c_void_p]
        L.ac_rope_tables.restype = c_int
        L.ac_rope_rows.argtypes = ([c_void_p, c_void_p, c_int64, c_int64] * 2 + [c_void_p, c_void_p] + [c_int] * 5 +
                                   [c_void_p, c_void_p, c_int, c_void_p, c_void_p, POINTER(AcRopeOptions)])
        L.ac_rope_rows.restype = c_int
        L.ac_cache_copy_pages.argtypes = [POINTER(AcPagePool), c_int, c_void_p, c_int, c_int, c_void_p, c_void_p]
        L.ac_cache_copy_pages.restype = c_int
        L.ac_cache_workspace_bytes.argtypes = [c_int] * 3
        L.ac_cache_workspace_bytes.restype = c_size_t
        L.ac_cache_reserve.argtypes = [c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p,
                                       c_size_t, c_void_p, c_void_p]
        L.ac_cache_reserve.restype = c_int
        L.ac_cache_fork.argtypes = [POINTER(AcPagePool), c_int, c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                    c_int, c_int, c_int, c_int, c_void_p, c_size_t, c_void_p, c_void_p]
        L.ac_cache_fork.restype = c_int
        L.ac_cache_release.argtypes = [c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int,
                                       c_void_p, c_void_p]
        L.ac_cache_release.restype = c_int
        L.ac_cache_trim.argtypes = [c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p]
        L.ac_cache_trim.restype = c_int
        L.ac_cache_compact.argtypes = [POINTER(AcPagePool), c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                                       c_void_p, c_int, c_int, c_int, c_void_p, c_void_p, c_size_t, c_void_p,
                                       c_void_p]
        L.ac_cache_compact.restype = c_int
        _lib = L
    return _lib


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, where: str) -> None:
    if status != 0:
        raise AcError(status, where)


def ac_init(device: int = -1) -> None:
    _check(lib().ac_init(device), "ac_init")


def ac_sm_count() -> int:
    return lib().ac_sm_count()


def ac_split_tokens(max_context_len: int, num_splits: int) -> int:
    return lib().ac_split_tokens(max_context_len, num_splits)


def ac_window_span(window: int, sinks: int = 0) -> int:
    return lib().ac_window_span(window, sinks)


def ac_workspace_bytes(B: int, Hq: int, d: int, num_splits: int) -> int:
    return lib().ac_workspace_bytes(B, Hq, d, num_splits)


def ac_decode_plan(B, Hq, Hkv, d, page_size, max_context_len, sm_count=0):
    """Returns (num_splits, split_tokens, workspace_bytes)."""
    ns, st, wb = c_int(0), c_int(0), c_size_t(0)
    _check(lib().ac_decode_plan(B, Hq, Hkv, d, page_size, max_context_len, sm_count,
                                ctypes.byref(ns), ctypes.byref(st), ctypes.byref(wb)), "ac_decode_plan")
    return ns.value, st.value, wb.value


def ac_decode_plan_for_lengths(token_counts, Hq, Hkv, d, page_size, max_context_len, sm_count=0):
    """token_counts: host sequence of B ints (tokens each row attends over; <= 0 = inactive row).
    Returns (num_splits, split_tokens, workspace_bytes)."""
    counts = (ctypes.c_int32 * len(token_counts))(*[int(t) for t in token_counts])
    ns, st, wb = c_int(0), c_int(0), c_size_t(0)
    _check(lib().ac_decode_plan_for_lengths(ctypes.cast(counts, c_void_p), len(token_counts), Hq, Hkv, d,
                                            page_size, max_context_len, sm_count, ctypes.byref(ns),
                                            ctypes.byref(st), ctypes.byref(wb)),
           "ac_decode_plan_for_lengths")
    return ns.value, st.value, wb.value


def ac_rope_kv_append(q_in, q_out, k_new, v_new, k_cache, v_cache, stride_page, stride_token,
                      stride_head, block_table, max_pages_per_seq, context_lens, rope_cos, rope_sin,
                      max_position, B, Hq, Hkv, d, page_size, num_pages, status_flag=None, stream=None):
    _check(lib().ac_rope_kv_append(_ptr(q_in), _ptr(q_out), _ptr(k_new), _ptr(v_new), _ptr(k_cache),
                                   _ptr(v_cache), stride_page, stride_token, stride_head,
                                   _ptr(block_table), max_pages_per_seq, _ptr(context_lens),
                                   _ptr(rope_cos), _ptr(rope_sin), max_position, B, Hq, Hkv, d,
                                   page_size, num_pages, _ptr(status_flag), _stream(stream)),
           "ac_rope_kv_append")


def ac_rope_kv_append_ex(q_in, q_out, k_new, v_new, k_cache, v_cache, stride_page, stride_token,
                         stride_head, block_table, max_pages_per_seq, context_lens, rope_cos, rope_sin,
                         max_position, B, Hq, Hkv, d, page_size, num_pages, status_flag=None, stream=None,
                         rotary_dim=0, interleaved=False, q_norm_weight=None, k_norm_weight=None,
                         norm_eps=0.0):
    opt = _rope_options(rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps)
    _check(lib().ac_rope_kv_append_ex(_ptr(q_in), _ptr(q_out), _ptr(k_new), _ptr(v_new), _ptr(k_cache),
                                      _ptr(v_cache), stride_page, stride_token, stride_head,
                                      _ptr(block_table), max_pages_per_seq, _ptr(context_lens),
                                      _ptr(rope_cos), _ptr(rope_sin), max_position, B, Hq, Hkv, d,
                                      page_size, num_pages, _ptr(status_flag), _stream(stream),
                                      ctypes.byref(opt)), "ac_rope_kv_append_ex")


def ac_qkv_rope_kv_append(x, w_qkv, H, q_out, k_cache, v_cache, stride_page, stride_token, stride_head,
                          block_table, max_pages_per_seq, context_lens, rope_cos, rope_sin, max_position,
                          B, Hq, Hkv, d, page_size, num_pages, status_flag=None, stream=None):
    _check(lib().ac_qkv_rope_kv_append(_ptr(x), _ptr(w_qkv), H, _ptr(q_out), _ptr(k_cache), _ptr(v_cache),
                                       stride_page, stride_token, stride_head, _ptr(block_table),
                                       max_pages_per_seq, _ptr(context_lens), _ptr(rope_cos),
                                       _ptr(rope_sin), max_position, B, Hq, Hkv, d, page_size, num_pages,
                                       _ptr(status_flag), _stream(stream)), "ac_qkv_rope_kv_append")


def ac_qkv_rope_kv_append_ex(x, w_qkv, H, q_out, k_cache, v_cache, stride_page, stride_token, stride_head,
                             block_table, max_pages_per_seq, context_lens, rope_cos, rope_sin, max_position,
                             B, Hq, Hkv, d, page_size, num_pages, status_flag=None, stream=None,
                             rotary_dim=0, interleaved=False, q_norm_weight=None, k_norm_weight=None,
                             norm_eps=0.0):
    opt = _rope_options(rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps)
    _check(lib().ac_qkv_rope_kv_append_ex(_ptr(x), _ptr(w_qkv), H, _ptr(q_out), _ptr(k_cache), _ptr(v_cache),
                                          stride_page, stride_token, stride_head, _ptr(block_table),
                                          max_pages_per_seq, _ptr(context_lens), _ptr(rope_cos),
                                          _ptr(rope_sin), max_position, B, Hq, Hkv, d, page_size, num_pages,
                                          _ptr(status_flag), _stream(stream), ctypes.byref(opt)),
           "ac_qkv_rope_kv_append_ex")


def ac_oproj_residual_rmsnorm(attn_out, w_o, K, N, residual_in, residual_out, norm_weight, norm_eps,
                              normed_out, B, stream=None):
    _check(lib().ac_oproj_residual_rmsnorm(_ptr(attn_out), _ptr(w_o), K, N, _ptr(residual_in),
                                           _ptr(residual_out), _ptr(norm_weight), norm_eps,
                                           _ptr(normed_out), B, _stream(stream)),
           "ac_oproj_residual_rmsnorm")


def ac_paged_decode_attn(q_rot, k_cache, v_cache, stride_page, stride_token, stride_head, block_table,
                         max_pages_per_seq, context_lens, new_tokens, softmax_scale, num_splits,
                         workspace, workspace_bytes, out, B, Hq, Hkv, d, page_size, num_pages,
                         max_context_len, status_flag=None, stream=None):
    _check(lib().ac_paged_decode_attn(_ptr(q_rot), _ptr(k_cache), _ptr(v_cache), stride_page,
                                      stride_token, stride_head, _ptr(block_table), max_pages_per_seq,
                                      _ptr(context_lens), new_tokens, softmax_scale, num_splits,
                                      _ptr(workspace), workspace_bytes, _ptr(out), B, Hq, Hkv, d,
                                      page_size, num_pages, max_context_len, _ptr(status_flag),
                                      _stream(stream)), "ac_paged_decode_attn")


def ac_fused_workspace_bytes(B: int, Hq: int, Hkv: int, d: int, num_splits: int) -> int:
    return lib().ac_fused_workspace_bytes(B, Hq, Hkv, d, num_splits)


def ac_fused_workspace_reset(workspace, workspace_bytes, B, Hq, Hkv, d, num_splits, stream=None):
    _check(lib().ac_fused_workspace_reset(_ptr(workspace), workspace_bytes, B, Hq, Hkv, d, num_splits,
                                          _stream(stream)), "ac_fused_workspace_reset")


def ac_paged_decode_attn_fused_merge(q_rot, k_cache, v_cache, stride_page, stride_token, stride_head,
                                     block_table, max_pages_per_seq, context_lens, new_tokens,
                                     softmax_scale, num_splits, workspace, workspace_bytes, out, B, Hq,
                                     Hkv, d, page_size, num_pages, max_context_len, status_flag=None,
                                     stream=None):
    _check(lib().ac_paged_decode_attn_fused_merge(
        _ptr(q_rot), _ptr(k_cache), _ptr(v_cache), stride_page, stride_token, stride_head,
        _ptr(block_table), max_pages_per_seq, _ptr(context_lens), new_tokens, softmax_scale, num_splits,
        _ptr(workspace), workspace_bytes, _ptr(out), B, Hq, Hkv, d, page_size, num_pages,
        max_context_len, _ptr(status_flag), _stream(stream)), "ac_paged_decode_attn_fused_merge")


def ac_decode_step_fused(q_in, q_rot_out, k_new, v_new, k_cache, v_cache, stride_page, stride_token,
                         stride_head, block_table, max_pages_per_seq, context_lens, rope_cos, rope_sin,
                         max_position, softmax_scale, num_splits, workspace, workspace_bytes, out, B, Hq,
                         Hkv, d, page_size, num_pages, max_context_len, status_flag=None, stream=None):
    _check(lib().ac_decode_step_fused(
        _ptr(q_in), _ptr(q_rot_out), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), stride_page,
        stride_token, stride_head, _ptr(block_table), max_pages_per_seq, _ptr(context_lens),
        _ptr(rope_cos), _ptr(rope_sin), max_position, softmax_scale, num_splits, _ptr(workspace),
        workspace_bytes, _ptr(out), B, Hq, Hkv, d, page_size, num_pages, max_context_len,
        _ptr(status_flag), _stream(stream)), "ac_decode_step_fused")


def _rope_options(rotary_dim=0, interleaved=False, q_norm_weight=None, k_norm_weight=None, norm_eps=0.0):
    opt = AcRopeOptions()
    opt.rotary_dim = int(rotary_dim)
    opt.interleaved = 1 if interleaved else 0
    opt.q_norm_weight = _ptr(q_norm_weight)
    opt.k_norm_weight = _ptr(k_norm_weight)
    opt.norm_eps = float(norm_eps)
    return opt


def _options(window: int = 0, fused_merge: bool = False, row_order=None, rope=None, sinks: int = 0):
    """rope: an AcRopeOptions instance (kept alive by the returned structure) or None."""
    opt = AcAttnOptions()
    opt.window = int(window)
    opt.fused_merge = 1 if fused_merge else 0
    opt.row_order = _ptr(row_order)
    opt.sinks = int(sinks)
    opt.rope = ctypes.addressof(rope) if rope is not None else None
    opt._keep = rope
    return opt


def ac_paged_decode_attn_ex(q_rot, k_cache, v_cache, stride_page, stride_token, stride_head, block_table,
                            max_pages_per_seq, context_lens, new_tokens, softmax_scale, num_splits,
                            workspace, workspace_bytes, out, B, Hq, Hkv, d, page_size, num_pages,
                            max_context_len, status_flag=None, stream=None, window=0, fused_merge=False,
                            row_order=None, sinks=0):
    _check(lib().ac_paged_decode_attn_ex(
        _ptr(q_rot), _ptr(k_cache), _ptr(v_cache), stride_page, stride_token, stride_head,
        _ptr(block_table), max_pages_per_seq, _ptr(context_lens), new_tokens, softmax_scale, num_splits,
        _ptr(workspace), workspace_bytes, _ptr(out), B, Hq, Hkv, d, page_size, num_pages,
        max_context_len, _ptr(status_flag), _stream(stream),
        ctypes.byref(_options(window, fused_merge, row_order, sinks=sinks))), "ac_paged_decode_attn_ex")


def ac_decode_step_fused_ex(q_in, q_rot_out, k_new, v_new, k_cache, v_cache, stride_page, stride_token,
                            stride_head, block_table, max_pages_per_seq, context_lens, rope_cos, rope_sin,
                            max_position, softmax_scale, num_splits, workspace, workspace_bytes, out, B,
                            Hq, Hkv, d, page_size, num_pages, max_context_len, status_flag=None,
                            stream=None, window=0, row_order=None, rotary_dim=0, interleaved=False,
                            q_norm_weight=None, k_norm_weight=None, norm_eps=0.0, sinks=0):
    """The rope keywords are those of ac_rope_kv_append_ex (all default = the plain rotation)."""
    variants = rotary_dim or interleaved or q_norm_weight is not None or k_norm_weight is not None
    rope = _rope_options(rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps) if variants else None
    opt = _options(window, False, row_order, rope, sinks)
    _check(lib().ac_decode_step_fused_ex(
        _ptr(q_in), _ptr(q_rot_out), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), stride_page,
        stride_token, stride_head, _ptr(block_table), max_pages_per_seq, _ptr(context_lens),
        _ptr(rope_cos), _ptr(rope_sin), max_position, softmax_scale, num_splits, _ptr(workspace),
        workspace_bytes, _ptr(out), B, Hq, Hkv, d, page_size, num_pages, max_context_len,
        _ptr(status_flag), _stream(stream), ctypes.byref(opt)), "ac_decode_step_fused_ex")


def ac_splitkv_merge(workspace, num_splits, context_lens, out, B, Hq, d, stream=None):
    _check(lib().ac_splitkv_merge(_ptr(workspace), num_splits, _ptr(context_lens), _ptr(out), B, Hq, d,
                                  _stream(stream)), "ac_splitkv_merge")


def ac_decode_step_host(q_host, k_new_host, v_new_host, block_table_host, context_lens_host, out_host,
                        q, k_new, v_new, block_table, context_lens, out, k_cache, v_cache, stride_page,
                        stride_token, stride_head, max_pages_per_seq, rope_cos, rope_sin, max_position,
                        softmax_scale, num_splits, workspace, workspace_bytes, B, Hq, Hkv, d, page_size,
                        num_pages, max_context_len, status_flag=None, stream=None):
    _check(lib().ac_decode_step_host(_ptr(q_host), _ptr(k_new_host), _ptr(v_new_host),
                                     _ptr(block_table_host), _ptr(context_lens_host), _ptr(out_host),
                                     _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(block_table),
                                     _ptr(context_lens), _ptr(out), _ptr(k_cache), _ptr(v_cache),
                                     stride_page, stride_token, stride_head, max_pages_per_seq,
                                     _ptr(rope_cos), _ptr(rope_sin), max_position, softmax_scale,
                                     num_splits, _ptr(workspace), workspace_bytes, B, Hq, Hkv, d,
                                     page_size, num_pages, max_context_len, _ptr(status_flag),
                                     _stream(stream)), "ac_decode_step_host")


def ac_paged_decode_attn_static_scratch(q_rot, k_cache, v_cache, stride_page, stride_token, stride_head,
                                        block_table, max_pages_per_seq, context_lens, new_tokens,
                                        softmax_scale, num_splits, out, B, Hq, Hkv, d, page_size,
                                        num_pages, max_context_len, status_flag=None, stream=None):
    """Attention + merge with the split partials in the library's built-in array (no workspace
    argument, no allocation anywhere in the call); see include/ac.h for the size limit and rules."""
    _check(lib().ac_paged_decode_attn_static_scratch(
        _ptr(q_rot), _ptr(k_cache), _ptr(v_cache), stride_page, stride_token, stride_head,
        _ptr(block_table), max_pages_per_seq, _ptr(context_lens), new_tokens, softmax_scale, num_splits,
        _ptr(out), B, Hq, Hkv, d, page_size, num_pages, max_context_len, _ptr(status_flag),
        _stream(stream)), "ac_paged_decode_attn_static_scratch")


def ac_hbm_read_probe(buffer, nbytes, sink=None, stream=None):
    """Enqueues one read-only pass over ``buffer`` (calibration; the caller times it)."""
    _check(lib().ac_hbm_read_probe(_ptr(buffer), nbytes, _ptr(sink), _stream(stream)), "ac_hbm_read_probe")


# ---- the 4-bit cache ---------------------------------------------------------------------------------------


def q4_cache(k_codes, v_codes, params, stride_page, stride_token, stride_head, group) -> AcQ4Cache:
    """The descriptor of a 4-bit cache; strides in bytes.  The tensors must outlive it."""
    return AcQ4Cache(_ptr(k_codes), _ptr(v_codes), _ptr(params), stride_page, stride_token, stride_head, group)


def ac_rope_kv_append_q4(q_in, q_out, k_new, v_new, cache, block_table, max_pages_per_seq, context_lens,
                         rope_cos, rope_sin, max_position, B, Hq, Hkv, d, page_size, num_pages,
                         status_flag=None, stream=None, rotary_dim=0, interleaved=False, q_norm_weight=None,
                         k_norm_weight=None, norm_eps=0.0):
    opt = _rope_options(rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps)
    _check(lib().ac_rope_kv_append_q4(_ptr(q_in), _ptr(q_out), _ptr(k_new), _ptr(v_new), cache,
                                      _ptr(block_table), max_pages_per_seq, _ptr(context_lens), _ptr(rope_cos),
                                      _ptr(rope_sin), max_position, B, Hq, Hkv, d, page_size, num_pages,
                                      _ptr(status_flag), _stream(stream), ctypes.byref(opt)),
           "ac_rope_kv_append_q4")


def ac_kv_store_q4(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv, d,
                   page_size, num_pages, status_flag=None, stream=None):
    _check(lib().ac_kv_store_q4(_ptr(k), _ptr(v), cache, _ptr(block_table), max_pages_per_seq, _ptr(start_pos),
                                _ptr(row_offsets), total_tokens, B, Hkv, d, page_size, num_pages,
                                _ptr(status_flag), _stream(stream)), "ac_kv_store_q4")


def ac_kv_load_q4(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv, d,
                  page_size, num_pages, status_flag=None, stream=None):
    _check(lib().ac_kv_load_q4(_ptr(k), _ptr(v), cache, _ptr(block_table), max_pages_per_seq, _ptr(start_pos),
                               _ptr(row_offsets), total_tokens, B, Hkv, d, page_size, num_pages,
                               _ptr(status_flag), _stream(stream)), "ac_kv_load_q4")


def _plan_quantised(name, token_counts, B, Hq, Hkv, d, page_size, max_context_len, sm_count):
    counts = None
    if token_counts is not None:
        if len(token_counts) != B:
            raise ValueError(f"{len(token_counts)} token counts for {B} rows")
        counts = ctypes.cast((ctypes.c_int32 * B)(*[int(t) for t in token_counts]), c_void_p)
    ns, st, wb = c_int(0), c_int(0), c_size_t(0)
    _check(getattr(lib(), name)(counts, B, Hq, Hkv, d, page_size, max_context_len, sm_count,
                                ctypes.byref(ns), ctypes.byref(st), ctypes.byref(wb)), name)
    return ns.value, st.value, wb.value


def ac_decode_plan_q4(token_counts, B, Hq, Hkv, d, page_size, max_context_len, sm_count=0):
    """token_counts: host sequence of B ints or None.  Returns (num_splits, split_tokens, workspace_bytes)."""
    return _plan_quantised("ac_decode_plan_q4", token_counts, B, Hq, Hkv, d, page_size, max_context_len, sm_count)


def ac_paged_decode_attn_q4(q_rot, cache, block_table, max_pages_per_seq, context_lens, new_tokens, softmax_scale,
                            num_splits, workspace, workspace_bytes, out, B, Hq, Hkv, d, page_size, num_pages,
                            max_context_len, status_flag=None, stream=None, window=0, sinks=0, row_order=None):
    _check(lib().ac_paged_decode_attn_q4(
        _ptr(q_rot), cache, _ptr(block_table), max_pages_per_seq, _ptr(context_lens), new_tokens, softmax_scale,
        num_splits, _ptr(workspace), workspace_bytes, _ptr(out), B, Hq, Hkv, d, page_size, num_pages,
        max_context_len, _ptr(status_flag), _stream(stream),
        ctypes.byref(_options(window, True, row_order, sinks=sinks))), "ac_paged_decode_attn_q4")


# ---- the 8-bit cache ---------------------------------------------------------------------------------------


def q8_cache(k_codes, v_codes, scales, stride_page, stride_token, stride_head, stride_scales, block, fmt) -> AcQ8Cache:
    """The descriptor of an 8-bit cache; strides of the codes in bytes, of the scales in floats.  The tensors must outlive it."""
    return AcQ8Cache(_ptr(k_codes), _ptr(v_codes), _ptr(scales), stride_page, stride_token, stride_head, stride_scales, block,
                     fmt)


def ac_rope_kv_append_q8(q_in, q_out, k_new, v_new, cache, block_table, max_pages_per_seq, context_lens,
                         rope_cos, rope_sin, max_position, B, Hq, Hkv, d, page_size, num_pages,
                         status_flag=None, stream=None, rotary_dim=0, interleaved=False, q_norm_weight=None,
                         k_norm_weight=None, norm_eps=0.0):
    opt = _rope_options(rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps)
    _check(lib().ac_rope_kv_append_q8(_ptr(q_in), _ptr(q_out), _ptr(k_new), _ptr(v_new), cache,
                                      _ptr(block_table), max_pages_per_seq, _ptr(context_lens), _ptr(rope_cos),
                                      _ptr(rope_sin), max_position, B, Hq, Hkv, d, page_size, num_pages,
                                      _ptr(status_flag), _stream(stream), ctypes.byref(opt)),
           "ac_rope_kv_append_q8")


def ac_kv_store_q8(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv, d,
                   page_size, num_pages, status_flag=None, stream=None):
    _check(lib().ac_kv_store_q8(_ptr(k), _ptr(v), cache, _ptr(block_table), max_pages_per_seq, _ptr(start_pos),
                                _ptr(row_offsets), total_tokens, B, Hkv, d, page_size, num_pages,
                                _ptr(status_flag), _stream(stream)), "ac_kv_store_q8")


def ac_kv_load_q8(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv, d,
                  page_size, num_pages, status_flag=None, stream=None):
    _check(lib().ac_kv_load_q8(_ptr(k), _ptr(v), cache, _ptr(block_table), max_pages_per_seq, _ptr(start_pos),
                               _ptr(row_offsets), total_tokens, B, Hkv, d, page_size, num_pages,
                               _ptr(status_flag), _stream(stream)), "ac_kv_load_q8")


def ac_decode_plan_q8(token_counts, B, Hq, Hkv, d, page_size, max_context_len, sm_count=0):
    """token_counts: host sequence of B ints or None.  Returns (num_splits, split_tokens, workspace_bytes)."""
    return _plan_quantised("ac_decode_plan_q8", token_counts, B, Hq, Hkv, d, page_size, max_context_len, sm_count)


def ac_paged_decode_attn_q8(q_rot, cache, block_table, max_pages_per_seq, context_lens, new_tokens, softmax_scale,
                            num_splits, workspace, workspace_bytes, out, B, Hq, Hkv, d, page_size, num_pages,
                            max_context_len, status_flag=None, stream=None, window=0, row_order=None, sinks=0):
    _check(lib().ac_paged_decode_attn_q8(
        _ptr(q_rot), cache, _ptr(block_table), max_pages_per_seq, _ptr(context_lens), new_tokens,
        softmax_scale, num_splits, _ptr(workspace), workspace_bytes, _ptr(out), B, Hq, Hkv, d, page_size, num_pages,
        max_context_len, _ptr(status_flag), _stream(stream),
        ctypes.byref(_options(window, True, row_order, sinks=sinks))), "ac_paged_decode_attn_q8")


# ---- rotary positions --------------------------------------------------------------------------------------


def rope_scaling(base=10000.0, kind=AC_ROPE_NONE, factor=1.0, original=0.0, low=0.0, high=0.0, magnitude=0.0) -> AcRopeScaling:
    return AcRopeScaling(kind, 0, base, factor, original, low, high, magnitude)


def ac_rope_tables(rope_cos, rope_sin, first_position, positions, rotary_dim, scaling, stream=None):
    _check(lib().ac_rope_tables(_ptr(rope_cos), _ptr(rope_sin), first_position, positions, rotary_dim,
                                ctypes.byref(scaling), _stream(stream)), "ac_rope_tables")


def ac_rope_rows(q_in, q_out, stride_q_in_token, stride_q_out_token, k_in, k_out, stride_k_in_token, stride_k_out_token,
                 start_pos, row_offsets, total_tokens, B, Hq, Hkv, d, rope_cos, rope_sin, max_position, status_flag=None,
                 stream=None, rotary_dim=0, interleaved=False, q_norm_weight=None, k_norm_weight=None, norm_eps=0.0):
    opt = _rope_options(rotary_dim, interleaved, q_norm_weight, k_norm_weight, norm_eps)
    _check(lib().ac_rope_rows(_ptr(q_in), _ptr(q_out), stride_q_in_token, stride_q_out_token, _ptr(k_in), _ptr(k_out),
                              stride_k_in_token, stride_k_out_token, _ptr(start_pos), _ptr(row_offsets), total_tokens, B,
                              Hq, Hkv, d, _ptr(rope_cos), _ptr(rope_sin), max_position, _ptr(status_flag),
                              _stream(stream), ctypes.byref(opt)), "ac_rope_rows")


# ---- pages -------------------------------------------------------------------------------------------------


def page_pools(pools):
    """``pools``: sequence of (tensor or address, page_bytes, segments[, whole]) -> a ctypes array of ac_page_pool; whole stands for
    AC_PAGE_WHOLE segments."""
    return (AcPagePool * max(1, len(pools)))(*[AcPagePool(_ptr(base), page_bytes, AC_PAGE_WHOLE if any(whole) else segments, 0)
                                               for base, page_bytes, segments, *whole in pools])


def ac_cache_copy_pages(pools, n_pools, pairs, n, num_pages, status_flag=None, stream=None):
    _check(lib().ac_cache_copy_pages(pools, n_pools, _ptr(pairs), n, num_pages, _ptr(status_flag),
                                     _stream(stream)), "ac_cache_copy_pages")


def ac_cache_workspace_bytes(rows: int, num_pages: int, n: int) -> int:
    return lib().ac_cache_workspace_bytes(rows, num_pages, n)


def ac_cache_reserve(block_table, max_pages_per_seq, context_lens, ref_counts, new_tokens, rows, page_size,
                     num_pages, workspace, workspace_bytes, status_flag=None, stream=None):
    _check(lib().ac_cache_reserve(_ptr(block_table), max_pages_per_seq, _ptr(context_lens), _ptr(ref_counts),
                                  new_tokens, rows, page_size, num_pages, _ptr(workspace), workspace_bytes,
                                  _ptr(status_flag), _stream(stream)), "ac_cache_reserve")


def ac_cache_fork(pools, n_pools, block_table, max_pages_per_seq, context_lens, ref_counts, pairs, n, rows,
                  page_size, num_pages, workspace, workspace_bytes, status_flag=None, stream=None):
    _check(lib().ac_cache_fork(pools, n_pools, _ptr(block_table), max_pages_per_seq, _ptr(context_lens),
                               _ptr(ref_counts), _ptr(pairs), n, rows, page_size, num_pages, _ptr(workspace),
                               workspace_bytes, _ptr(status_flag), _stream(stream)), "ac_cache_fork")


def ac_cache_release(block_table, max_pages_per_seq, context_lens, ref_counts, row_list, n, rows, page_size,
                     num_pages, status_flag=None, stream=None):
    _check(lib().ac_cache_release(_ptr(block_table), max_pages_per_seq, _ptr(context_lens), _ptr(ref_counts),
                                  _ptr(row_list), n, rows, page_size, num_pages, _ptr(status_flag),
                                  _stream(stream)), "ac_cache_release")


def ac_cache_trim(block_table, max_pages_per_seq, context_lens, ref_counts, rows, page_size, num_pages,
                  status_flag=None, stream=None):
    _check(lib().ac_cache_trim(_ptr(block_table), max_pages_per_seq, _ptr(context_lens), _ptr(ref_counts), rows,
                               page_size, num_pages, _ptr(status_flag), _stream(stream)), "ac_cache_trim")


def ac_cache_compact(pools, n_pools, block_table, block_table_out, max_pages_per_seq, context_lens, ref_counts,
                     ref_counts_out, rows, page_size, num_pages, live_out, workspace, workspace_bytes,
                     status_flag=None, stream=None):
    _check(lib().ac_cache_compact(pools, n_pools, _ptr(block_table), _ptr(block_table_out), max_pages_per_seq,
                                  _ptr(context_lens), _ptr(ref_counts), _ptr(ref_counts_out), rows, page_size,
                                  num_pages, _ptr(live_out), _ptr(workspace), workspace_bytes,
                                  _ptr(status_flag), _stream(stream)), "ac_cache_compact")
