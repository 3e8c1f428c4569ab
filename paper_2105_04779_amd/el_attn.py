"""Thin Python binding of the C ABI in include/el_attn.h (argument marshalling only).

Every step of the decode path runs in the HIP library; torch is used for device
memory and the stream handle, nothing else.  Loading fails loudly when the
library has not been built -- there is no CPU fallback.
"""
from __future__ import annotations

import collections
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libelattn.so")

EL_OK, EL_ERR_INVALID_ARG, EL_ERR_UNSUPPORTED, EL_ERR_ALLOC, EL_ERR_HIP, EL_ERR_WORKSPACE = range(6)
EL_F32, EL_F16, EL_BF16 = 0, 1, 2
EL_E4M3, EL_INT8 = 1, 2
EL_FLAG_FORCE_GENERIC = 1

DTYPE_CODES = {"f32": EL_F32, "f16": EL_F16, "bf16": EL_BF16}

EXPORTED_SYMBOLS = (
    "el_attn_prepare", "el_attn_workspace_bytes", "el_attn_bind_workspace", "el_attn_decode_step",
    "el_attn_expand_query", "el_attn_set_splits", "el_attn_max_splits", "el_attn_set_row_groups",
    "el_attn_uses_mfma", "el_attn_plan_preview", "el_attn_plan_short_core", "el_attn_plan_step", "el_attn_check_step_operands",
    "el_attn_decode_step_static",
    "el_attn_core_timing_enable", "el_attn_core_timing_read",
    "el_attn_gather_batch", "el_attn_check_inputs",
    "el_attn_decode_segment", "el_attn_merge_segments", "el_attn_max_segments",
    "el_attn_paged_workspace_bytes", "el_attn_paged_attend", "el_attn_paged_append", "el_attn_paged_copy",
    "el_attn_max_alternatives", "el_attn_score_workspace_bytes", "el_attn_score_tokens",
    "el_attn_quantized_workspace_bytes", "el_attn_quantized_attend", "el_attn_quantized_append", "el_attn_quantized_copy",
    "el_attn_plan_workspace_bytes", "el_attn_plan_pages", "el_attn_plan_pages_exclusive", "el_attn_sample_workspace_bytes", "el_attn_sample_tokens",
    "el_attn_destroy", "el_attn_status_string", "el_attn_version",
)


class ElAttnConfig(ctypes.Structure):
    _fields_ = [
        ("heads", ctypes.c_int32), ("d_model", ctypes.c_int32), ("d_k", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
        ("max_batch", ctypes.c_int32), ("max_beam", ctypes.c_int32), ("max_n", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
    ]


class ElAttnPages(ctypes.Structure):
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p),
        ("page_stride", ctypes.c_int64), ("position_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32), ("d_head", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
    ]


class ElAttnScoreRule(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("window", ctypes.c_int32),
                ("slopes", ctypes.c_void_p)]


class ElAttnPages8(ctypes.Structure):
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("K_scale", ctypes.c_void_p), ("V_scale", ctypes.c_void_p),
        ("page_stride", ctypes.c_int64), ("position_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("d_head", ctypes.c_int32),
        ("block", ctypes.c_int32), ("format", ctypes.c_int32),
    ]


class ElAttnSampleRule(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("top_k", ctypes.c_int32), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("row_temperature", ctypes.c_void_p), ("row_top_k", ctypes.c_void_p), ("row_top_p", ctypes.c_void_p), ("row_min_p", ctypes.c_void_p)]


class ElAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2105_04779_amd.build` "
            "(or __graft_entry__.build()); there is no fallback path.")
    # PyTorch ships a HIP runtime of its own.  The tensors this binding is handed live in that runtime, so it has to
    # be in the process before the library is loaded: loaded the other way round, the library binds to the system's
    # copy and the two runtimes then disagree about the device ("no ROCm-capable device", crashes).
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.el_attn_prepare.argtypes = [ctypes.POINTER(ElAttnConfig)] + [vp] * 8 + [vp, ctypes.POINTER(vp)]
    lib.el_attn_prepare.restype = ctypes.c_int
    lib.el_attn_workspace_bytes.argtypes = [vp]
    lib.el_attn_workspace_bytes.restype = sz
    lib.el_attn_bind_workspace.argtypes = [vp, vp, sz]
    lib.el_attn_bind_workspace.restype = ctypes.c_int
    lib.el_attn_decode_step.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, i32, vp]
    lib.el_attn_decode_step.restype = ctypes.c_int
    lib.el_attn_decode_step_static.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, i32, vp]
    lib.el_attn_decode_step_static.restype = ctypes.c_int
    lib.el_attn_expand_query.argtypes = [vp, vp, vp, i32, i32, vp]
    lib.el_attn_expand_query.restype = ctypes.c_int
    lib.el_attn_set_splits.argtypes = [vp, i32]
    lib.el_attn_set_splits.restype = ctypes.c_int
    lib.el_attn_set_row_groups.argtypes = [vp, i32]
    lib.el_attn_set_row_groups.restype = ctypes.c_int
    lib.el_attn_max_splits.argtypes = []
    lib.el_attn_max_splits.restype = i32
    lib.el_attn_plan_preview.argtypes = [i32] * 6 + [ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.el_attn_plan_preview.restype = ctypes.c_int
    lib.el_attn_plan_short_core.argtypes = [i32] * 7
    lib.el_attn_plan_short_core.restype = i32
    lib.el_attn_plan_step.argtypes = [i32] * 7 + [ctypes.POINTER(i32)] * 3
    lib.el_attn_plan_step.restype = ctypes.c_int
    lib.el_attn_uses_mfma.argtypes = [vp]
    lib.el_attn_uses_mfma.restype = i32
    lib.el_attn_check_step_operands.argtypes = [ctypes.POINTER(ElAttnConfig), i32, vp, i64, vp, vp, vp, i32, i32, i32]
    lib.el_attn_check_step_operands.restype = ctypes.c_int
    lib.el_attn_core_timing_enable.argtypes = [vp, i32]
    lib.el_attn_core_timing_enable.restype = ctypes.c_int
    lib.el_attn_core_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(i32)]
    lib.el_attn_core_timing_read.restype = ctypes.c_int
    lib.el_attn_gather_batch.argtypes = [ctypes.c_int, i32, vp, i64, vp, i32, vp, i64, vp, i32, vp, i32, vp]
    lib.el_attn_gather_batch.restype = ctypes.c_int
    lib.el_attn_check_inputs.argtypes = [ctypes.c_int, i32, vp, i64, vp, i32, i32, vp, vp]
    lib.el_attn_check_inputs.restype = ctypes.c_int
    lib.el_attn_decode_segment.argtypes = [vp, vp, i64, vp, vp, vp, vp, i32, i32, i32, vp]
    lib.el_attn_decode_segment.restype = ctypes.c_int
    lib.el_attn_merge_segments.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), vp, i32, i32, vp]
    lib.el_attn_merge_segments.restype = ctypes.c_int
    lib.el_attn_max_segments.argtypes = []
    lib.el_attn_max_segments.restype = i32
    pages, rule = ctypes.POINTER(ElAttnPages), ctypes.POINTER(ElAttnScoreRule)
    lib.el_attn_paged_workspace_bytes.argtypes = [pages, i32, i32, i32, i32]
    lib.el_attn_paged_workspace_bytes.restype = sz
    lib.el_attn_paged_attend.argtypes = [pages, vp, i64, i32, vp, vp, i64, i32, rule, vp, i32, vp, i32, i32, i32, vp, sz, vp]
    lib.el_attn_paged_attend.restype = ctypes.c_int
    lib.el_attn_paged_append.argtypes = [pages, vp, i64, i32, vp, vp, vp, vp, i64, i64, i32, i32, vp]
    lib.el_attn_paged_append.restype = ctypes.c_int
    lib.el_attn_paged_copy.argtypes = [pages, vp, vp, vp, i32, vp]
    lib.el_attn_paged_copy.restype = ctypes.c_int
    lib.el_attn_max_alternatives.argtypes = []
    lib.el_attn_max_alternatives.restype = i32
    lib.el_attn_score_workspace_bytes.argtypes = [i32, i32, i32]
    lib.el_attn_score_workspace_bytes.restype = sz
    lib.el_attn_score_tokens.argtypes = [ctypes.c_int, vp, i64, i32, i32, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.el_attn_score_tokens.restype = ctypes.c_int
    pages8 = ctypes.POINTER(ElAttnPages8)
    lib.el_attn_quantized_workspace_bytes.argtypes = [pages8, i32, i32, i32, i32, i32, i32]
    lib.el_attn_quantized_workspace_bytes.restype = sz
    lib.el_attn_quantized_attend.argtypes = [pages8, i32, vp, i64, i32, vp, vp, i64, i32, rule, vp, i32, vp, i32, i32, i32, vp, sz, vp]
    lib.el_attn_quantized_attend.restype = ctypes.c_int
    lib.el_attn_quantized_append.argtypes = [pages8, i32, vp, i64, i32, vp, vp, vp, vp, i64, i64, i32, i32, vp]
    lib.el_attn_quantized_append.restype = ctypes.c_int
    lib.el_attn_quantized_copy.argtypes = [pages8, vp, vp, vp, i32, vp]
    lib.el_attn_quantized_copy.restype = ctypes.c_int
    lib.el_attn_plan_workspace_bytes.argtypes = [i32, i32]
    lib.el_attn_plan_workspace_bytes.restype = sz
    for plan in (lib.el_attn_plan_pages, lib.el_attn_plan_pages_exclusive):
        plan.argtypes = [vp, i64, i32, vp, i32, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        plan.restype = ctypes.c_int
    lib.el_attn_sample_workspace_bytes.argtypes = [ctypes.c_int, i32, i32]
    lib.el_attn_sample_workspace_bytes.restype = sz
    lib.el_attn_sample_tokens.argtypes = [ctypes.c_int, vp, i64, i32, i32, vp, ctypes.POINTER(ElAttnSampleRule), vp, vp, vp, sz, vp]
    lib.el_attn_sample_tokens.restype = ctypes.c_int
    lib.el_attn_destroy.argtypes = [vp]
    lib.el_attn_destroy.restype = ctypes.c_int
    lib.el_attn_status_string.argtypes = [ctypes.c_int]
    lib.el_attn_status_string.restype = ctypes.c_char_p
    lib.el_attn_version.argtypes = []
    lib.el_attn_version.restype = i32
    return lib


lib = _load()


# ---- functions with the C names (raw pointers as ints / None) ---------------------------------
def status_string(status: int) -> str:
    return lib.el_attn_status_string(int(status)).decode()


el_attn_status_string = status_string


def el_attn_version() -> int:
    return int(lib.el_attn_version())


def el_attn_max_splits() -> int:
    return int(lib.el_attn_max_splits())


def el_attn_prepare(cfg: ElAttnConfig, Wq, bq, Wk, bk, Wv, bv, Wo, bo, stream=None):
    """Returns (status, ctx_handle).  Pointers are device addresses (int) or None."""
    ctx = ctypes.c_void_p()
    st = lib.el_attn_prepare(ctypes.byref(cfg), Wq, bq, Wk, bk, Wv, bv, Wo, bo, stream, ctypes.byref(ctx))
    return st, ctx


def el_attn_workspace_bytes(ctx) -> int:
    return int(lib.el_attn_workspace_bytes(ctx))


def el_attn_bind_workspace(ctx, dev_ptr, nbytes) -> int:
    return lib.el_attn_bind_workspace(ctx, dev_ptr, nbytes)


def el_attn_decode_step(ctx, H, H_batch_stride, lengths, queries, out, B, beam, n, stream=None) -> int:
    return lib.el_attn_decode_step(ctx, H, H_batch_stride, lengths, queries, out, B, beam, n, stream)


def el_attn_decode_step_static(ctx, H, H_batch_stride, lengths, queries, out, B, beam, n, stream=None) -> int:
    return int(lib.el_attn_decode_step_static(ctx, H, H_batch_stride, lengths, queries, out, B, beam, n, stream))


def el_attn_expand_query(ctx, queries, elq_out, B, beam, stream=None) -> int:
    return lib.el_attn_expand_query(ctx, queries, elq_out, B, beam, stream)


def el_attn_set_splits(ctx, splits) -> int:
    return lib.el_attn_set_splits(ctx, splits)


def el_attn_set_row_groups(ctx, row_groups) -> int:
    return lib.el_attn_set_row_groups(ctx, row_groups)


def el_attn_plan_preview(B, beam, heads, d_model, n, compute_units):
    """Returns (status, row_groups, splits)."""
    rg, sp = ctypes.c_int32(0), ctypes.c_int32(0)
    st = lib.el_attn_plan_preview(B, beam, heads, d_model, n, compute_units, ctypes.byref(rg), ctypes.byref(sp))
    return st, rg.value, sp.value


def el_attn_plan_short_core(max_batch, B, beam, heads, d_model, n, compute_units) -> int:
    return int(lib.el_attn_plan_short_core(max_batch, B, beam, heads, d_model, n, compute_units))


def el_attn_plan_step(max_batch, B, beam, heads, d_model, n, compute_units):
    """Returns (status, positions, row_groups, spans)."""
    out = [ctypes.c_int32(0) for _ in range(3)]
    st = lib.el_attn_plan_step(max_batch, B, beam, heads, d_model, n, compute_units, *map(ctypes.byref, out))
    return (st, *(v.value for v in out))


def el_attn_uses_mfma(ctx) -> int:
    return int(lib.el_attn_uses_mfma(ctx))


def el_attn_check_step_operands(cfg: ElAttnConfig, mfma, H, H_batch_stride, lengths, queries, out, B, beam, n) -> int:
    return int(lib.el_attn_check_step_operands(ctypes.byref(cfg), int(mfma), H, H_batch_stride, lengths, queries, out, B, beam, n))


def el_attn_gather_batch(dtype, d_model, H_src, src_batch_stride, lengths_src, B_src,
                         H_dst, dst_batch_stride, lengths_dst, B_dst, index, n, stream=None) -> int:
    return lib.el_attn_gather_batch(dtype, d_model, H_src, src_batch_stride, lengths_src, B_src,
                                    H_dst, dst_batch_stride, lengths_dst, B_dst, index, n, stream)


def el_attn_check_inputs(dtype, d_model, H, H_batch_stride, lengths, B, n, report, stream=None) -> int:
    return lib.el_attn_check_inputs(dtype, d_model, H, H_batch_stride, lengths, B, n, report, stream)


def el_attn_decode_segment(ctx, H, H_batch_stride, lengths, queries, seg_A, seg_lse, B, beam, n, stream=None) -> int:
    return lib.el_attn_decode_segment(ctx, H, H_batch_stride, lengths, queries, seg_A, seg_lse, B, beam, n, stream)


def el_attn_merge_segments(ctx, nseg, seg_A, seg_lse, out, B, beam, stream=None) -> int:
    """seg_A, seg_lse: sequences of device addresses (int, c_void_p or None), or None."""
    def arr(ptrs):
        if ptrs is None:
            return None
        vals = [p.value if isinstance(p, ctypes.c_void_p) else p for p in ptrs]
        return (ctypes.c_void_p * max(len(vals), 1))(*vals)
    return lib.el_attn_merge_segments(ctx, nseg, arr(seg_A), arr(seg_lse), out, B, beam, stream)


def el_attn_max_segments() -> int:
    return int(lib.el_attn_max_segments())


def el_attn_paged_workspace_bytes(cache: ElAttnPages, heads, B, beam, n) -> int:
    return int(lib.el_attn_paged_workspace_bytes(cache, heads, B, beam, n))


def el_attn_paged_attend(cache: ElAttnPages, table, table_stride, table_pages, lengths, queries, query_stride, heads,
                         rule: ElAttnScoreRule, out, out_dtype, lse, B, beam, n, workspace=None, workspace_bytes=0,
                         stream=None) -> int:
    return lib.el_attn_paged_attend(cache, table, table_stride, table_pages, lengths, queries, query_stride, heads, rule,
                                    out, out_dtype, lse, B, beam, n, workspace, workspace_bytes, stream)


def el_attn_paged_append(cache: ElAttnPages, table, table_stride, table_pages, lengths, counts, K_new, V_new,
                         batch_stride, token_stride, B, T, stream=None) -> int:
    return lib.el_attn_paged_append(cache, table, table_stride, table_pages, lengths, counts, K_new, V_new,
                                    batch_stride, token_stride, B, T, stream)


def el_attn_paged_copy(cache: ElAttnPages, src, dst, counts, pairs, stream=None) -> int:
    return lib.el_attn_paged_copy(cache, src, dst, counts, pairs, stream)


def el_attn_max_alternatives() -> int:
    return int(lib.el_attn_max_alternatives())


def el_attn_score_workspace_bytes(rows, vocab, k) -> int:
    return int(lib.el_attn_score_workspace_bytes(rows, vocab, k))


def el_attn_score_tokens(dtype, logits, row_stride, rows, vocab, tokens, logprob, entropy, k, top_logprob, top_index,
                         workspace=None, workspace_bytes=0, stream=None) -> int:
    return lib.el_attn_score_tokens(dtype, logits, row_stride, rows, vocab, tokens, logprob, entropy, k,
                                    top_logprob, top_index, workspace, workspace_bytes, stream)


def el_attn_quantized_workspace_bytes(cache: ElAttnPages8, dtype, out_dtype, heads, B, beam, n) -> int:
    return int(lib.el_attn_quantized_workspace_bytes(cache, dtype, out_dtype, heads, B, beam, n))


def el_attn_quantized_attend(cache: ElAttnPages8, dtype, table, table_stride, table_pages, lengths, queries, query_stride, heads,
                             rule: ElAttnScoreRule, out, out_dtype, lse, B, beam, n, workspace=None, workspace_bytes=0, stream=None) -> int:
    return lib.el_attn_quantized_attend(cache, dtype, table, table_stride, table_pages, lengths, queries, query_stride, heads, rule,
                                        out, out_dtype, lse, B, beam, n, workspace, workspace_bytes, stream)


def el_attn_quantized_append(cache: ElAttnPages8, dtype, table, table_stride, table_pages, lengths, counts, K_new, V_new,
                             batch_stride, token_stride, B, T, stream=None) -> int:
    return lib.el_attn_quantized_append(cache, dtype, table, table_stride, table_pages, lengths, counts, K_new, V_new,
                                        batch_stride, token_stride, B, T, stream)


def el_attn_quantized_copy(cache: ElAttnPages8, src, dst, counts, pairs, stream=None) -> int:
    return lib.el_attn_quantized_copy(cache, src, dst, counts, pairs, stream)


def el_attn_plan_workspace_bytes(B, pages) -> int:
    return int(lib.el_attn_plan_workspace_bytes(B, pages))


def el_attn_plan_pages(table, table_stride, columns, lengths, B_old, parents, counts, reserved, pages, page_size, B, T,
                       new_table, new_lengths, granted, slots, copies, free_pages, workspace=None, workspace_bytes=0, stream=None) -> int:
    return lib.el_attn_plan_pages(table, table_stride, columns, lengths, B_old, parents, counts, reserved, pages, page_size, B, T,
                                  new_table, new_lengths, granted, slots, copies, free_pages, workspace, workspace_bytes, stream)


def el_attn_plan_pages_exclusive(table, table_stride, columns, lengths, B_old, parents, counts, reserved, pages, page_size, B, T,
                                 new_table, new_lengths, granted, slots, copies, free_pages, workspace=None, workspace_bytes=0, stream=None) -> int:
    return lib.el_attn_plan_pages_exclusive(table, table_stride, columns, lengths, B_old, parents, counts, reserved, pages, page_size, B, T,
                                            new_table, new_lengths, granted, slots, copies, free_pages, workspace, workspace_bytes, stream)


def el_attn_sample_workspace_bytes(dtype, rows, vocab) -> int:
    return int(lib.el_attn_sample_workspace_bytes(dtype, rows, vocab))


def el_attn_sample_tokens(dtype, logits, row_stride, rows, vocab, uniform, rule: ElAttnSampleRule, tokens, logprob,
                          workspace=None, workspace_bytes=0, stream=None) -> int:
    return lib.el_attn_sample_tokens(dtype, logits, row_stride, rows, vocab, uniform, rule, tokens, logprob, workspace, workspace_bytes, stream)


def el_attn_core_timing_enable(ctx, max_steps) -> int:
    return lib.el_attn_core_timing_enable(ctx, max_steps)


def el_attn_core_timing_read(ctx, capacity):
    """Returns (status, [milliseconds of each recorded step's core kernel])."""
    buf = (ctypes.c_float * max(capacity, 1))()
    n = ctypes.c_int32(0)
    st = lib.el_attn_core_timing_read(ctx, buf, capacity, ctypes.byref(n))
    return st, [buf[i] for i in range(n.value)]


def el_attn_destroy(ctx) -> int:
    return lib.el_attn_destroy(ctx)


# ---- torch convenience wrapper (still marshalling only) ------------------------------------
def _torch_dtype(code):
    import torch
    return {EL_F32: torch.float32, EL_F16: torch.float16, EL_BF16: torch.bfloat16}[code]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream_handle():
    """The current device's current stream as an address.  The stream object that torch.cuda.current_stream() builds costs
    2.9 us, a sixth of what the host spends on a whole step; torch's own accessor of the address 0.2."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream


def to_device(x32, dtype: str, device="cuda"):
    """float32 values already rounded to `dtype` ("f32", "f16", "bf16") -> device tensor of that dtype, bit-exact
    (argument marshalling for numpy-side callers; bf16 has no numpy type, so its bit pattern travels as int16)."""
    import numpy as np
    import torch
    from . import workloads as wl
    bits = wl.storage_bits(x32, dtype)
    if dtype == "bf16":
        return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(bits).to(device)


def device_weights(W: dict, dtype: str):
    """The weight dictionary of `workloads.weights` (numpy float32, rounded to `dtype`) on the device."""
    return {k: (None if v is None else to_device(v, dtype)) for k, v in W.items()}


def gather_batch(H_src, lengths_src, index, *, H_dst=None, lengths_dst=None):
    """H_dst[i, :len] = H_src[index[i], :len], lengths_dst[i] = len (marshalling only; see el_attn_gather_batch).

    H_src [B_src, n, d_m] device tensor (last two dimensions contiguous), lengths_src int32 [B_src] or None,
    index int32 [B_dst] device tensor.  Returns (H_dst, lengths_dst); fresh destination rows beyond a length
    are left as allocated.
    """
    import torch
    if H_src.dim() != 3 or H_src.stride(2) != 1 or H_src.stride(1) != H_src.shape[2]:
        raise ValueError("H_src must be [B, n, d_m] with contiguous rows")
    code = {torch.float32: EL_F32, torch.float16: EL_F16, torch.bfloat16: EL_BF16}[H_src.dtype]
    B_src, n, d_m = H_src.shape
    B_dst = int(index.shape[0])
    if index.dtype != torch.int32 or not index.is_cuda:
        raise ValueError("index must be an int32 device tensor")
    if H_dst is None:
        H_dst = torch.empty((B_dst, n, d_m), dtype=H_src.dtype, device=H_src.device)
    if lengths_dst is None and lengths_src is not None:
        lengths_dst = torch.empty((B_dst,), dtype=torch.int32, device=H_src.device)
    st = el_attn_gather_batch(code, d_m, _ptr(H_src), H_src.stride(0), _ptr(lengths_src), B_src,
                              _ptr(H_dst), H_dst.stride(0), _ptr(lengths_dst), B_dst, _ptr(index), n, _stream_handle())
    if st != EL_OK:
        raise ElAttnError(st, "el_attn_gather_batch")
    return H_dst, lengths_dst


def check_inputs(H, lengths, report=None):
    """Counts of what a decode step assumes about (H, lengths): returns a device int64 tensor
    [bad lengths, non-finite elements, elements beyond the fp16 range, elements examined] (see el_attn_check_inputs)."""
    import torch
    if H.dim() != 3 or H.stride(2) != 1 or H.stride(1) != H.shape[2]:
        raise ValueError("H must be [B, n, d_m] with contiguous rows")
    code = {torch.float32: EL_F32, torch.float16: EL_F16, torch.bfloat16: EL_BF16}[H.dtype]
    B, n, d_m = H.shape
    if lengths is not None and lengths.dtype != torch.int32:
        raise ValueError("lengths must be int32")
    if report is None:
        report = torch.empty(4, dtype=torch.int64, device=H.device)
    st = el_attn_check_inputs(code, d_m, _ptr(H), H.stride(0) if B > 1 else n * d_m, _ptr(lengths), B, n,
                              _ptr(report), _stream_handle())
    if st != EL_OK:
        raise ElAttnError(st, "el_attn_check_inputs")
    return report


def _dtype_code(t):
    import torch
    code = {torch.float32: EL_F32, torch.float16: EL_F16, torch.bfloat16: EL_BF16}.get(t.dtype)
    if code is None:
        raise ValueError(f"unsupported dtype {t.dtype}: float32, float16 or bfloat16")
    return code


def _check_index(name, t, device, shape):
    """An index operand: contiguous int32 of that shape on `device`."""
    import torch
    if t.dtype is not torch.int32 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on {device}")


def _check_tangent(name, t):
    import torch
    fw = torch.autograd.forward_ad       # (outside of a dual level, where no tensor has one, 0.25 us; with torch's accessor 0.5)
    if getattr(fw, "_current_level", 0) >= 0 and fw.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} has a tangent, and none is computed: pass its primal")


def _check_values(name, t, device, dtype):
    """A floating operand on `device`, one that nobody waits for a gradient or a tangent of: none is computed."""
    if t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor on {device}")
    if t.requires_grad:
        import torch
        if torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, and none is computed: detach it or use torch.no_grad()")
    _check_tangent(name, t)


def _call(where, device, fn, *args):
    """fn(*args, stream) on `device` (the operands'), on the stream that is current there."""
    import torch
    if device.index == torch.cuda.current_device():
        st = fn(*args, _stream_handle())
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream_handle())
    if st != EL_OK:
        raise ElAttnError(st, where)


_INT32_MAX = 2 ** 31 - 1


def _check_pools(K, V):
    """Pools of a paged cache, given as K and V: what holds for both storage widths."""
    if K.dim() != 4 or K.shape != V.shape or K.dtype != V.dtype or K.stride() != V.stride():
        raise ValueError("K and V must be [pages, page_size, kv_heads, d_head] of one dtype and the same strides")
    if not K.is_cuda or K.device != V.device:
        raise ValueError("K and V must be on one device")
    if K.stride(3) != 1 or max(K.shape) > _INT32_MAX:
        raise ValueError("the last dimension of K and V must be contiguous, and every dimension below 2^31")


class _Pages:
    """What the paged caches share: tables, new tokens, queries, copies.  A cache sets _torch, device, page_size, kv_heads, d_head, _pages, and _types: the type that
    it takes, as a code and as torch's, or None where each call says (a cache in 8 bits).  The calls of the two are written out: the smallest ones are as long as this takes."""

    @property
    def K(self):
        """The pool of keys that the cache was made of; another one needs another cache."""
        return self._K

    @property
    def V(self):
        return self._V

    def _table(self, table, B):
        """(address, row stride, columns) of a table for B sequences."""
        shape, strides = table.shape, table.stride()
        if len(shape) != 2 or shape[0] != B or (shape[1] > 1 and strides[1] != 1):
            raise ValueError(f"table must be [{B}, columns] with contiguous rows")
        if table.dtype is not self._torch.int32 or table.device != self.device:
            raise ValueError(f"table must be an int32 tensor on {self.device}")
        return table.data_ptr(), strides[0] if B > 1 else shape[1], shape[1]

    def _append(self, k, v, table, lengths, counts):
        shape, strides, device = k.shape, k.stride(), self.device
        code, element = self._types or (_dtype_code(k), k.dtype)
        if len(shape) != 4 or shape != v.shape or shape[2] != self.kv_heads or shape[3] != self.d_head:
            raise ValueError(f"k and v must be [B, T, {self.kv_heads}, {self.d_head}]")
        if strides[3] != 1 or (self.kv_heads > 1 and strides[2] != self.d_head) or v.stride() != strides:
            raise ValueError("a token's heads must be contiguous, and k and v have the same strides")
        _check_values("k", k, device, element)
        _check_values("v", v, device, element)
        B, T = shape[0], shape[1]
        _check_index("lengths", lengths, device, (B,))
        if counts is not None:
            _check_index("counts", counts, device, (B,))
        row = self.kv_heads * self.d_head
        at, stride, columns = self._table(table, B)
        if B == 0 or T == 0:
            return
        if self._types:
            _call("el_attn_paged_append", device, lib.el_attn_paged_append, self._pages, at, stride, columns, lengths.data_ptr(),
                  _ptr(counts), k.data_ptr(), v.data_ptr(), strides[0] if B > 1 else T * row, strides[1] if T > 1 else row, B, T)
        else:
            _call("el_attn_quantized_append", device, lib.el_attn_quantized_append, self._pages, code, at, stride, columns, lengths.data_ptr(),
                  _ptr(counts), k.data_ptr(), v.data_ptr(), strides[0] if B > 1 else T * row, strides[1] if T > 1 else row, B, T)

    def _attend(self, queries, table, lengths, n, scale, softcap, window, slopes, out, out_code, lse):
        """`queries` has been found to be [B, beam, heads, d_head] of a type that this cache takes."""
        (B, beam, heads, d), strides, device = queries.shape, queries.stride(), self.device
        if strides[3] != 1 or (heads > 1 and strides[2] != d):
            raise ValueError("the heads of a query must be contiguous")
        if B > 1 and beam > 1 and strides[0] != beam * strides[1]:
            raise ValueError("query rows must be evenly spaced")
        if lengths is not None:
            _check_index("lengths", lengths, device, (B,))
        if slopes is not None:
            _check_values("slopes", slopes, device, self._torch.float32)
            if slopes.shape != (heads,) or not slopes.is_contiguous():
                raise ValueError(f"slopes must be contiguous [{heads}]")
        at, stride, columns = self._table(table, B)
        if B == 0 or beam == 0:
            return
        if n is None:
            n = min(columns * self.page_size, _INT32_MAX)
        if abs(n) > _INT32_MAX or abs(window) > _INT32_MAX:
            raise ValueError("n and window must be 32-bit numbers")
        rule = ElAttnScoreRule(d ** -0.5 if scale is None else scale, softcap, window, _ptr(slopes))
        if self._types:
            nbytes = lib.el_attn_paged_workspace_bytes(self._pages, heads, B, beam, n)
            ws = self._torch.empty(nbytes, dtype=self._torch.uint8, device=device) if nbytes else None
            _call("el_attn_paged_attend", device, lib.el_attn_paged_attend, self._pages, at, stride, columns, _ptr(lengths),
                  queries.data_ptr(), strides[1] if beam > 1 else strides[0] if B > 1 else heads * d, heads, rule,
                  out.data_ptr(), out_code, _ptr(lse), B, beam, n, _ptr(ws), nbytes)
        else:
            code = _dtype_code(queries)
            nbytes = lib.el_attn_quantized_workspace_bytes(self._pages, code, out_code, heads, B, beam, n)
            ws = self._torch.empty(nbytes, dtype=self._torch.uint8, device=device) if nbytes else None
            _call("el_attn_quantized_attend", device, lib.el_attn_quantized_attend, self._pages, code, at, stride, columns, _ptr(lengths),
                  queries.data_ptr(), strides[1] if beam > 1 else strides[0] if B > 1 else heads * d, heads, rule,
                  out.data_ptr(), out_code, _ptr(lse), B, beam, n, _ptr(ws), nbytes)

    def _check_queries(self, queries):
        """The queries' type, as a code and as torch's."""
        shape = queries.shape
        if len(shape) != 4 or shape[3] != self.d_head or shape[2] % self.kv_heads != 0:
            raise ValueError(f"queries must be [B, beam, heads, {self.d_head}], heads a multiple of {self.kv_heads}")
        types = self._types or (_dtype_code(queries), queries.dtype)
        _check_values("queries", queries, self.device, types[1])
        return types

    def attend(self, queries, table, lengths, *, n=None, scale=None, softcap=0.0, window=0, slopes=None,
               out_dtype=None, out=None):
        """Attention of queries [B, beam, heads, d_head] over each sequence's lengths[b] positions (None: n; n: the most that
        any sequence has, default what the table holds).  Returns out [B, beam, heads, d_head] in `out_dtype` ("f32" or the
        queries' own, the default).  See el_attn_score_rule for scale (default d_head ** -0.5), softcap, window and slopes."""
        own, own_element = self._check_queries(queries)
        code = own if out_dtype is None else DTYPE_CODES[out_dtype]
        element = own_element if code == own else _torch_dtype(code)
        if out is None:
            out = self._torch.empty(queries.shape, dtype=element, device=self.device)
        elif out.shape != queries.shape or not out.is_contiguous():
            raise ValueError(f"out must be a contiguous {element} tensor of the queries' shape")
        else:
            _check_values("out", out, self.device, element)
        self._attend(queries, table, lengths, n, scale, softcap, window, slopes, out, code, None)
        return out

    def attend_segment(self, queries, table, lengths, *, n=None, scale=None, softcap=0.0, window=0, slopes=None):
        """The same as a segment (seg_A [B*beam, heads*d_head], seg_lse [B*beam, heads], float32) for
        ElAttention.merge_segments.  decode_segment has no cap, window or slopes, and the scale d_k ** -0.5: joined with one of its segments, neither may
        this one."""
        torch = self._torch
        self._check_queries(queries)
        B, beam, heads, d = queries.shape
        A = torch.empty((B * beam, heads * d), dtype=torch.float32, device=self.device)
        lse = torch.empty((B * beam, heads), dtype=torch.float32, device=self.device)
        self._attend(queries, table, lengths, n, scale, softcap, window, slopes, A, EL_F32, lse)
        return A, lse

    def _copy_pages(self, where, fn, src, dst, counts):
        device, shape = self.device, (src.numel(),)
        _check_index("src", src, device, shape)
        _check_index("dst", dst, device, shape)
        if counts is not None:
            _check_index("counts", counts, device, shape)
        if shape[0] == 0:
            return
        _call(where, device, fn, self._pages, src.data_ptr(), dst.data_ptr(), _ptr(counts), shape[0])


class PagedCache(_Pages):
    """Projected keys and values of one attention layer, in pages (see el_attn_pages): new tokens in, attention of one token
    per query row out (no causal form for several new tokens of a sequence), pages copied for beams that fork.

    K, V: device tensors [pages, page_size, kv_heads, d_head], the last dimension contiguous, with the same strides (a
    transposed view of [pages, kv_heads, page_size, d_head] is as good).  The table [B, columns] int32 and the lengths
    int32 [B] are the caller's, shared by all layers: position t of sequence b lies in page table[b, t // page_size];
    an entry outside the pool (-1) holds no positions.  Scratch memory comes from torch per call, so calls on several streams
    and captured graphs keep apart.  No work (no sequence, no token, no pair, no beam) is no error.
    """

    def __init__(self, K, V):
        import torch
        self._torch = torch
        _check_pools(K, V)
        if K.requires_grad or V.requires_grad:
            raise ValueError("K and V are written in place: they must not require a gradient")
        _check_tangent("K", K)
        _check_tangent("V", V)
        self._K, self._V = K, V
        self.device = K.device
        pages, self.page_size, self.kv_heads, self.d_head = K.shape
        self.dtype = _dtype_code(K)
        self._types = self.dtype, K.dtype
        self._pages = ElAttnPages(_ptr(K), _ptr(V), K.stride(0), K.stride(1), K.stride(2),
                                  pages, self.page_size, self.kv_heads, self.d_head, self.dtype)

    def append(self, k, v, table, lengths, counts=None):
        """New tokens k, v [B, T, kv_heads, d_head] (heads of a token contiguous, other strides free, the same for both) to
        the positions lengths[b] - counts[b] + i, i < counts[b] (default T): `lengths` counts them already.  B up to 65535."""
        self._append(k, v, table, lengths, counts)

    def copy_pages(self, src, dst, counts=None):
        """Positions [0, counts[i]) (default all) of page dst[i] become those of page src[i]; int32 device tensors.  No page
        may be the destination of two pairs, or the destination of one and the source of another."""
        self._copy_pages("el_attn_paged_copy", lib.el_attn_paged_copy, src, dst, counts)


class PagedCache8(_Pages):
    """The paged cache in 8 bits (see el_attn_pages8): keys and values as codes, with a scale for each block of positions and head.

    K, V: device tensors [pages, page_size, kv_heads, d_head], torch.float8_e4m3fn or torch.int8, strides as for PagedCache; d_head a
    multiple of 16.  K_scale, V_scale: float32 [pages, kv_heads, page_size // block], contiguous; a value is code times scale.  What `append`
    has not written needs neither codes nor scales.  Queries and new tokens are float32, float16 or bfloat16, whichever a call is given.
    Everything else is as with PagedCache: the table and lengths may be the same.
    """

    def __init__(self, K, V, K_scale, V_scale):
        import torch
        self._torch = torch
        _check_pools(K, V)
        self.format = {torch.float8_e4m3fn: EL_E4M3, torch.int8: EL_INT8}.get(K.dtype)
        if self.format is None:
            raise ValueError(f"unsupported dtype {K.dtype}: float8_e4m3fn or int8")
        pages, self.page_size, self.kv_heads, self.d_head = K.shape
        self.device, self._types = K.device, None
        shape = K_scale.shape
        if len(shape) != 3 or tuple(shape[:2]) != (pages, self.kv_heads) or shape[2] < 1 or self.page_size % shape[2] != 0 or V_scale.shape != shape:
            raise ValueError("K_scale and V_scale must be [pages, kv_heads, blocks of a page], the blocks all of one size")
        for name, t in (("K", K), ("V", V), ("K_scale", K_scale), ("V_scale", V_scale)):
            if t.requires_grad:
                raise ValueError(f"{name} is written in place: it must not require a gradient")
            _check_tangent(name, t)
        for name, t in (("K_scale", K_scale), ("V_scale", V_scale)):
            _check_values(name, t, self.device, torch.float32)
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        self._K, self._V, self._K_scale, self._V_scale = K, V, K_scale, V_scale
        self.block = self.page_size // shape[2]
        self._pages = ElAttnPages8(_ptr(K), _ptr(V), _ptr(K_scale), _ptr(V_scale), K.stride(0), K.stride(1), K.stride(2),
                                   pages, self.page_size, self.kv_heads, self.d_head, self.block, self.format)

    @property
    def K_scale(self):
        return self._K_scale

    @property
    def V_scale(self):
        return self._V_scale

    def append(self, k, v, table, lengths, counts=None):
        """New tokens as in PagedCache.append, rounded to codes: a block's scale is its largest value over the largest code, and grows (what the block
        holds is rounded again) where a later token needs it.  No other sequence may hold or write positions of a block that is written:
        plan_pages with exclusive=True sees to that."""
        self._append(k, v, table, lengths, counts)

    def copy_pages(self, src, dst, counts=None):
        """Positions [0, counts[i]) (default all) of page dst[i], and the scales of their blocks, become those of page src[i]; as PagedCache.copy_pages."""
        self._copy_pages("el_attn_quantized_copy", lib.el_attn_quantized_copy, src, dst, counts)


PagePlan = collections.namedtuple("PagePlan", "table lengths granted slots copies free")
PagePlan.__doc__ = """The table of a step (see plan_pages): table [B, columns], lengths [B] with the new positions, granted [B] of them, slots [B, tokens] (int64;
page * page_size + place, -1 for none), copies [3, B] (the operands of copy_pages), free [1] pages left; int32 where not said otherwise."""


def plan_pages(table, lengths, counts=None, *, pages, page_size, tokens=1, parents=None, reserved=None, slots=True, exclusive=False):
    """The next step's table from what every sequence holds and needs, on the device (see el_attn_plan_pages).

    table int32 [B_old, columns] (rows strided, a row contiguous) and lengths int32 [B_old]: what the sequences hold.  parents int32 [B] (None: each goes on
    from itself): whom sequence b goes on from; -1 starts a new one.  counts int32 [B] (None: `tokens` each): positions that it needs, up to `tokens`.
    pages, page_size: of the pool; reserved uint8 or bool [pages]: pages that others use.  A page that the new sequences do not name is free.
    exclusive: a page that is written is kept only if nothing else names it.  A PagedCache8 needs that: what it holds of a block is rounded again when a larger token comes,
    also for a sequence that shares the block and writes nothing.  A PagedCache does without: sequences may share what they have in common of a page.

        plan = plan_pages(table, lengths, counts, pages=cache.K.shape[0], page_size=cache.page_size, parents=parents, exclusive=isinstance(cache, PagedCache8))
        cache.copy_pages(*plan.copies)
        cache.append(k, v, plan.table, plan.lengths, plan.granted)

    Returns a PagePlan of new tensors (slots=False: None in the place of its slots).  Where the free pages do not suffice, the first sequences
    are served: granted is 0 for the others.  No sequence, of the old or of the new, is no error."""
    import torch
    shape, device, i32 = table.shape, table.device, torch.int32
    if len(shape) != 2 or not table.is_cuda or table.dtype is not i32 or (shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be an int32 device tensor [B, columns] with contiguous rows")
    B_old, columns = shape
    _check_index("lengths", lengths, device, (B_old,))
    B = B_old if parents is None else parents.numel()
    if parents is not None:
        _check_index("parents", parents, device, (B,))
    if counts is not None:
        _check_index("counts", counts, device, (B,))
    if reserved is not None and (reserved.dtype not in (torch.uint8, torch.bool) or reserved.device != device or reserved.shape != (pages,) or not reserved.is_contiguous()):
        raise ValueError(f"reserved must be a contiguous uint8 or bool tensor [{pages}] on {device}")
    if max(pages, page_size, tokens, columns, B, B_old) > _INT32_MAX or columns < 1:
        raise ValueError("sizes must be 32-bit numbers, with at least one column")
    if B_old == 0:                                                   # there is none to go on from
        table, lengths, B_old, parents = table.new_zeros((1, columns)), lengths.new_zeros(1), 1, lengths.new_full((B,), -1)
    none = B == 0
    if none:                                                         # one that needs nothing tells of the free pages
        parents, counts, B = lengths.new_full((1,), -1), lengths.new_zeros(1), 1
    new_table = torch.empty((B, columns), dtype=i32, device=device)
    small = torch.empty(5 * B + 1, dtype=i32, device=device)         # lengths, granted, copies, free
    places = torch.empty((B, tokens), dtype=torch.int64, device=device) if slots and tokens > 0 else None
    nbytes = lib.el_attn_plan_workspace_bytes(B, pages)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    at = small.data_ptr()
    where, fn = ("el_attn_plan_pages_exclusive", lib.el_attn_plan_pages_exclusive) if exclusive else ("el_attn_plan_pages", lib.el_attn_plan_pages)
    _call(where, device, fn, table.data_ptr(), table.stride(0) if B_old > 1 else columns, columns, lengths.data_ptr(), B_old,
          _ptr(parents), _ptr(counts), _ptr(reserved), pages, page_size, B, tokens, new_table.data_ptr(), at, at + 4 * B, _ptr(places), at + 8 * B, at + 20 * B,
          ws.data_ptr(), nbytes)
    new_lengths, granted, copies, free = torch.split_with_sizes(small, (B, B, 3 * B, 1))
    copies = copies.view(3, B)
    if none:
        return PagePlan(new_table[:0], new_lengths[:0], granted[:0], None if places is None else places[:0], copies[:, :0], free)
    return PagePlan(new_table, new_lengths, granted, places, copies, free)


def _setting(name, value, rows, device, dtype):
    """A filter's setting: (number, address of a number for each row or None)."""
    import torch
    if not isinstance(value, torch.Tensor):
        return value, None
    if value.dtype is not dtype or value.device != device or value.shape != (rows,) or not value.is_contiguous():
        raise ValueError(f"{name} must be a number or a contiguous {dtype} tensor [{rows}] on {device}")
    if dtype is torch.float32:
        _check_values(name, value, device, dtype)
    return 0, value.data_ptr()


def sample_tokens(logits, uniform, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The next token of every row of logits [rows, vocab] (rows strided, a row contiguous): (tokens int32 [rows], logprob float32 [rows]).

    uniform float32 [rows]: random numbers in [0, 1), one a row; the token is the first of the vocabulary at which the probabilities left by the filters add up to
    more.  temperature, top_k, top_p, min_p: numbers, or a tensor [rows] (float32; top_k int32) with a setting for each row, in this order; off: 1.0, 0, 1.0, 0.0.  A
    temperature of 0 takes the largest logit.  logprob is the token's among what is left.  See el_attn_sample_tokens."""
    import torch
    shape = logits.shape
    if len(shape) != 2 or not logits.is_cuda or (shape[1] > 1 and logits.stride(1) != 1) or max(shape) > _INT32_MAX:
        raise ValueError("logits must be a device tensor [rows, vocab] with contiguous rows")
    rows, vocab = shape
    device, code, f32 = logits.device, _dtype_code(logits), torch.float32
    _check_values("logits", logits, device, logits.dtype)
    _check_values("uniform", uniform, device, f32)
    if uniform.shape != (rows,) or not uniform.is_contiguous():
        raise ValueError(f"uniform must be contiguous [{rows}]")
    t, row_t = _setting("temperature", temperature, rows, device, f32)
    k, row_k = _setting("top_k", top_k, rows, device, torch.int32)
    p, row_p = _setting("top_p", top_p, rows, device, f32)
    m, row_m = _setting("min_p", min_p, rows, device, f32)
    if abs(k) > _INT32_MAX:
        raise ValueError("top_k must be a 32-bit number")
    tokens = torch.empty(rows, dtype=torch.int32, device=device)
    logprob = torch.empty(rows, dtype=f32, device=device)
    if rows == 0:
        return tokens, logprob
    nbytes = lib.el_attn_sample_workspace_bytes(code, rows, vocab)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    _call("el_attn_sample_tokens", device, lib.el_attn_sample_tokens, code, logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, rows, vocab,
          uniform.data_ptr(), ElAttnSampleRule(t, k, p, m, row_t, row_k, row_p, row_m), tokens.data_ptr(), logprob.data_ptr(), _ptr(ws), nbytes)
    return tokens, logprob


def score_tokens(logits, tokens=None, *, k=0):
    """What rows of logits [rows, vocab] (rows strided, a row contiguous) say about the next token: (logprob, entropy,
    top_logprob, top_index), float32 [rows], [rows], [rows, k] and int32 [rows, k].  logprob is that of tokens (int32 [rows];
    None: logprob is None); the k best alternatives come in descending order.  No rows: empty results.  See el_attn_score_tokens."""
    import torch
    shape = logits.shape
    if len(shape) != 2 or not logits.is_cuda or (shape[1] > 1 and logits.stride(1) != 1) or max(shape) > _INT32_MAX:
        raise ValueError("logits must be a device tensor [rows, vocab] with contiguous rows")
    rows, vocab = shape
    device, code = logits.device, _dtype_code(logits)
    _check_values("logits", logits, device, logits.dtype)
    if tokens is not None:
        _check_index("tokens", tokens, device, (rows,))
    if not 0 <= k <= _MAX_ALTERNATIVES:
        raise ValueError(f"k must lie in [0, {_MAX_ALTERNATIVES}]")
    f32 = torch.float32
    logprob = None if tokens is None else torch.empty(rows, dtype=f32, device=device)
    entropy = torch.empty(rows, dtype=f32, device=device)
    top_logprob = torch.empty((rows, k), dtype=f32, device=device)
    top_index = torch.empty((rows, k), dtype=torch.int32, device=device)
    if rows == 0:
        return logprob, entropy, top_logprob, top_index
    nbytes = lib.el_attn_score_workspace_bytes(rows, vocab, k)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    _call("el_attn_score_tokens", device, lib.el_attn_score_tokens, code, logits.data_ptr(), logits.stride(0) if rows > 1 else vocab,
          rows, vocab, _ptr(tokens), _ptr(logprob), entropy.data_ptr(), k, top_logprob.data_ptr(), top_index.data_ptr(), _ptr(ws), nbytes)
    return logprob, entropy, top_logprob, top_index


_MAX_ALTERNATIVES = el_attn_max_alternatives()


class ElAttention:
    """One attention layer prepared for decode steps on the current CUDA/HIP device.

    weights: dict with Wq, Wk, Wv [d_m, h*d_k], Wo [h*d_k, d_m] and optional bq, bk, bv, bo
    as torch tensors on the device in the storage dtype.
    """

    def __init__(self, weights, *, heads, d_k, dtype, max_batch, max_beam, max_n,
                 out_dtype="f32", flags=0):
        import torch
        self._torch = torch
        d_m = weights["Wq"].shape[0]
        self.cfg = ElAttnConfig(heads, d_m, d_k, DTYPE_CODES[dtype], DTYPE_CODES[out_dtype],
                                max_batch, max_beam, max_n, flags)
        td = _torch_dtype(self.cfg.dtype)
        for k, v in weights.items():
            if v is not None:
                if not v.is_cuda or v.dtype != td or not v.is_contiguous():
                    raise ValueError(f"weight {k} must be a contiguous device tensor of dtype {td}")
        g = lambda k: _ptr(weights.get(k))
        st, ctx = el_attn_prepare(self.cfg, g("Wq"), g("bq"), g("Wk"), g("bk"), g("Wv"), g("bv"),
                                  g("Wo"), g("bo"), _stream_handle())
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_prepare")
        self.ctx = ctx
        self.d_m = d_m
        nbytes = el_attn_workspace_bytes(ctx)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=weights["Wq"].device)
        st = el_attn_bind_workspace(ctx, _ptr(self.workspace), nbytes)
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_bind_workspace")

    @property
    def uses_mfma(self) -> bool:
        return bool(el_attn_uses_mfma(self.ctx))

    def set_splits(self, splits: int):
        st = el_attn_set_splits(self.ctx, splits)
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_set_splits")

    def set_row_groups(self, row_groups: int):
        st = el_attn_set_row_groups(self.ctx, row_groups)
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_set_row_groups")

    def decode_step(self, H, lengths, queries, out=None):
        """H [B,n,d_m] (batch stride free, rows contiguous), lengths int32 [B] or None,
        queries [B,beam,d_m] contiguous.  Returns out [B,beam,d_m]."""
        torch = self._torch
        B, n, d_m = H.shape
        beam = queries.shape[1]
        if H.stride(2) != 1 or H.stride(1) != d_m:
            raise ValueError("rows of H must be contiguous with stride d_m")
        if not queries.is_contiguous():
            raise ValueError("queries must be contiguous")
        if out is None:
            out = torch.empty((B, beam, d_m), dtype=_torch_dtype(self.cfg.out_dtype), device=H.device)
        if lengths is not None and lengths.dtype != torch.int32:
            raise ValueError("lengths must be int32")
        st = el_attn_decode_step(self.ctx, _ptr(H), H.stride(0) if B > 1 else n * d_m, _ptr(lengths),
                                 _ptr(queries), _ptr(out), B, beam, n, _stream_handle())
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_decode_step")
        return out

    def decode_segment(self, H, lengths, queries):
        """a1..a6 on one key set: returns (seg_A [B*beam, h*d_k], seg_lse [B*beam, h]) in fp32."""
        torch = self._torch
        B, n, d_m = H.shape
        beam = queries.shape[1]
        if H.stride(2) != 1 or H.stride(1) != d_m:
            raise ValueError("rows of H must be contiguous with stride d_m")
        if not queries.is_contiguous():
            raise ValueError("queries must be contiguous")
        if lengths is not None and lengths.dtype != torch.int32:
            raise ValueError("lengths must be int32")
        hd = self.cfg.heads * self.cfg.d_k
        seg_A = torch.empty((B * beam, hd), dtype=torch.float32, device=H.device)
        seg_lse = torch.empty((B * beam, self.cfg.heads), dtype=torch.float32, device=H.device)
        st = el_attn_decode_segment(self.ctx, _ptr(H), H.stride(0) if B > 1 else n * d_m, _ptr(lengths),
                                    _ptr(queries), _ptr(seg_A), _ptr(seg_lse), B, beam, n, _stream_handle())
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_decode_segment")
        return seg_A, seg_lse

    def merge_segments(self, segments, B, beam, out=None):
        """segments: list of (seg_A, seg_lse) fp32 device tensors over the same B*beam rows.  Returns out [B,beam,d_m]."""
        torch = self._torch
        for A, S in segments:
            if A.dtype != torch.float32 or S.dtype != torch.float32 or not A.is_contiguous() or not S.is_contiguous():
                raise ValueError("segments must be contiguous float32 tensors")
            if A.shape[0] != B * beam or S.shape[0] != B * beam:
                raise ValueError("every segment must cover the same B*beam query rows")
        if out is None:
            out = torch.empty((B, beam, self.d_m), dtype=_torch_dtype(self.cfg.out_dtype), device=segments[0][0].device)
        st = el_attn_merge_segments(self.ctx, len(segments), [_ptr(A) for A, _ in segments],
                                    [_ptr(S) for _, S in segments], _ptr(out), B, beam, _stream_handle())
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_merge_segments")
        return out

    def core_timing(self, max_steps: int):
        st = el_attn_core_timing_enable(self.ctx, max_steps)
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_core_timing_enable")

    def read_core_timing(self, capacity: int):
        st, ms = el_attn_core_timing_read(self.ctx, capacity)
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_core_timing_read")
        return ms

    def expand_query(self, queries):
        torch = self._torch
        B, beam, d_m = queries.shape
        elq = torch.empty((B, self.cfg.heads * beam, d_m), dtype=torch.float32, device=queries.device)
        st = el_attn_expand_query(self.ctx, _ptr(queries), _ptr(elq), B, beam, _stream_handle())
        if st != EL_OK:
            raise ElAttnError(st, "el_attn_expand_query")
        return elq

    def close(self):
        if getattr(self, "ctx", None):
            el_attn_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
