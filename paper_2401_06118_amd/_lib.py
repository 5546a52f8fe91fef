"""ctypes binding of ``libaqlm_mi355x.so`` (C ABI in ``include/aqlm.h``).

Argument marshalling only: shapes and dtypes are read from torch tensors,
device pointers and the current HIP stream are passed through, and every
step of the computation runs in the library's kernels.  There is no CPU
fallback: without the built library every call raises.
"""
from __future__ import annotations

import ctypes
import os
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libaqlm_mi355x.so")

AQLM_OK = 0
STATUS_NAMES = {0: "AQLM_OK", 1: "AQLM_ERR_NULL", 2: "AQLM_ERR_SHAPE", 3: "AQLM_ERR_UNSUPPORTED",
                4: "AQLM_ERR_ALIGN", 5: "AQLM_ERR_HIP", 6: "AQLM_ERR_WORKSPACE", 7: "AQLM_ERR_SCRATCH",
                8: "AQLM_ERR_TIMEOUT"}
PATH_AUTO, PATH_GATHER, PATH_TABLE = 0, 1, 2
EXPORTS = ("aqlm_dequantize", "aqlm_gemv", "aqlm_gemv_grouped", "aqlm_gemv_grouped_path", "aqlm_gemm_small_batch",
           "aqlm_gemm_workspace_bytes", "aqlm_gemm", "aqlm_gemm_noalloc", "aqlm_backward", "aqlm_beam_search",
           "aqlm_packed_row_words", "aqlm_gemv_step_plan_bytes", "aqlm_gemv_step_plan", "aqlm_gemv_step",
           "aqlm_gemv_step_status", "aqlm_sort_codes_size", "aqlm_sort_codes", "aqlm_gemv_sorted_workspace_bytes",
           "aqlm_gemv_sorted", "aqlm_gemv_sorted_grouped", "aqlm_status_string", "aqlm_tiled_codes_bytes",
           "aqlm_tile_codes", "aqlm_gemv_grouped_tiled", "aqlm_gemm_small_batch_tiled", "aqlm_rotary_table",
           "aqlm_rope", "aqlm_rope_backward_workspace_bytes", "aqlm_rope_backward", "aqlm_paged_append",
           "aqlm_paged_attention_workspace_bytes", "aqlm_paged_attention", "aqlm_process_logits")
MAX_GROUPED = 8
PACKED = 0x100  # OR-ed into B: bit-packed codes
STEP_SYNC_BYTES = 256


class GemvProblem(ctypes.Structure):
    """Mirror of ``aqlm_gemv_problem`` in include/aqlm.h."""
    _fields_ = [("codes", ctypes.c_void_p), ("codebooks", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("d_out", ctypes.c_int64),
                ("d_in", ctypes.c_int64)]

class SortedProblem(ctypes.Structure):
    """Mirror of ``aqlm_sorted_problem`` in include/aqlm.h."""
    _fields_ = [("entries", ctypes.c_void_p), ("entry_words", ctypes.c_int64), ("index", ctypes.c_void_p),
                ("index_host", ctypes.c_void_p), ("codebooks", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("x", ctypes.c_void_p),
                ("y", ctypes.c_void_p), ("d_out", ctypes.c_int64), ("d_in", ctypes.c_int64)]


class Heads(ctypes.Structure):
    """Mirror of ``aqlm_heads`` in include/aqlm.h."""
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32)]


class Rotation(ctypes.Structure):
    """Mirror of ``aqlm_rotation`` in include/aqlm.h."""
    _fields_ = [("table", ctypes.c_void_p), ("rows", ctypes.c_int64), ("rot", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float)]


class PagedCache(ctypes.Structure):
    """Mirror of ``aqlm_paged_cache`` in include/aqlm.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_page_stride", ctypes.c_int64),
                ("k_slot_stride", ctypes.c_int64), ("k_head_stride", ctypes.c_int64), ("v_page_stride", ctypes.c_int64),
                ("v_slot_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64), ("pages", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("kv_lens", ctypes.c_void_p),
                ("cu_new", ctypes.c_void_p), ("table_width", ctypes.c_int32), ("seqs", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class LogitRules(ctypes.Structure):
    """Mirror of ``aqlm_logit_rules`` in include/aqlm.h."""
    _fields_ = [("tokens", ctypes.c_void_p), ("token_lens", ctypes.c_void_p), ("prompt_lens", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("token_stride", ctypes.c_int64), ("bias_stride", ctypes.c_int64), ("mask_stride", ctypes.c_int64),
                ("history", ctypes.c_int32), ("biases", ctypes.c_int32)]


class Norm(ctypes.Structure):
    """Mirror of ``aqlm_norm`` in include/aqlm.h."""
    _fields_ = [("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("rms", ctypes.c_int32)]


class Sampling(ctypes.Structure):
    """Mirror of ``aqlm_sampling`` in include/aqlm.h."""
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p)]


_lock = threading.Lock()
_lib = None


class AqlmError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {STATUS_NAMES.get(status, status)} ({status_string(status)})")


def load():
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2401_06118_amd.build` "
                "(hipcc, gfx950). There is no CPU fallback.")
        lib = ctypes.CDLL(LIB_PATH)
        p, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        lib.aqlm_dequantize.argtypes = [p, p, p, i64, i64, i32, i32, i32, p, p]
        lib.aqlm_dequantize.restype = ctypes.c_int
        lib.aqlm_gemv.argtypes = [p, p, p, i64, i64, i32, i32, i32, p, p, p]
        lib.aqlm_gemv.restype = ctypes.c_int
        lib.aqlm_gemv_grouped.argtypes = [ctypes.POINTER(GemvProblem), i32, i32, i32, i32, p]
        lib.aqlm_gemv_grouped.restype = ctypes.c_int
        lib.aqlm_gemv_grouped_path.argtypes = [ctypes.POINTER(GemvProblem), i32, i32, i32, i32, i32, p]
        lib.aqlm_gemv_grouped_path.restype = ctypes.c_int
        lib.aqlm_tiled_codes_bytes.argtypes = [i64, i64, i32, i32, i32]
        lib.aqlm_tiled_codes_bytes.restype = i64
        lib.aqlm_tile_codes.argtypes = [p, i64, i64, i32, i32, i32, p, i64, p]
        lib.aqlm_tile_codes.restype = ctypes.c_int
        lib.aqlm_gemv_grouped_tiled.argtypes = [ctypes.POINTER(GemvProblem), i32, i32, i32, i32, p]
        lib.aqlm_gemv_grouped_tiled.restype = ctypes.c_int
        lib.aqlm_gemm_small_batch_tiled.argtypes = [p, p, p, i64, i64, i32, i32, i32, i64, p, p, p]
        lib.aqlm_gemm_small_batch_tiled.restype = ctypes.c_int
        lib.aqlm_gemm_small_batch.argtypes = [p, p, p, i64, i64, i32, i32, i32, i64, p, p, p]
        lib.aqlm_gemm_small_batch.restype = ctypes.c_int
        lib.aqlm_gemm_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i64]
        lib.aqlm_gemm_workspace_bytes.restype = ctypes.c_size_t
        lib.aqlm_gemm.argtypes = [p, p, p, i64, i64, i32, i32, i32, i64, p, p, p, ctypes.c_size_t, p]
        lib.aqlm_gemm.restype = ctypes.c_int
        lib.aqlm_gemm_noalloc.argtypes = [p, p, p, i64, i64, i32, i32, i32, i64, p, p, p]
        lib.aqlm_gemm_noalloc.restype = ctypes.c_int
        lib.aqlm_backward.argtypes = [p, p, p, i64, i64, i32, i32, i32, i64, p, p, p, p, p]
        lib.aqlm_backward.restype = ctypes.c_int
        lib.aqlm_beam_search.argtypes = [p, p, p, p, p, i64, i64, i32, i32, i32, i32, i32, p, p]
        lib.aqlm_beam_search.restype = ctypes.c_int
        lib.aqlm_packed_row_words.argtypes = [i64, i32, i32, i32]
        lib.aqlm_packed_row_words.restype = ctypes.c_int64
        lib.aqlm_gemv_step_plan_bytes.argtypes = [i32]
        lib.aqlm_gemv_step_plan_bytes.restype = ctypes.c_int64
        lib.aqlm_gemv_step_plan.argtypes = [ctypes.POINTER(GemvProblem), ctypes.POINTER(ctypes.c_int32), i32, i32,
                                            i32, i32, p, i64]
        lib.aqlm_gemv_step_plan.restype = ctypes.c_int
        lib.aqlm_gemv_step.argtypes = [p, p, p, ctypes.c_uint32, p]
        lib.aqlm_gemv_step.restype = ctypes.c_int
        lib.aqlm_gemv_step_status.argtypes = [p, p]
        lib.aqlm_gemv_step_status.restype = ctypes.c_int
        lib.aqlm_sort_codes_size.argtypes = [p, i64, i64, i32, i32, i32, ctypes.POINTER(ctypes.c_int64),
                                             ctypes.POINTER(ctypes.c_int64)]
        lib.aqlm_sort_codes_size.restype = ctypes.c_int
        lib.aqlm_sort_codes.argtypes = [p, i64, i64, i32, i32, i32, p, i64, p, i64]
        lib.aqlm_sort_codes.restype = ctypes.c_int
        lib.aqlm_gemv_sorted_workspace_bytes.argtypes = [i64, i32, i32]
        lib.aqlm_gemv_sorted_workspace_bytes.restype = ctypes.c_size_t
        lib.aqlm_gemv_sorted.argtypes = [p, i64, p, p, p, p, i64, i64, i32, i32, i32, p, p, p, ctypes.c_size_t, p]
        lib.aqlm_gemv_sorted.restype = ctypes.c_int
        lib.aqlm_gemv_sorted_grouped.argtypes = [ctypes.POINTER(SortedProblem), i32, i32, i32, i32, p,
                                                 ctypes.c_size_t, p]
        lib.aqlm_gemv_sorted_grouped.restype = ctypes.c_int
        heads, rotation, cache = (ctypes.POINTER(t) for t in (Heads, Rotation, PagedCache))
        lib.aqlm_rotary_table.argtypes = [p, i64, i32, ctypes.c_double, p, p]
        lib.aqlm_rotary_table.restype = ctypes.c_int
        lib.aqlm_rope.argtypes = [heads, heads, heads, heads, i32, i64, i32, p, rotation, p]
        lib.aqlm_rope.restype = ctypes.c_int
        lib.aqlm_rope_backward_workspace_bytes.argtypes = [i32]
        lib.aqlm_rope_backward_workspace_bytes.restype = ctypes.c_size_t
        lib.aqlm_rope_backward.argtypes = [heads, heads, heads, heads, heads, heads, p, p, i32, i64, i32, p, rotation,
                                           p, ctypes.c_size_t, p]
        lib.aqlm_rope_backward.restype = ctypes.c_int
        lib.aqlm_paged_append.argtypes = [heads, heads, heads, heads, cache, i64, rotation, p]
        lib.aqlm_paged_append.restype = ctypes.c_int
        lib.aqlm_paged_attention_workspace_bytes.argtypes = [i32]
        lib.aqlm_paged_attention_workspace_bytes.restype = ctypes.c_size_t
        lib.aqlm_paged_attention.argtypes = [heads, heads, p, cache, i64, i64, ctypes.c_float, i32, i32, p,
                                             ctypes.c_size_t, p]
        lib.aqlm_paged_attention.restype = ctypes.c_int
        lib.aqlm_process_logits.argtypes = [p, i64, p, i64, i32, i64, i64, ctypes.POINTER(LogitRules), p]
        lib.aqlm_process_logits.restype = ctypes.c_int
        f32, size = ctypes.c_float, ctypes.c_size_t
        lib.aqlm_embed.argtypes = [p, i64, p, p, i64, i32, i64, i64, i64, f32, p]
        lib.aqlm_embed.restype = ctypes.c_int
        lib.aqlm_embed_backward_workspace_bytes.argtypes = [i64, i64, i64, i32]
        lib.aqlm_embed_backward_workspace_bytes.restype = size
        lib.aqlm_embed_backward.argtypes = [p, i64, p, p, i64, i32, i32, i64, i64, i64, f32, p, size, p]
        lib.aqlm_embed_backward.restype = ctypes.c_int
        lib.aqlm_layer_norm.argtypes = [p, i64, p, i64, p, i64, p, i64, i32, i64, i64, ctypes.POINTER(Norm), p]
        lib.aqlm_layer_norm.restype = ctypes.c_int
        lib.aqlm_layer_norm_backward_workspace_bytes.argtypes = [i64]
        lib.aqlm_layer_norm_backward_workspace_bytes.restype = size
        lib.aqlm_layer_norm_backward.argtypes = [p, i64, p, i64, p, i64, p, i64, p, p, i32, i64, i64,
                                                 ctypes.POINTER(Norm), p, size, p]
        lib.aqlm_layer_norm_backward.restype = ctypes.c_int
        lib.aqlm_distill_loss_workspace_bytes.argtypes = [i64, i64, i64, i32]
        lib.aqlm_distill_loss_workspace_bytes.restype = size
        lib.aqlm_distill_loss.argtypes = [p, i64, i32, p, i64, i32, p, i64, p, p, f32, p, p, i64, i64, i64, i64, p, size,
                                          p]
        lib.aqlm_distill_loss.restype = ctypes.c_int
        lib.aqlm_sample_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(Sampling)]
        lib.aqlm_sample_workspace_bytes.restype = size
        lib.aqlm_sample.argtypes = [p, i64, i32, i64, i64, p, ctypes.POINTER(Sampling), p, p, p, size, p]
        lib.aqlm_sample.restype = ctypes.c_int
        lib.aqlm_status_string.argtypes = [ctypes.c_int]
        lib.aqlm_status_string.restype = ctypes.c_char_p
        _lib = lib
        return lib


def status_string(status: int) -> str:
    try:
        return load().aqlm_status_string(int(status)).decode()
    except RuntimeError:
        return STATUS_NAMES.get(status, "unknown")
