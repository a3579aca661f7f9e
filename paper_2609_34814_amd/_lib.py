"""ctypes declarations of libwavealign.so (the C ABI in include/wavealign.h)."""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import POINTER, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libwavealign.so")

WA_OK = 0
WA_ERR_INVALID_ARG = -1
WA_ERR_UNSUPPORTED = -2
WA_ERR_ALIGNMENT = -3
WA_ERR_WORKSPACE = -4
WA_ERR_INVALID_PERM = -5
WA_ERR_HIP = -6

WA_SKIP_AUTO, WA_SKIP_NEVER, WA_SKIP_ALWAYS = 0, 1, 2
FLAG_FITS_CACHE, FLAG_LITTLE_WORK, FLAG_LOCAL, FLAG_UNSTRUCTURED, FLAG_DEGENERATE, FLAG_IDENTITY = 1, 2, 4, 8, 16, 64
WA_ATTN_BAD_PERM, WA_ATTN_BAD_KV_INDEX = 1, 2
WA_PRODUCE_WAIT_EXPIRED = 1
WA_HEADS_IN_ORDER, WA_HEADS_INTERLEAVED = 0, 1
WA_NOALLOC_SCRATCH_BYTES = 4 * 1024 * 1024
WA_BF16, WA_F16, WA_F32 = 0, 1, 2
WA_PAGE_BAD_INDEX, WA_PAGE_EXHAUSTED, WA_PAGE_BUSY = 1, 2, 4
WA_ROTARY_HALF, WA_ROTARY_INTERLEAVED = 0, 1
WA_ROTARY_PLAIN, WA_ROTARY_LINEAR, WA_ROTARY_NTK, WA_ROTARY_YARN = 0, 1, 2, 3


class WaShape(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("heads", c_int32), ("seq_len", c_int32), ("head_dim", c_int32),
                ("block", c_int32)]


class WaSkipProfile(ctypes.Structure):
    _fields_ = [("cache_bytes", c_double), ("gain_ns_per_block", c_double), ("ovh_ns_fixed", c_double),
                ("ovh_ns_per_row", c_double), ("ovh_ns_per_nnz", c_double), ("j_max", c_double),
                ("eta_min", c_double), ("fused_max_blocks", c_double), ("ovh_fused_ns_fixed", c_double),
                ("ovh_fused_ns_per_row", c_double), ("ovh_fused_ns_per_nnz", c_double)]


class WaPermParams(ctypes.Structure):
    _fields_ = [("wave_per_xcd", c_int32), ("n_xcd", c_int32), ("iters", c_int32), ("skip_mode", c_int32),
                ("seed", c_uint64), ("profile", POINTER(WaSkipProfile))]


class WaAttnOptions(ctypes.Structure):
    _fields_ = [("softmax_scale", c_float), ("n_xcd", c_int32), ("head_order", c_int32)]


class WaRotaryParams(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("tokens", c_int32), ("head_dim", c_int32), ("dtype", c_int32), ("layout", c_int32),
                ("pairs", c_int32), ("axes", c_int32), ("axis_pairs", c_int32 * 3), ("position_batch", c_int32),
                ("backward", c_int32), ("scale", c_double)]


class WaRotaryTensor(ctypes.Structure):
    _fields_ = [("inp", c_void_p), ("out", c_void_p), ("heads", c_int32), ("in_stride", c_int64 * 3),
                ("out_stride", c_int64 * 3)]


class WaRotaryScaling(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("factor", c_double), ("original_len", c_double), ("beta_fast", c_double),
                ("beta_slow", c_double)]


# The two rotary structures as bytes, laid out as above (a call of one token costs about as much host time as its structures
# built field by field: 2.7 us, 0.4 packed).
ROTARY_PARAMS = struct.Struct("@12id")
ROTARY_TENSOR = struct.Struct("@PPi4x6q")


class WaDiffShape(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("heads", c_int32), ("kv_heads", c_int32), ("q_len", c_int32), ("kv_len", c_int32),
                ("head_dim", c_int32), ("value_dim", c_int32), ("block", c_int32)]


class WaDiffOptions(ctypes.Structure):
    _fields_ = [("softmax_scale", c_float), ("causal", c_int32)]


# The structures of packed sequences and of the paged cache as bytes (see ROTARY_PARAMS): wa_token_rows, wa_seq_shape, wa_seq_options,
# wa_pages, wa_page_tables, wa_page_state, wa_page_pool.
TOKEN_ROWS = struct.Struct("@Pqq")
SEQ_SHAPE = struct.Struct("@6i")
SEQ_OPTIONS = struct.Struct("@fi")
PAGES = struct.Struct("@Pqqq")
PAGE_TABLES = struct.Struct("@Pq3i4x")
PAGE_STATE = struct.Struct("@3P4i")
PAGE_POOL = struct.Struct("@Pqi4x")


class WaError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"wavealign error {status}: {detail}")
        self.status = status


_SIGNATURES = {
    "wa_abi_version": (c_int32, []),
    "wa_status_string": (c_char_p, [c_int32]),
    "wa_last_error": (c_char_p, []),
    "wa_default_skip_profile": (c_int32, [POINTER(WaSkipProfile)]),
    "wa_wave_size": (c_int32, [c_int32, c_int32, POINTER(c_int32)]),
    "wa_mask_stats": (c_int32, [c_void_p, POINTER(WaShape), c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                c_void_p]),
    "wa_perm_workspace_size": (c_int32, [POINTER(WaShape), POINTER(c_size_t)]),
    "wa_build_permutation": (c_int32, [c_void_p, POINTER(WaShape), POINTER(WaPermParams), c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "wa_compact_mask": (c_int32, [c_void_p, POINTER(WaShape), c_void_p, c_void_p, c_void_p]),
    "wa_mask_producer_workspace_size": (c_int32, [POINTER(WaShape), POINTER(c_size_t)]),
    "wa_check_perm_workspace_size": (c_int32, [POINTER(WaShape), POINTER(c_size_t)]),
    "wa_check_perm": (c_int32, [c_void_p, POINTER(WaShape), c_void_p, c_void_p, c_size_t, c_void_p]),
    "wa_produce_block_mask": (c_int32, [c_void_p, c_void_p, POINTER(WaShape), c_int32, c_int32, c_void_p, c_void_p,
                                        c_void_p, c_void_p, c_size_t, c_void_p]),
    "wa_attn_workspace_size": (c_int32, [POINTER(WaShape), POINTER(c_size_t)]),
    "wa_attn_split_workspace_size": (c_int32, [POINTER(WaShape), POINTER(c_size_t)]),
    "wa_sparse_attn": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, POINTER(WaShape),
                                 c_float, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "wa_sparse_attn_csr": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                     POINTER(WaShape), c_float, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                     c_size_t, c_void_p]),
    "wa_sparse_attn_vt_noalloc": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                            POINTER(WaShape), POINTER(WaAttnOptions), c_void_p, c_void_p, c_void_p,
                                            c_void_p]),
    "wa_transpose_v": (c_int32, [c_void_p, POINTER(WaShape), c_void_p, c_void_p]),
    "wa_attn_vt_workspace_size": (c_int32, [POINTER(WaShape), POINTER(c_size_t)]),
    "wa_sparse_attn_vt": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                    POINTER(WaShape), POINTER(WaAttnOptions), c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_size_t, c_void_p]),
    "wa_rotary": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p]),
    "wa_rotary_frequencies": (c_int32, [c_int32, c_double, POINTER(WaRotaryScaling), c_void_p, c_void_p]),
    "wa_diff_attn_workspace_size": (c_int32, [POINTER(WaDiffShape), POINTER(c_size_t)]),
    "wa_diff_attn": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                               POINTER(WaDiffShape), POINTER(WaDiffOptions), c_void_p, c_void_p, c_void_p, c_void_p,
                               c_size_t, c_void_p]),
    "wa_diff_attn_backward_workspace_size": (c_int32, [POINTER(WaDiffShape), POINTER(c_size_t)]),
    "wa_diff_attn_backward": (c_int32, [c_void_p] * 10 + [POINTER(WaDiffShape), POINTER(WaDiffOptions)] + [c_void_p] * 5
                              + [c_size_t, c_void_p]),
    "wa_seq_attn_workspace_size": (c_int32, [c_void_p, POINTER(c_size_t)]),
    "wa_packed_attn": (c_int32, [c_void_p] * 9 + [c_size_t, c_void_p]),
    "wa_packed_attn_backward_workspace_size": (c_int32, [c_void_p, POINTER(c_size_t)]),
    "wa_packed_attn_backward": (c_int32, [c_void_p] * 13 + [c_size_t, c_void_p]),
    "wa_paged_attn": (c_int32, [c_void_p] * 12 + [c_size_t, c_void_p]),
    "wa_page_store": (c_int32, [c_void_p] * 10),
    "wa_page_workspace_size": (c_int32, [c_void_p, c_int32, POINTER(c_size_t)]),
    "wa_page_grow": (c_int32, [c_void_p] * 4 + [c_size_t, c_void_p]),
    "wa_page_fork": (c_int32, [c_void_p] * 4 + [c_int32, c_void_p, c_void_p, c_size_t, c_void_p]),
    "wa_page_free": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p, c_void_p]),
    "wa_page_compact": (c_int32, [c_void_p] * 7 + [c_size_t, c_void_p]),
    "wa_page_copy": (c_int32, [c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_void_p]),
    "wa_fp64_probe": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_void_p]),
    "wa_xcc_probe": (c_int32, [c_void_p, c_int32, c_void_p]),
}

_LIB = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built (there is no fallback)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2609_34814_amd.build` "
                          "(the path has no CPU fallback)")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def check(status: int) -> None:
    if status != WA_OK:
        lib = load()
        raise WaError(status, (lib.wa_last_error() or b"").decode())
