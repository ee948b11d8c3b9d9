"""ctypes declarations for libcaddtree.so (the C ABI in include/caddtree.h)."""

from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcaddtree.so")

OK, E_INVALID, E_UNSUPPORTED, E_COST, E_WORKSPACE, E_HIP = range(6)
DTYPES = {"f32": 0, "bf16": 1}
ATTENTION_DTYPES = {"bf16": 1, "f16": 2}
LOGIT_DTYPES = {"f32": 0, "bf16": 1, "f16": 2}
ORDERS = {"chain": 0, "block": 1, "tree": 2}
MASKS = {"none": 0, "u8": 1, "bits": 2}
ALLOW_NONCONVEX = 1
FIXED_BUDGET = 2
MAX_L, MAX_K, MAX_CAP, MAX_CTX = 32, 16, 4096, 64
NOALLOC_SCRATCH_BYTES = 8 << 20


class CaddtreeError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"caddtree status {status}: {message}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [
        ("L", ctypes.c_int32),
        ("V", ctypes.c_int64),
        ("K", ctypes.c_int32),
        ("budget_cap", ctypes.c_int32),
        ("dtype", ctypes.c_int),
        ("mask", ctypes.c_int),
        ("flags", ctypes.c_uint32),
        ("t_draft", ctypes.c_double),
        ("t_verify_host", ctypes.POINTER(ctypes.c_double)),
        ("n_ctx", ctypes.c_int32),
        ("ctx_grid_host", ctypes.POINTER(ctypes.c_int64)),
    ]


class Outputs(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in (
        "token_ids", "parent", "depth", "path_prob", "n_star", "phi", "theta",
        "mask", "pos_ids", "topk_ids", "topk_logit", "topk_lq", "lse")]


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64),
                ("stride_h", ctypes.c_int64)]


class Cache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_pages", ctypes.c_int64), ("pages", ctypes.c_void_p)]


class Attention(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int),
        *((n, ctypes.c_int32) for n in ("B", "T", "S", "n_heads", "n_kv_heads", "head_dim")),
        *((n, View) for n in ("q", "k", "v", "out")),
        *((n, ctypes.c_void_p) for n in ("lse", "q_len", "k_len")),
        ("scale", ctypes.c_float),
        *((n, ctypes.c_int32) for n in ("window", "sinks")),
        ("order", ctypes.c_int),
        ("mask_kind", ctypes.c_int),
        *((n, ctypes.c_void_p) for n in ("mask", "depth")),
        ("cap", ctypes.c_int32),
        ("page_table", ctypes.c_void_p),
        ("table_pages", ctypes.c_int32),
        ("ctx_len", ctypes.c_void_p),
        ("lse_strided", ctypes.c_int32),
        *((n, ctypes.c_int64) for n in ("lse_stride_b", "lse_stride_t", "lse_stride_h")),
    ]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64)]


_SIZES = [("dtype", ctypes.c_int), *((n, ctypes.c_int32) for n in ("B", "T", "V"))]


class Adjust(ctypes.Structure):
    _fields_ = _SIZES + [
        ("logits", Rows), ("out", Rows),
        *((n, ctypes.c_void_p) for n in ("count", "history", "history_len")),
        ("H", ctypes.c_int32),
        *((n, ctypes.c_void_p) for n in ("repetition", "presence", "frequency", "bias_ids", "bias")),
        ("n_bias", ctypes.c_int32),
        ("allowed", ctypes.c_void_p), ("allowed_stride_b", ctypes.c_int64), ("allowed_stride_t", ctypes.c_int64),
        *((n, ctypes.c_void_p) for n in ("token_ids", "parent")),
        ("fill", ctypes.c_float),
    ]


class Verify(ctypes.Structure):
    _fields_ = _SIZES + [
        ("logits", Rows),
        *((n, ctypes.c_void_p) for n in ("chosen", "token_ids", "parent", "count")),
        ("M", ctypes.c_int32),
        *((n, ctypes.c_void_p) for n in ("accepted", "index", "tokens", "weight")),
    ]


class Distill(ctypes.Structure):
    _fields_ = _SIZES + [
        ("logits", Rows),
        ("K", ctypes.c_int32),
        *((n, ctypes.c_void_p) for n in ("ids", "target", "weight")),
        ("temperature", ctypes.c_float),
        ("tail", ctypes.c_int32),
        *((n, ctypes.c_void_p) for n in ("loss", "stats")),
        ("grad", Rows),
    ]


EXPORTS = [
    "caddtree_plan_create", "caddtree_plan_destroy", "caddtree_workspace_bytes", "caddtree_build",
    "caddtree_build_noalloc",
    "caddtree_reduce_topk", "caddtree_expand", "caddtree_emit", "caddtree_accept", "caddtree_fit_cost", "caddtree_status_string",
    "caddtree_last_error",
    "caddtree_attention_workspace_bytes", "caddtree_window_attention", "caddtree_cache_attention",
    "caddtree_cache_write", "caddtree_cache_read", "caddtree_cache_score", "caddtree_cache_evict",
    "caddtree_evict_workspace_bytes",
    "caddtree_adjust_logits", "caddtree_verify_tree", "caddtree_verify_workspace_bytes",
    "caddtree_distill", "caddtree_distill_grad", "caddtree_distill_workspace_bytes",
]


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build the HIP library first (python -m paper_2606_01813_amd._build)")
    # PyTorch-ROCm ships its own HIP runtime under the same soname (libamdhip64.so.7).  Importing
    # torch first makes this library bind to that runtime, so the tensors' memory and streams and
    # the kernels share one runtime; in the other order torch would later find no GPU.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.caddtree_plan_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(vp)]
    lib.caddtree_plan_create.restype = ctypes.c_int
    lib.caddtree_plan_destroy.argtypes = [vp]
    lib.caddtree_plan_destroy.restype = None
    lib.caddtree_workspace_bytes.argtypes = [vp, i64]
    lib.caddtree_workspace_bytes.restype = sz
    lib.caddtree_build.argtypes = [vp, vp, i64, i64, i32, vp, ctypes.POINTER(Outputs), vp, sz, vp]
    lib.caddtree_build.restype = ctypes.c_int
    lib.caddtree_build_noalloc.argtypes = [vp, vp, i64, i64, i32, vp, ctypes.POINTER(Outputs), vp]
    lib.caddtree_build_noalloc.restype = ctypes.c_int
    lib.caddtree_reduce_topk.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp]
    lib.caddtree_reduce_topk.restype = ctypes.c_int
    lib.caddtree_expand.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.caddtree_expand.restype = ctypes.c_int
    lib.caddtree_emit.argtypes = [vp, vp, vp, vp, i64, i32, vp, vp, vp]
    lib.caddtree_emit.restype = ctypes.c_int
    lib.caddtree_accept.argtypes = [vp, vp, vp, vp, i64, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.caddtree_accept.restype = ctypes.c_int
    lib.caddtree_fit_cost.argtypes = [vp, vp, i64, vp, i32, vp]
    lib.caddtree_fit_cost.restype = ctypes.c_int
    ap, cp, wp = ctypes.POINTER(Attention), ctypes.POINTER(Cache), ctypes.POINTER(View)
    lib.caddtree_attention_workspace_bytes.argtypes = [ap]
    lib.caddtree_attention_workspace_bytes.restype = sz
    lib.caddtree_window_attention.argtypes = [ap, vp, sz, vp]
    lib.caddtree_window_attention.restype = ctypes.c_int
    lib.caddtree_cache_attention.argtypes = [cp, ap, vp, sz, vp]
    lib.caddtree_cache_attention.restype = ctypes.c_int
    lib.caddtree_cache_write.argtypes = [cp, wp, wp, i32, i32, i32, vp, vp, vp, vp, i32, vp]
    lib.caddtree_cache_write.restype = ctypes.c_int
    lib.caddtree_cache_read.argtypes = [cp, wp, wp, i32, i32, vp, vp, vp, i32, vp]
    lib.caddtree_cache_read.restype = ctypes.c_int
    lib.caddtree_cache_score.argtypes = [cp, ap, vp, vp, vp, i64, vp]
    lib.caddtree_cache_score.restype = ctypes.c_int
    lib.caddtree_cache_evict.argtypes = [cp, i32, vp, i32, vp, vp, i64, i32, i32, i32, vp, i32, vp, i64, vp, vp, vp, sz, vp]
    lib.caddtree_cache_evict.restype = ctypes.c_int
    lib.caddtree_evict_workspace_bytes.argtypes = [cp, i32, i32, i64]
    lib.caddtree_evict_workspace_bytes.restype = sz
    xp, tp, dp = ctypes.POINTER(Adjust), ctypes.POINTER(Verify), ctypes.POINTER(Distill)
    lib.caddtree_adjust_logits.argtypes = [xp, vp]
    lib.caddtree_adjust_logits.restype = ctypes.c_int
    lib.caddtree_verify_tree.argtypes = [tp, vp, sz, vp]
    lib.caddtree_verify_tree.restype = ctypes.c_int
    lib.caddtree_verify_workspace_bytes.argtypes = [tp]
    lib.caddtree_verify_workspace_bytes.restype = sz
    lib.caddtree_distill.argtypes = [dp, vp, sz, vp]
    lib.caddtree_distill.restype = ctypes.c_int
    lib.caddtree_distill_grad.argtypes = [dp, vp]
    lib.caddtree_distill_grad.restype = ctypes.c_int
    lib.caddtree_distill_workspace_bytes.argtypes = [dp]
    lib.caddtree_distill_workspace_bytes.restype = sz
    lib.caddtree_status_string.argtypes = [ctypes.c_int]
    lib.caddtree_status_string.restype = ctypes.c_char_p
    lib.caddtree_last_error.argtypes = []
    lib.caddtree_last_error.restype = ctypes.c_char_p
    return lib


_LIB = None


def lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        _LIB = load()
    return _LIB


def check(status: int) -> None:
    if status != OK:
        msg = lib().caddtree_last_error().decode(errors="replace")
        name = lib().caddtree_status_string(status).decode()
        raise CaddtreeError(status, f"{name}: {msg}")


_BINDING = None


def binding():
    """The native calls of the binding (csrc/binding.cpp); None where they were not built."""
    global _BINDING
    if _BINDING is None and os.path.exists(os.path.join(_HERE, "_binding.so")):
        import torch  # noqa: F401  (the module uses torch's libraries)
        from . import _binding
        _BINDING = _binding
    return _BINDING


def call_spec(lib_, handle: int, device: int, L: int, V: int, K: int, cap: int, dtype: str, mask: str):
    """What the native calls need of a plan: its handle, the shapes of its tensors and the library's functions.
    None where the native calls were not built."""
    if binding() is None:
        return None
    fns = (lib_.caddtree_build, lib_.caddtree_build_noalloc, lib_.caddtree_reduce_topk, lib_.caddtree_expand,
           lib_.caddtree_emit, lib_.caddtree_accept)
    return binding().spec(handle, device, L, V, K, cap, DTYPES[dtype], MASKS[mask],
                          *(ctypes.cast(f, ctypes.c_void_p).value for f in fns))


_OPS = None


def attention_ops():
    """The native attention and cache calls: the binding and the library's functions for it, or None where the
    native calls were not built."""
    global _OPS
    if _OPS is None and binding() is not None:
        l = lib()
        fns = (l.caddtree_window_attention, l.caddtree_cache_attention, l.caddtree_cache_write, l.caddtree_cache_read,
               l.caddtree_cache_score, l.caddtree_cache_evict)
        _OPS = binding(), binding().ops(0, *(ctypes.cast(f, ctypes.c_void_p).value for f in fns))
    return _OPS


_LOGITS_OPS = None


def logits_ops():
    """The native calls on logits, as attention_ops: the library's functions for the binding, or None."""
    global _LOGITS_OPS
    if _LOGITS_OPS is None and binding() is not None:
        l = lib()
        fns = (l.caddtree_adjust_logits, l.caddtree_verify_tree, l.caddtree_distill, l.caddtree_distill_grad)
        _LOGITS_OPS = binding().logits_ops(0, *(ctypes.cast(f, ctypes.c_void_p).value for f in fns))
    return _LOGITS_OPS
