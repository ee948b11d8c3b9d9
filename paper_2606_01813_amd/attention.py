"""Verification: attention over a built tree, the 4-bit cache it reads, windowed attention, eviction.

After ``Plan.build`` the target verifies the tree: its queries are the root (bonus token) and the nodes,
and each sees the cached context, the root, its ancestors and itself.

    cache = KVCache(n_kv_heads=8, head_dim=128, num_pages=4096)          # bf16 keys and values, kept in 4 bits
    out = window_attention(q, k, v, window=4096, sinks=4)                # a prompt, [B, T, heads, 128]
    cache.write(k, v, table, start)                                      # ... goes into the cache
    plan.build(logits, tree, workspace=ws, ctx_len=ctx_len)              # a draft tree
    aws = attention_workspace(q, cache=cache, page_table=table)          # (without one, a row's keys stay in one part)
    o = cache.attention(q, table, ctx_len, k, v, mask=tree.mask, depth=tree.depth, count=tree.n_star, lse=lse, workspace=aws)
    cache.write(k, v, table, ctx_len, count=accepted, index=path)        # the accepted path
    cache.score(q, table, ctx_len, lse, scores, weight=on_path, count=tree.n_star, depth=tree.depth)
    cache.evict(table, ctx_len, scores, new_table, new_len, new_scores, kept, budget=2048, sinks=4, recent=256)

Every call checks its tensors, then enqueues kernels on the stream (default: torch's current one) and
returns; lengths and page tables stay on the device.  include/caddtree.h states what is computed.  Nothing here has
a backward pass: queries, keys and values that require a gradient are refused while gradients are recorded.

As a plan's calls do, these go to the native binding first, which checks the tensors and calls the library
(about 2 us of host time where the checks here take 10 to 15); what it cannot vouch for comes back as None
and takes the Python checks here, which raise what is wrong.
"""

from __future__ import annotations

import ctypes
import math
from typing import Optional

from . import _lib

__all__ = ["KVCache", "window_attention", "attention_workspace"]


def _torch():
    import torch
    return torch


def _on_device(t, device: int) -> bool:
    return bool(t.is_cuda) and t.device.index == device


def _dtype_name(dtype) -> str:
    torch = _torch()
    if dtype == torch.bfloat16:
        return "bf16"
    if dtype == torch.float16:
        return "f16"
    raise TypeError(f"queries, keys and values must be torch.bfloat16 or torch.float16, got {dtype}")


def _device() -> int:
    return _torch().cuda.current_device()


def _stream(stream, device: int) -> int:
    if stream is None:
        return _torch()._C._cuda_getCurrentRawStream(device)
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _native(stream):
    """(binding, its functions, device, raw stream) of the native calls, or None where the Python path is to
    decide."""
    ops = _lib.attention_ops()
    if ops is None:
        return None
    torch = _torch()
    device = torch._C._cuda_getDevice()
    if stream is None:
        return ops[0], ops[1], device, torch._C._cuda_getCurrentRawStream(device)
    return (ops[0], ops[1], device, stream.cuda_stream) if isinstance(stream, torch.cuda.Stream) else None


def _done(status) -> bool:
    """Whether a native call was made; raises its error."""
    if status is None:
        return False
    if status:
        _lib.check(status)
    return True


def _made(q, out, stream):
    """out, or where it is not given a new one (of zeros, on the call's stream: rows without a query keep them)."""
    torch = _torch()
    if out is not None or not isinstance(q, torch.Tensor):
        return out
    if stream is None:
        return torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    if not hasattr(stream, "cuda_stream"):
        raise ValueError("out is required with a raw stream handle")
    with torch.cuda.stream(stream):
        return torch.zeros(q.shape, dtype=q.dtype, device=q.device)


def _no_gradient(**inputs) -> None:
    torch = _torch()
    if torch.is_grad_enabled():
        for name, t in inputs.items():
            if isinstance(t, torch.Tensor) and t.requires_grad:
                raise ValueError(f"{name} requires a gradient, and attention has no backward pass: call it under "
                                 f"torch.no_grad(), or detach {name}")


def _tensor(name: str, t, dtype, device: int):
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor, got {type(t).__name__}")
    if not _on_device(t, device):
        raise ValueError(f"{name} must be on cuda:{device} (the current device), got {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _int32(name: str, n) -> int:
    """n as the 32-bit integer that the library takes: a larger one would lose its upper bits on the way."""
    i = int(n)
    if i != n or not -2 ** 31 <= i < 2 ** 31:
        raise ValueError(f"{name} must be an integer below 2^31, got {n}")
    return i


def _sizes(name: str, t) -> None:
    if any(n >= 2 ** 31 for n in t.shape):
        raise ValueError(f"{name} must have sizes below 2^31, got {tuple(t.shape)}")


def _array(name: str, t, dtype, shape, device: int, contiguous: bool = True) -> int:
    """The pointer of a tensor of exactly this shape (None in a place: any size), contiguous unless that is not asked."""
    _tensor(name, t, dtype, device)
    if t.dim() != len(shape) or any(w is not None and w != g for w, g in zip(shape, t.shape)):
        raise ValueError(f"{name} must have shape {tuple('any' if w is None else w for w in shape)}, got {tuple(t.shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    _sizes(name, t)
    return t.data_ptr()


def _view(name: str, t, dtype, shape, device: int) -> _lib.View:
    """A [B, tokens, heads, head_dim] tensor with a unit last stride, 16-byte aligned rows."""
    _tensor(name, t, dtype, device)
    if t.dim() != 4 or any(w is not None and w != g for w, g in zip(shape, t.shape)):
        raise ValueError(f"{name} must have shape {tuple('any' if w is None else w for w in shape)}, got {tuple(t.shape)}")
    _sizes(name, t)
    sb, st, sh, sd = t.stride()
    n = t.shape
    sb, st, sh = (s if m > 1 else 0 for s, m in zip((sb, st, sh), n))     # the stride of one element is free
    if sd != 1 and n[3] > 1 or (sb | st | sh) % 8 or t.data_ptr() % 16:
        raise ValueError(f"{name} must have a unit last stride, the others multiples of 8, and be 16-byte aligned; "
                         f"got strides {t.stride()}")
    return _lib.View(t.data_ptr(), sb, st, sh)


def _output(name: str, t, dtype, shape, device: int) -> _lib.View:
    """As _view, and no two elements in one place."""
    v = _view(name, t, dtype, shape, device)
    dims = sorted((s, n) for s, n in zip((v.stride_b, v.stride_t, v.stride_h), t.shape) if n > 1)
    room = t.shape[3]
    for s, n in dims:
        if s < room:
            raise ValueError(f"{name} must not overlap itself, got strides {t.stride()}")
        room = s * (n - 1) + room
    return v


def _scale(scale, head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim) if scale is None else float(scale)


def _workspace(workspace, device: int):
    if workspace is None:
        return None, 0
    if not isinstance(workspace, _torch().Tensor) or not _on_device(workspace, device) or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _queries(q, device: int):
    """(attention arguments with what the queries say, their dtype's name)"""
    torch = _torch()
    if not isinstance(q, torch.Tensor):
        raise TypeError(f"q must be a torch tensor, got {type(q).__name__}")
    name = _dtype_name(q.dtype)
    a = _lib.Attention()
    a.q = _view("q", q, q.dtype, (None,) * 4, device)
    a.dtype = _lib.ATTENTION_DTYPES[name]
    a.B, a.T, a.n_heads, a.head_dim = q.shape
    return a, name


def _results(q, out, lse, a, device: int) -> None:
    a.out = _output("out", out, q.dtype, tuple(q.shape), device)
    if lse is not None:
        a.lse = _array("lse", lse, _torch().float32, tuple(q.shape[:3]), device)


def window_attention(q, k, v, *, window: int = 0, sinks: int = 0, causal: bool = True, scale: Optional[float] = None,
                     q_len=None, k_len=None, out=None, lse=None, workspace=None, stream=None):
    """Attention of q [B, T, heads, D] over k, v [B, S, kv heads, D], the queries being the last positions
    (query i of a sequence at k_len - q_len + i; lengths int32 [B], default T and S).  A query sees the
    last ``window`` positions (0: all) and the first ``sinks``; ``causal=False`` lets it see later keys too.
    Writes ``out`` (made of zeros if not given) and ``lse`` (float32 [B, T, heads], if given); rows past
    q_len are left as they are.  Returns out."""
    out = _made(q, out, stream)
    native = _native(stream)
    if native is not None:
        binding, ops, device, raw = native
        if _done(binding.window_attention(ops, device, raw, q, k, v, window, sinks, causal, scale, q_len, k_len, out, lse, workspace)):
            return out
    _no_gradient(q=q, k=k, v=v)
    torch = _torch()
    device = _device()
    a, _ = _queries(q, device)
    if not isinstance(k, torch.Tensor):
        raise TypeError(f"k must be a torch tensor, got {type(k).__name__}")
    shape = (a.B, k.shape[1] if k.dim() == 4 else None, k.shape[2] if k.dim() == 4 else None, a.head_dim)
    a.k = _view("k", k, q.dtype, shape, device)
    a.v = _view("v", v, q.dtype, shape, device)
    a.S, a.n_kv_heads = shape[1], shape[2]
    a.scale, a.window, a.sinks = _scale(scale, a.head_dim), _int32("window", window), _int32("sinks", sinks)
    a.order = _lib.ORDERS["chain" if causal else "block"]
    if q_len is not None:
        a.q_len = _array("q_len", q_len, torch.int32, (a.B,), device)
    if k_len is not None:
        a.k_len = _array("k_len", k_len, torch.int32, (a.B,), device)
    _results(q, out, lse, a, device)
    ws, n = _workspace(workspace, device)
    _lib.check(_lib.lib().caddtree_window_attention(ctypes.byref(a), ws, n, _stream(stream, device)))
    return out


def attention_workspace(q, k=None, cache: Optional["KVCache"] = None, page_table=None):
    """A workspace for ``window_attention`` of these q and k, or for ``cache.attention`` of these q and
    page_table (uint8, as large as any call of these shapes uses; the contents do not matter)."""
    torch = _torch()
    a = _lib.Attention()
    for name, t in (("q", q), ("k", k), ("page_table", page_table)):
        if t is not None:
            _sizes(name, t)
    a.B, a.T, a.n_heads, a.head_dim = q.shape
    a.dtype = _lib.ATTENTION_DTYPES[_dtype_name(q.dtype)]
    if cache is not None:
        a.n_kv_heads, a.S, a.table_pages = cache.n_kv_heads, a.T, page_table.shape[1]
    else:
        a.n_kv_heads, a.S = k.shape[2], k.shape[1]
    n = int(_lib.lib().caddtree_attention_workspace_bytes(ctypes.byref(a)))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=q.device)


class KVCache:
    """A paged cache of keys and values in 4 bits (see caddtree_cache_t for the layout of a page).

    ``pages`` is a uint8 tensor [num_pages, n_kv_heads, page_bytes(head_dim)], the caller's or made here
    (of zeros).  Which pages a sequence has is the caller's to say: page tables are int32 [B, pages per
    sequence], slot t of sequence b being token t % 64 of page table[b, t // 64].  Lengths (ctx_len, start,
    end, new_len) are int64 [B], counts int32 [B], as ``Plan.build`` reads and writes them."""

    def __init__(self, n_kv_heads: int, head_dim: int, num_pages: Optional[int] = None, dtype: str = "bf16",
                 pages=None, device=None):
        torch = _torch()
        if dtype not in _lib.ATTENTION_DTYPES:
            raise ValueError(f"dtype must be one of {sorted(_lib.ATTENTION_DTYPES)}")
        self.n_kv_heads, self.head_dim, self.dtype = _int32("n_kv_heads", n_kv_heads), _int32("head_dim", head_dim), dtype
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float16
        self.page_bytes = 68 * self.head_dim
        if pages is None:
            if num_pages is None:
                raise ValueError("num_pages or pages is required")
            pages = torch.zeros((int(num_pages), self.n_kv_heads, self.page_bytes), dtype=torch.uint8, device=device or "cuda")
        elif not isinstance(pages, torch.Tensor) or pages.dtype != torch.uint8 or not pages.is_contiguous() or \
                pages.dim() != 3 or tuple(pages.shape[1:]) != (self.n_kv_heads, self.page_bytes):
            raise ValueError(f"pages must be a contiguous uint8 tensor [num_pages, {self.n_kv_heads}, {self.page_bytes}]")
        self._pages = pages
        self._device = pages.device.index if pages.is_cuda else -1
        self._c = _lib.Cache(_lib.ATTENTION_DTYPES[dtype], self.n_kv_heads, self.head_dim, pages.shape[0], pages.data_ptr())
        self._at = ctypes.addressof(self._c)

    @property
    def pages(self):
        """The cache's memory.  (Not to be replaced: calls go to the address of the tensor that it was made with.)"""
        return self._pages

    def _native(self, stream):
        """As the module's _native, and the address of the cache's description."""
        native = _native(stream)
        return None if native is None or native[2] != self._device else native

    def _on(self) -> int:
        device = _device()
        if not _on_device(self.pages, device):
            raise ValueError(f"the cache's pages must be on cuda:{device} (the current device), got {self.pages.device}")
        return device

    def _table(self, name: str, table, B, device: int):
        p = _array(name, table, _torch().int32, (B, None), device)
        return p, int(table.shape[1])

    # ------------------------------------------------------------ tokens in and out
    def write(self, k, v, page_table, start, count=None, index=None, stream=None) -> None:
        """Puts the first ``count[b]`` tokens (default: all) of k, v [B, rows, kv heads, D] into the slots from
        start[b] on.  With ``index`` (int32 [B, T]) token j is row index[b, j]: the accepted path of a tree."""
        native = self._native(stream)
        if native is not None:
            binding, ops, device, raw = native
            if _done(binding.cache_write(ops, device, raw, self._at, k, v, page_table, start, count, index)):
                return
        torch = _torch()
        device = self._on()
        B = page_table.shape[0] if isinstance(page_table, torch.Tensor) and page_table.dim() == 2 else None
        table, pages = self._table("page_table", page_table, B, device)
        shape = (B, k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 4 else None, self.n_kv_heads, self.head_dim)
        kv, vv = _view("k", k, self.torch_dtype, shape, device), _view("v", v, self.torch_dtype, shape, device)
        st = _array("start", start, torch.int64, (B,), device)
        n = None if count is None else _array("count", count, torch.int32, (B,), device)
        T, at = int(k.shape[1]), None
        if index is not None:
            at = _array("index", index, torch.int32, (B, None), device)
            T = int(index.shape[1])
        _lib.check(_lib.lib().caddtree_cache_write(ctypes.byref(self._c), ctypes.byref(kv), ctypes.byref(vv), B, T,
                                                   int(k.shape[1]), st, n, at, table, pages, _stream(stream, device)))

    def read(self, page_table, end, k, v, start=None, stream=None) -> None:
        """Writes the values of the slots start[b] (default 0) .. end[b] - 1 into k, v [B, T, kv heads, D], at most
        T of them; further rows are left as they are."""
        native = self._native(stream)
        if native is not None:
            binding, ops, device, raw = native
            if _done(binding.cache_read(ops, device, raw, self._at, k, v, page_table, start, end)):
                return
        torch = _torch()
        device = self._on()
        B = page_table.shape[0] if isinstance(page_table, torch.Tensor) and page_table.dim() == 2 else None
        table, pages = self._table("page_table", page_table, B, device)
        shape = (B, k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 4 else None, self.n_kv_heads, self.head_dim)
        kv, vv = _output("k", k, self.torch_dtype, shape, device), _output("v", v, self.torch_dtype, shape, device)
        e = _array("end", end, torch.int64, (B,), device)
        st = None if start is None else _array("start", start, torch.int64, (B,), device)
        _lib.check(_lib.lib().caddtree_cache_read(ctypes.byref(self._c), ctypes.byref(kv), ctypes.byref(vv), B, int(k.shape[1]),
                                                  st, e, table, pages, _stream(stream, device)))

    # ------------------------------------------------------------ attention
    def _attention(self, q, page_table, ctx_len, count, depth, window, sinks, scale, device):
        torch = _torch()
        a, name = _queries(q, device)
        if name != self.dtype:
            raise TypeError(f"q must be {self.torch_dtype}, the cache's type, got {q.dtype}")
        if a.head_dim != self.head_dim:
            raise ValueError(f"q must have head dimension {self.head_dim}, the cache's, got {a.head_dim}")
        a.n_kv_heads, a.S = self.n_kv_heads, a.T
        a.page_table, a.table_pages = self._table("page_table", page_table, a.B, device)
        a.ctx_len = _array("ctx_len", ctx_len, torch.int64, (a.B,), device)
        if count is not None:
            a.q_len = _array("count", count, torch.int32, (a.B,), device)
        if depth is not None:
            a.depth = _array("depth", depth, torch.int32, (a.B, None), device)
            a.cap = depth.shape[1]
            a.order = _lib.ORDERS["tree"]
        a.scale, a.window, a.sinks = _scale(scale, a.head_dim), _int32("window", window), _int32("sinks", sinks)
        return a

    def attention(self, q, page_table, ctx_len, k=None, v=None, *, count=None, causal: bool = True, mask=None, depth=None,
                  window: int = 0, sinks: int = 0, scale: Optional[float] = None, out=None, lse=None, workspace=None,
                  stream=None):
        """Attention of q [B, T, heads, D] over the ctx_len cached slots and the new k, v [B, T, kv heads, D]
        (which are not written to the cache).  The new tokens are a chain (``causal=True``), a block that all
        its queries see (``causal=False``), or with ``mask`` and ``depth`` a draft tree as a plan built it: row 0
        its root, row i node i - 1.  ``count`` int32 [B]: the tokens of each sequence, in a tree its n_star.
        Writes ``out`` (made of zeros if not given) and ``lse`` (float32 [B, T, heads], if given); rows without a
        query are left as they are.  Returns out."""
        out = _made(q, out, stream)
        native = self._native(stream)
        if native is not None:
            binding, ops, device, raw = native
            if _done(binding.cache_attention(ops, device, raw, self._at, q, page_table, ctx_len, k, v, count, causal, mask, depth,
                                             window, sinks, scale, out, lse, workspace)):
                return out
        _no_gradient(q=q, k=k, v=v)
        torch = _torch()
        device = self._on()
        if (mask is None) != (depth is None) and k is not None:
            raise ValueError("a tree needs both mask and depth")
        if (k is None) != (v is None):
            raise ValueError("k and v are given together")
        a = self._attention(q, page_table, ctx_len, count, depth, window, sinks, scale, device)
        if depth is None:
            a.order = _lib.ORDERS["chain" if causal else "block"]
        if mask is not None:
            if depth is None:
                raise ValueError("a tree needs both mask and depth")
            if isinstance(mask, torch.Tensor) and mask.dtype == torch.uint8:
                a.mask_kind = _lib.MASKS["u8"]
                a.mask = _array("mask", mask, torch.uint8, (a.B, a.cap, a.cap), device)
            else:
                if not isinstance(mask, torch.Tensor) or mask.dtype not in (torch.int32, getattr(torch, "uint32", torch.int32)):
                    raise TypeError("mask must be a uint8 tensor, or int32 or uint32 words")
                a.mask_kind = _lib.MASKS["bits"]
                a.mask = _array("mask", mask, mask.dtype, (a.B, a.cap, (a.cap + 31) // 32), device)
        if k is not None:
            shape = (a.B, a.T, self.n_kv_heads, self.head_dim)
            a.k, a.v = _view("k", k, q.dtype, shape, device), _view("v", v, q.dtype, shape, device)
        _results(q, out, lse, a, device)
        ws, n = _workspace(workspace, device)
        _lib.check(_lib.lib().caddtree_cache_attention(ctypes.byref(self._c), ctypes.byref(a), ws, n, _stream(stream, device)))
        return out

    # ------------------------------------------------------------ eviction
    def score(self, q, page_table, ctx_len, lse, scores, new_scores=None, *, weight=None, count=None, depth=None,
              window: int = 0, sinks: int = 0, scale: Optional[float] = None, stream=None) -> None:
        """Adds the attention weight of the cached slots to ``scores`` (float32 [B, kv heads, slots]), in place or
        into ``new_scores``: the arguments of the ``attention`` call that wrote ``lse`` (read here in any strides),
        and ``weight`` (float32 [B, T], default 1) to pick and weigh its queries (in a tree: the accepted ones).
        ``depth`` says that the queries are a tree's."""
        native = self._native(stream)
        if native is not None:
            binding, ops, device, raw = native
            if _done(binding.cache_score(ops, device, raw, self._at, q, page_table, ctx_len, lse, scores, new_scores, weight, count,
                                         depth, window, sinks, scale)):
                return
        torch = _torch()
        device = self._on()
        a = self._attention(q, page_table, ctx_len, count, depth, window, sinks, scale, device)
        shape = (a.B, a.T, a.n_heads)
        if isinstance(lse, torch.Tensor) and lse.dim() == 3 and not lse.is_contiguous():
            a.lse, a.lse_strided = _array("lse", lse, torch.float32, shape, device, contiguous=False), 1
            a.lse_stride_b, a.lse_stride_t, a.lse_stride_h = lse.stride()
        else:
            a.lse = _array("lse", lse, torch.float32, shape, device)
        w = None if weight is None else _array("weight", weight, torch.float32, (a.B, a.T), device)
        old = _array("scores", scores, torch.float32, (a.B, self.n_kv_heads, None), device)
        new = old if new_scores is None else _array("new_scores", new_scores, torch.float32, tuple(scores.shape), device)
        _lib.check(_lib.lib().caddtree_cache_score(ctypes.byref(self._c), ctypes.byref(a), w, old, new, int(scores.shape[2]),
                                                   _stream(stream, device)))

    def evict(self, page_table, ctx_len, scores, new_table, new_len, new_scores, kept, *, budget: int, sinks: int = 0,
              recent: int = 0, workspace=None, stream=None) -> None:
        """Cuts every sequence to at most ``budget`` slots a kv head: the first ``sinks``, the last ``recent`` and
        the largest scores of the rest, in their old order; slots of pages outside the cache hold no key and are
        left out.  The kept slots go to the pages of ``new_table`` (int32 [B, pages], none of them in use), their
        scores to ``new_scores`` (float32 [B, kv heads, slots], zeros behind), how many they are to ``new_len``
        (int64 [B]) and the old slots to ``kept`` (int32 [B, kv heads, budget], -1 behind).  These four are tensors
        apart from the ones that are read.  Rows of more than 16384 slots need a workspace, made here if not given
        (with a raw stream handle it has to be).  Positions are slot numbers, so a window over an evicted cache
        counts kept slots."""
        if workspace is None and (stream is None or hasattr(stream, "cuda_stream")):
            workspace = self.evict_workspace(page_table, scores, stream)
        native = self._native(stream)
        if native is not None:
            binding, ops, device, raw = native
            if _done(binding.cache_evict(ops, device, raw, self._at, page_table, ctx_len, scores, new_table, new_len, new_scores, kept,
                                         budget, sinks, recent, workspace)):
                return
        torch = _torch()
        device = self._on()
        B = page_table.shape[0] if isinstance(page_table, torch.Tensor) and page_table.dim() == 2 else None
        table, pages = self._table("page_table", page_table, B, device)
        new, new_pages = self._table("new_table", new_table, B, device)
        f32 = torch.float32
        args = (_array("ctx_len", ctx_len, torch.int64, (B,), device),
                _array("scores", scores, f32, (B, self.n_kv_heads, None), device), int(scores.shape[2]),
                _int32("budget", budget), _int32("sinks", sinks), _int32("recent", recent), new, new_pages,
                _array("new_scores", new_scores, f32, (B, self.n_kv_heads, None), device), int(new_scores.shape[2]),
                _array("new_len", new_len, torch.int64, (B,), device),
                _array("kept", kept, torch.int32, (B, self.n_kv_heads, int(budget)), device))
        _lib.check(_lib.lib().caddtree_cache_evict(ctypes.byref(self._c), B, table, pages, *args,
                                                   *_workspace(workspace, device), _stream(stream, device)))

    def evict_workspace(self, page_table, scores, stream=None):
        """A workspace for ``evict`` of these page_table and scores (uint8; the contents do not matter), allocated on
        the stream; None where it needs none."""
        torch = _torch()
        if not isinstance(page_table, torch.Tensor) or not isinstance(scores, torch.Tensor) \
                or page_table.dim() != 2 or scores.dim() != 3 or scores.shape[2] <= 16384:
            return None
        n = _lib.lib().caddtree_evict_workspace_bytes(ctypes.byref(self._c), page_table.shape[0], page_table.shape[1], scores.shape[2])
        if n == 0:
            return None
        if stream is None:
            return torch.empty(n, dtype=torch.uint8, device=self.pages.device)
        with torch.cuda.stream(stream):
            return torch.empty(n, dtype=torch.uint8, device=self.pages.device)
