"""What the attention and cache calls refuse (CPU, no GPU needed): the Python checks, the native calls against
them, and the library's own checks of a C caller's arguments.

Over forms of every argument a native call either passes the library exactly what the Python path passes it, or
returns None and leaves the call to the Python path; what the Python path refuses it never passes on.  Host
tensors stand in for device ones, and recording functions for the library's.
"""

import ctypes

import numpy as np
import pytest
import torch

from paper_2606_01813_amd import KVCache, _lib, attention, attention_workspace, window_attention

STREAM = 0x1234
B, T, Hq, Hkv, D, CAP, PAGES = 2, 5, 4, 2, 64, 7, 3
BF = torch.bfloat16
NAMES = ("window_attention", "cache_attention", "cache_write", "cache_read", "cache_score", "cache_evict")


def _flat(a):
    """A call's argument as plain values, structures field by field."""
    if hasattr(a, "contents"):
        a = a.contents if a else None
    if isinstance(a, ctypes.Structure):
        return tuple(_flat(getattr(a, f)) for f, _ in a._fields_)
    return a


class _Recorder:
    def __init__(self):
        self.calls = []
        real = _lib.lib()
        for name in NAMES:
            types = getattr(real, "caddtree_" + name).argtypes
            f = ctypes.CFUNCTYPE(ctypes.c_int, *types)(self._make(name))
            f.argtypes = types
            setattr(self, "caddtree_" + name, f)

    def _make(self, name):
        def record(*args):
            self.calls.append((name, tuple(_flat(a) for a in args)))
            return 0
        return record

    def ops(self):
        return _lib.binding().ops(1, *(ctypes.cast(getattr(self, "caddtree_" + n), ctypes.c_void_p).value for n in NAMES))


@pytest.fixture
def rec(monkeypatch):
    r = _Recorder()
    monkeypatch.setattr(attention, "_on_device", lambda t, device: t.device.type == "cpu")
    monkeypatch.setattr(attention, "_device", lambda: 0)
    monkeypatch.setattr(attention, "_stream", lambda stream, device: STREAM)
    monkeypatch.setattr(attention, "_native", lambda stream: None)
    monkeypatch.setattr(_lib, "lib", lambda: r)
    return r


def _aligned(shape, dtype):
    n = int(np.prod(shape))
    raw = torch.zeros(n * dtype.itemsize + 256, dtype=torch.uint8)
    off = -raw.data_ptr() % 256
    return raw[off:off + n * dtype.itemsize].view(dtype).view(shape)


def _state():
    i32, i64, f32 = torch.int32, torch.int64, torch.float32
    z = lambda shape, dtype: _aligned(shape, dtype)
    return {"q": z((B, T, Hq, D), BF), "k": z((B, T, Hkv, D), BF), "v": z((B, T, Hkv, D), BF), "out": z((B, T, Hq, D), BF),
            "lse": z((B, T, Hq), f32), "workspace": z((4096,), torch.uint8), "q_len": z((B,), i32), "k_len": z((B,), i32),
            "table": z((B, PAGES), i32), "ctx_len": z((B,), i64), "count": z((B,), i32), "mask": z((B, CAP, CAP), torch.uint8),
            "depth": z((B, CAP), i32), "start": z((B,), i64), "index": z((B, 3), i32), "end": z((B,), i64),
            "scores": z((B, Hkv, 100), f32), "new_scores": z((B, Hkv, 100), f32), "weight": z((B, T), f32),
            "new_table": z((B, 2), i32), "new_len": z((B,), i64), "cut": z((B, Hkv, 90), f32), "kept": z((B, Hkv, 80), i32),
            "window": 3, "sinks": 1, "scale": 0.5, "causal": True, "budget": 80, "recent": 4, "ko": z((B, T, Hkv, D), BF),
            "vo": z((B, T, Hkv, D), BF)}


CALLS = {
    "window": (lambda c, s: window_attention(s["q"], s["k"], s["v"], window=s["window"], sinks=s["sinks"], causal=s["causal"],
                                             scale=s["scale"], q_len=s["q_len"], k_len=s["k_len"], out=s["out"], lse=s["lse"],
                                             workspace=s["workspace"]),
               ("q", "k", "v", "q_len", "k_len", "out", "lse", "workspace", "window", "sinks", "scale", "causal")),
    "tree": (lambda c, s: c.attention(s["q"], s["table"], s["ctx_len"], s["k"], s["v"], count=s["count"], mask=s["mask"], depth=s["depth"],
                                      window=s["window"], sinks=s["sinks"], scale=s["scale"], out=s["out"], lse=s["lse"],
                                      workspace=s["workspace"]),
             ("q", "table", "ctx_len", "k", "v", "count", "mask", "depth", "out", "lse", "workspace", "window", "sinks", "scale")),
    "chain": (lambda c, s: c.attention(s["q"], s["table"], s["ctx_len"], s["k"], s["v"], causal=s["causal"], out=s["out"]),
              ("q", "table", "ctx_len", "k", "v", "causal", "out")),
    "write": (lambda c, s: c.write(s["k"], s["v"], s["table"], s["start"], count=s["count"], index=s["index"]),
              ("k", "v", "table", "start", "count", "index")),
    "read": (lambda c, s: c.read(s["table"], s["end"], s["ko"], s["vo"], start=s["start"]), ("table", "end", "ko", "vo", "start")),
    "score": (lambda c, s: c.score(s["q"], s["table"], s["ctx_len"], s["lse"], s["scores"], s["new_scores"], weight=s["weight"],
                                   count=s["count"], depth=s["depth"], window=s["window"], sinks=s["sinks"], scale=s["scale"]),
              ("q", "table", "ctx_len", "lse", "scores", "new_scores", "weight", "count", "depth", "window", "sinks", "scale")),
    "evict": (lambda c, s: c.evict(s["table"], s["ctx_len"], s["scores"], s["new_table"], s["new_len"], s["cut"], s["kept"],
                                   budget=s["budget"], sinks=s["sinks"], recent=s["recent"]),
              ("table", "ctx_len", "scores", "new_table", "new_len", "cut", "kept", "budget", "sinks", "recent")),
}


def _forms(x):
    """Other forms of an argument."""
    yield None
    yield "text"
    if not isinstance(x, torch.Tensor):
        yield from (0, 1, -1, 7, 2 ** 31 - 1, 2 ** 31, 1.5, 0.0, float("inf"), True, False, np.int64(3))
        return
    yield np.zeros(3)
    yield torch.nn.Parameter(x.clone(), requires_grad=False) if x.is_floating_point() else x.clone()
    for dt in (torch.int32, torch.int64, torch.float32, BF, torch.float16, torch.uint8, torch.uint32):
        yield _aligned(x.shape, dt)
    for d in range(x.dim()):
        for n in (0, 1, x.shape[d] - 1, x.shape[d] + 1):
            yield _aligned(x.shape[:d] + (n,) + x.shape[d + 1:], x.dtype)
        yield _aligned(x.shape[:d] + (2 * x.shape[d],) + x.shape[d + 1:], x.dtype)[(slice(None),) * d + (slice(None, None, 2),)]
        yield _aligned(x.shape[:d] + (1,) + x.shape[d + 1:], x.dtype).expand(x.shape)
    yield _aligned(tuple(x.shape) + (1,), x.dtype)
    yield _aligned((x.numel() + 1,), x.dtype)[1:].view(x.shape)             # not aligned
    if x.dim() == 4:
        yield _aligned((x.shape[0], x.shape[2], x.shape[1], x.shape[3]), x.dtype).transpose(1, 2)
        yield _aligned(x.shape[:3] + (x.shape[3] + 4,), x.dtype)[..., :x.shape[3]]      # strides of 68
        yield _aligned(x.shape[:3] + (x.shape[3] + 8,), x.dtype)[..., :x.shape[3]]
        yield _aligned(x.shape[:2] + (x.shape[3], x.shape[2]), x.dtype).transpose(2, 3)


def _cache():
    c = KVCache(Hkv, D, pages=_aligned((9, Hkv, 68 * D), torch.uint8))
    c._device = 0
    return c


@pytest.mark.parametrize("name", CALLS)
def test_native_calls_pass_on_what_the_python_path_does_or_leave_it_to_it(name, rec, monkeypatch):
    call, args = CALLS[name]
    cache, ops, passed = _cache(), rec.ops(), 0

    def run(state, native):
        monkeypatch.setattr(attention, "_native", lambda stream: (_lib.binding(), ops, 0, STREAM) if native else None)
        rec.calls.clear()
        try:
            call(cache, state)
        except Exception as e:
            return type(e), list(rec.calls)
        return None, list(rec.calls)

    base = _state()
    assert run(base, False) == run(base, True) and rec.calls
    # the native call itself took the plain form (the Python path is not there to fall back on)
    monkeypatch.setattr(attention, "_tensor", lambda *a: pytest.fail("the Python checks were needed"))
    assert run(base, True)[0] is None
    monkeypatch.undo()
    monkeypatch.setattr(attention, "_on_device", lambda t, device: t.device.type == "cpu")
    monkeypatch.setattr(attention, "_device", lambda: 0)
    monkeypatch.setattr(attention, "_stream", lambda stream, device: STREAM)
    monkeypatch.setattr(_lib, "lib", lambda: rec)
    for arg in args:
        for form in _forms(base[arg]):
            state = dict(base, **{arg: form})
            if arg == "out" and form is None:
                continue                                          # made by the call: another place each time
            plain, native = run(state, False), run(state, True)
            assert plain == native, (arg, form if not isinstance(form, torch.Tensor) else (form.dtype, form.shape, form.stride()))
            passed += plain[0] is None
    assert passed > len(args)


REFUSED = [
    ("window", "q", lambda s: s["q"].float(), TypeError),
    ("window", "q", lambda s: s["q"][0], ValueError),
    ("window", "k", lambda s: s["k"].half(), TypeError),
    ("window", "k", lambda s: s["k"][:1], ValueError),
    ("window", "v", lambda s: s["v"][:, 1:], ValueError),
    ("window", "q_len", lambda s: s["q_len"].long(), TypeError),
    ("window", "q_len", lambda s: torch.zeros(B + 1, dtype=torch.int32), ValueError),
    ("window", "lse", lambda s: s["lse"].transpose(0, 1), ValueError),
    ("window", "out", lambda s: s["out"][:, :1].expand(B, T, Hq, D), ValueError),
    ("window", "workspace", lambda s: 3, ValueError),
    ("window", "q", lambda s: _aligned((B, T, Hq, D + 4), BF)[..., :D], ValueError),
    ("window", "q", lambda s: _aligned((B * T * Hq * D + 1,), BF)[1:].view(B, T, Hq, D), ValueError),
    ("tree", "mask", lambda s: None, ValueError),
    ("tree", "depth", lambda s: None, ValueError),
    ("tree", "v", lambda s: None, ValueError),
    ("tree", "mask", lambda s: s["mask"].float(), TypeError),
    ("tree", "mask", lambda s: s["mask"][:, 1:], ValueError),
    ("tree", "mask", lambda s: torch.zeros((B, CAP, 2), dtype=torch.int32), ValueError),
    ("tree", "q", lambda s: s["q"].half(), TypeError),
    ("tree", "q", lambda s: _aligned((B, T, Hq, 128), BF), ValueError),
    ("tree", "ctx_len", lambda s: s["count"], TypeError),
    ("tree", "table", lambda s: s["table"].long(), TypeError),
    ("tree", "table", lambda s: s["table"][:1], ValueError),
    ("write", "index", lambda s: s["index"][:1], ValueError),
    ("write", "k", lambda s: s["k"][:, :, :1], ValueError),
    ("write", "start", lambda s: None, TypeError),
    ("read", "ko", lambda s: s["ko"][:, :1].expand(B, T, Hkv, D), ValueError),
    ("read", "end", lambda s: s["count"], TypeError),
    ("score", "weight", lambda s: s["weight"].double(), TypeError),
    ("score", "lse", lambda s: s["lse"][:, :3], ValueError),
    ("score", "new_scores", lambda s: s["new_scores"][..., :50], ValueError),
    ("evict", "kept", lambda s: s["kept"][..., :5], ValueError),
    ("evict", "new_len", lambda s: s["count"], TypeError),
]


@pytest.mark.parametrize("case", REFUSED, ids=[f"{c[0]}-{c[1]}-{i}" for i, c in enumerate(REFUSED)])
def test_refused_before_the_library_is_called(case, rec):
    name, arg, form, error = case
    s = _state()
    s[arg] = form(s)
    with pytest.raises(error, match=arg if arg in ("q", "k", "v", "lse", "out") else None):
        CALLS[name][0](_cache(), s)
    assert not rec.calls


def test_host_tensors_and_other_devices_are_refused(monkeypatch):
    monkeypatch.setattr(attention, "_device", lambda: 0)
    monkeypatch.setattr(attention, "_native", lambda stream: None)
    s = _state()
    with pytest.raises(ValueError, match="cuda:0"):
        CALLS["window"][0](None, s)
    c = _cache()
    for name in ("chain", "write", "read", "score", "evict"):
        with pytest.raises(ValueError, match="cuda:0"):
            CALLS[name][0](c, s)


def test_cache_and_workspace_arguments():
    with pytest.raises(ValueError, match="dtype"):
        KVCache(2, 64, 4, dtype="f32")
    with pytest.raises(ValueError, match="num_pages"):
        KVCache(2, 64)
    with pytest.raises(ValueError, match="pages"):
        KVCache(2, 64, pages=torch.zeros((4, 2, 68 * 128), dtype=torch.uint8))
    with pytest.raises(TypeError):
        attention_workspace(torch.zeros((1, 1, 1, 64)), torch.zeros((1, 1, 1, 64)))
    ws = attention_workspace(_aligned((1, 16, 32, 128), BF), _aligned((1, 4096, 8, 128), BF))
    assert ws.dtype == torch.uint8 and ws.numel() >= 1


# ---------------------------------------------------------------- a C caller's arguments

def _attention(**kw):
    q = 0x1000
    a = _lib.Attention()
    d = dict(dtype=1, B=2, T=5, S=5, n_heads=4, n_kv_heads=2, head_dim=64, q=(q, 640, 128, 64), k=(q, 640, 128, 64), v=(q, 640, 128, 64),
             out=(q, 640, 128, 64), scale=1.0, window=0, sinks=0, order=0, mask_kind=0, mask=0x1000, depth=0x1000, cap=7, page_table=0x1000,
             table_pages=3, ctx_len=0x1000, lse=0x1000)
    d.update(kw)
    for f, v in d.items():
        setattr(a, f, _lib.View(*v) if isinstance(v, tuple) else v)
    return a


def _c_cache(**kw):
    d = dict(dtype=1, n_kv_heads=2, head_dim=64, n_pages=9, pages=0x1000)
    d.update(kw)
    return _lib.Cache(*(d[f] for f, _ in _lib.Cache._fields_))


INVALID, UNSUPPORTED, WORKSPACE = _lib.E_INVALID, _lib.E_UNSUPPORTED, _lib.E_WORKSPACE
BAD_ATTENTION = [
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=9), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), INVALID),
    (dict(B=-1), INVALID), (dict(B=65536), UNSUPPORTED), (dict(T=-1), INVALID), (dict(S=-1), INVALID), (dict(n_heads=3), INVALID),
    (dict(n_heads=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_heads=65538), UNSUPPORTED), (dict(T=2 ** 31 - 1), UNSUPPORTED),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(order=3), INVALID), (dict(q=(0, 0, 0, 0)), INVALID), (dict(q=(0x1008, 640, 128, 64)), INVALID),
    (dict(q=(0x1000, 641, 128, 64)), INVALID), (dict(out=(0, 0, 0, 0)), INVALID), (dict(out=(0x1000, 640, 128, 4)), INVALID),
    (dict(q=(0x1000, 640, -128, 64)), INVALID), (dict(q=(0x1000, 640, 2 ** 24, 64)), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_ATTENTION + [
    (dict(k=(0, 0, 0, 0)), INVALID), (dict(v=(0, 0, 0, 0)), INVALID), (dict(k=(0x1000, 640, 4, 64)), INVALID), (dict(order=2), INVALID)])
def test_window_attention_validation(kw, status):
    a = _attention(**kw)
    assert _lib.lib().caddtree_window_attention(ctypes.byref(a), None, 0, None) == status, _lib.lib().caddtree_last_error()
    assert _lib.lib().caddtree_last_error()


@pytest.mark.parametrize("kw,status", BAD_ATTENTION + [
    (dict(v=(0, 0, 0, 0)), INVALID), (dict(k=(0, 0, 0, 0)), INVALID), (dict(order=2, mask_kind=7), INVALID),
    (dict(order=2, mask_kind=0), INVALID), (dict(order=2, mask_kind=1, mask=None), INVALID), (dict(order=2, mask_kind=1, depth=None), INVALID),
    (dict(order=2, mask_kind=1, cap=3), INVALID), (dict(order=2, mask_kind=1, cap=4097), INVALID), (dict(page_table=None), INVALID),
    (dict(table_pages=-1), INVALID), (dict(table_pages=2 ** 25), INVALID), (dict(ctx_len=None), INVALID), (dict(n_kv_heads=4), INVALID),
    (dict(dtype=2), INVALID), (dict(head_dim=128), INVALID)])
def test_cache_attention_validation(kw, status):
    a, c = _attention(**kw), _c_cache()
    lib = _lib.lib()
    assert lib.caddtree_cache_attention(ctypes.byref(c), ctypes.byref(a), None, 0, None) == status, lib.caddtree_last_error()


@pytest.mark.parametrize("kw,status", [(dict(dtype=0), UNSUPPORTED), (dict(dtype=5), INVALID), (dict(head_dim=80), UNSUPPORTED),
                                       (dict(n_kv_heads=0), INVALID), (dict(n_pages=-1), INVALID), (dict(n_pages=2 ** 31), INVALID),
                                       (dict(pages=None), INVALID), (dict(pages=0x1010), INVALID)])
def test_cache_validation(kw, status):
    lib, c, a, v = _lib.lib(), _c_cache(**kw), _attention(), _lib.View(0x1000, 640, 128, 64)
    r = ctypes.byref
    assert lib.caddtree_cache_write(r(c), r(v), r(v), 2, 5, 5, 0x1000, None, None, 0x1000, 3, None) == status
    assert lib.caddtree_cache_read(r(c), r(v), r(v), 2, 5, None, 0x1000, 0x1000, 3, None) == status
    assert lib.caddtree_cache_evict(r(c), 2, 0x1000, 3, 0x1000, 0x1000, 100, 64, 1, 1, 0x1000, 1, 0x1000, 64, 0x1000, 0x1000, None, 0, None) == status
    assert lib.caddtree_cache_score(r(c), r(a), None, 0x1000, 0x1000, 100, None) == status
    assert lib.caddtree_cache_attention(r(c), r(a), None, 0, None) == status


def test_other_refusals_and_calls_of_nothing():
    lib, c, a, v, r = _lib.lib(), _c_cache(), _attention(), _lib.View(0x1000, 640, 128, 64), ctypes.byref
    none = _lib.View(None, 0, 0, 0)
    assert lib.caddtree_window_attention(None, None, 0, None) == INVALID
    assert lib.caddtree_window_attention(r(a), 0x1010, 100, None) == WORKSPACE
    assert lib.caddtree_cache_attention(None, r(a), None, 0, None) == INVALID
    assert lib.caddtree_cache_attention(r(c), r(a), 0x1010, 100, None) == WORKSPACE
    assert lib.caddtree_attention_workspace_bytes(None) == 0
    write = lambda *x: lib.caddtree_cache_write(*x, None)
    assert write(None, r(v), r(v), 2, 5, 5, 0x1000, None, None, 0x1000, 3) == INVALID
    assert write(r(c), None, r(v), 2, 5, 5, 0x1000, None, None, 0x1000, 3) == INVALID
    assert write(r(c), r(none), r(v), 2, 5, 5, 0x1000, None, None, 0x1000, 3) == INVALID
    assert write(r(c), r(v), r(v), 2, 5, 4, 0x1000, None, None, 0x1000, 3) == INVALID      # fewer rows than tokens
    assert write(r(c), r(v), r(v), 2, -1, 5, 0x1000, None, None, 0x1000, 3) == INVALID
    assert write(r(c), r(v), r(v), 2, 2 ** 30, 2 ** 30, 0x1000, None, None, 0x1000, 3) == UNSUPPORTED
    assert write(r(c), r(v), r(v), 2, 5, 5, None, None, None, 0x1000, 3) == INVALID
    assert write(r(c), r(v), r(v), 2, 5, 5, 0x1000, None, None, None, 3) == INVALID
    read = lambda *x: lib.caddtree_cache_read(*x, None)
    assert read(r(c), r(v), r(v), 2, 5, None, None, 0x1000, 3) == INVALID
    assert read(r(c), r(v), r(none), 2, 5, None, 0x1000, 0x1000, 3) == INVALID
    score = lambda *x: lib.caddtree_cache_score(*x, None)
    assert score(r(c), r(a), None, None, 0x1000, 100) == INVALID
    assert score(r(c), r(a), None, 0x1000, 0x1000, -1) == INVALID
    assert score(r(c), r(_attention(lse=None)), None, 0x1000, 0x1000, 100) == INVALID
    evict = lambda **kw: lib.caddtree_cache_evict(r(c), *{**dict(
        B=2, table=0x1000, pages=3, ctx=0x1000, scores=0x1000, slots=100, budget=64, sinks=4, recent=9, new_table=0x1000, new_pages=1,
        new_scores=0x1000, new_slots=64, new_len=0x1000, kept=0x1000, workspace=None, bytes=0), **kw}.values(), None)
    for kw in (dict(B=-1), dict(table=None), dict(budget=-1), dict(sinks=-1), dict(recent=-1), dict(sinks=60), dict(slots=-1),
               dict(new_slots=63), dict(new_pages=0), dict(new_table=None), dict(ctx=None), dict(new_len=None), dict(scores=None),
               dict(new_scores=None), dict(kept=None)):
        assert evict(**kw) == INVALID, kw
    long = dict(pages=257, slots=20000)
    need = lib.caddtree_evict_workspace_bytes(r(c), 2, 257, 20000)
    assert need > 0 and lib.caddtree_evict_workspace_bytes(r(c), 2, 256, 20000) == 0
    assert lib.caddtree_evict_workspace_bytes(None, 2, 257, 20000) == 0
    for kw in (long, dict(**long, workspace=0x1000, bytes=need - 1), dict(workspace=0x1010, bytes=need)):
        assert evict(**kw) == WORKSPACE, kw
    # nothing to do: no HIP call is made, pointers may be NULL
    e = _attention(B=0, q=(0, 0, 0, 0), k=(0, 0, 0, 0), v=(0, 0, 0, 0), out=(0, 0, 0, 0), ctx_len=None)
    assert lib.caddtree_window_attention(r(e), None, 0, None) == _lib.OK
    assert lib.caddtree_cache_attention(r(c), r(e), None, 0, None) == _lib.OK
    assert write(r(c), r(none), r(none), 0, 0, 0, None, None, None, None, 0) == _lib.OK
    assert read(r(c), r(none), r(none), 0, 0, None, None, None, 0) == _lib.OK
    assert score(r(c), r(e), None, None, None, 0) == _lib.OK
    assert evict(B=0, ctx=None, new_len=None, scores=None, new_scores=None, kept=None) == _lib.OK


def test_workspace_sizes():
    """No more than a call's splits use, and none where rows alone fill the card."""
    size = lambda **kw: _lib.lib().caddtree_attention_workspace_bytes(ctypes.byref(_attention(**kw)))
    assert size(B=0) == size(T=0) == 0
    assert size(B=64, T=2048, S=4096, n_heads=32, n_kv_heads=8, table_pages=0) == 0
    one = size(B=1, T=1, S=1, n_heads=8, n_kv_heads=8, table_pages=2048)
    assert 0 < one <= 8 * 128 * (64 * 4 + 8) + 256


def test_workspace_of_sizes_that_are_refused():
    """A query of sizes that no call takes returns 0, as the call returns its error."""
    lib = _lib.lib()
    good = dict(B=1, T=1, S=4096, n_heads=8, n_kv_heads=4, table_pages=0)
    size = lambda **kw: lib.caddtree_attention_workspace_bytes(ctypes.byref(_attention(**dict(good, **kw))))
    assert size() > 0 and size(window=2 ** 31 - 1, sinks=2 ** 31 - 1) > 0 and size(window=1000) > 0
    for kw in (dict(n_heads=2), dict(n_heads=2, window=10), dict(n_heads=0), dict(n_heads=10), dict(n_kv_heads=0), dict(n_kv_heads=-4),
               dict(n_heads=-8), dict(head_dim=96), dict(head_dim=-64), dict(dtype=0), dict(dtype=7), dict(B=-1), dict(B=65536),
               dict(T=-1), dict(T=2 ** 31 - 1), dict(S=-1), dict(S=2 ** 31 - 1), dict(window=-1), dict(sinks=-1), dict(n_heads=2 ** 17),
               dict(table_pages=-1), dict(table_pages=2 ** 25), dict(B=65535, T=2 ** 29)):
        assert size(**kw) == 0, kw
        if "table_pages" not in kw:
            a = _attention(**dict(good, **kw))
            assert lib.caddtree_window_attention(ctypes.byref(a), None, 0, None) in (INVALID, UNSUPPORTED), kw


INTEGERS = [("window", "window"), ("window", "sinks"), ("tree", "window"), ("tree", "sinks"), ("score", "window"), ("score", "sinks"),
            ("evict", "budget"), ("evict", "sinks"), ("evict", "recent")]


@pytest.mark.parametrize("native", [False, True], ids=["python", "native"])
@pytest.mark.parametrize("name,arg", INTEGERS, ids=["-".join(x) for x in INTEGERS])
def test_integers_keep_all_their_bits(name, arg, native, rec, monkeypatch):
    """What does not fit 32 bits is refused; ctypes would pass on its lower half."""
    ops = rec.ops()
    if native:
        monkeypatch.setattr(attention, "_native", lambda stream: (_lib.binding(), ops, 0, STREAM))
    for n in (2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 64 + 80, -2 ** 32 + 3, 2.5, np.int64(2 ** 33 + 1)):
        s = _state()
        s[arg] = n
        with pytest.raises(ValueError, match=arg):
            CALLS[name][0](_cache(), s)
        assert not rec.calls, n
    s = _state()
    s[arg] = np.int64(s[arg])
    CALLS[name][0](_cache(), s)
    assert rec.calls


def test_sizes_keep_all_their_bits(rec):
    """Inputs may repeat (stride 0), so a tensor's sizes can pass 32 bits in little memory."""
    s = _state()
    far = lambda *dims: _aligned((1,) * (len(dims) - 1) + (dims[-1],), BF).expand(dims)
    s["k"] = s["v"] = far(B, 2 ** 32 + T, Hkv, D)
    with pytest.raises(ValueError, match="sizes below"):
        CALLS["window"][0](None, s)
    with pytest.raises(ValueError, match="sizes below"):
        attention_workspace(s["q"], s["k"])
    with pytest.raises(ValueError, match="sizes below"):
        CALLS["write"][0](_cache(), s)
    with pytest.raises(ValueError, match="n_kv_heads"):
        KVCache(2 ** 32 + 1, D, pages=torch.zeros((0, 2 ** 32 + 1, 68 * D), dtype=torch.uint8))
    assert not rec.calls


def test_the_pages_of_a_cache_are_not_replaced():
    c = _cache()
    first, at = c.pages, c._c.pages
    with pytest.raises(AttributeError):
        c.pages = _aligned((20, Hkv, 68 * D), torch.uint8)
    assert c.pages is first and c._c.pages == at == first.data_ptr()


@pytest.mark.parametrize("native", [False, True], ids=["python", "native"])
@pytest.mark.parametrize("name", ["window", "tree", "chain"])
def test_inputs_that_require_a_gradient(name, native, rec, monkeypatch):
    """There is no backward pass: such inputs are refused, and taken where no gradient is recorded."""
    ops = rec.ops()
    if native:
        monkeypatch.setattr(attention, "_native", lambda stream: (_lib.binding(), ops, 0, STREAM))
    for arg in "qkv":
        s = _state()
        s[arg].requires_grad_()
        with pytest.raises(ValueError, match=f"{arg} requires a gradient"):
            CALLS[name][0](_cache(), s)
        assert not rec.calls
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                CALLS[name][0](_cache(), s)
            assert rec.calls
            rec.calls.clear()
    # what is written to a cache, or weighed, has no gradient to lose
    s = _state()
    for arg in "qkv":
        s[arg].requires_grad_()
    for other in ("write", "score"):
        CALLS[other][0](_cache(), s)
        assert rec.calls
        rec.calls.clear()


def test_scores_that_overlap_in_part():
    """One array or two that are apart: a score read after another's new one was written would be wrong."""
    lib, c, a, r = _lib.lib(), _c_cache(), _attention(), ctypes.byref
    size = 2 * 2 * 100 * 4                                # of the scores
    for off in (4, 400, size - 4, -4, 4 - size):
        assert lib.caddtree_cache_score(r(c), r(a), None, 0x10000, 0x10000 + off, 100, None) == INVALID, off
        assert b"overlap" in lib.caddtree_last_error()


def test_keys_and_values_are_not_read_into_one_place():
    lib, c, v, r = _lib.lib(), _c_cache(), _lib.View(0x1000, 640, 128, 64), ctypes.byref
    assert lib.caddtree_cache_read(r(c), r(v), r(v), 2, 5, None, 0x1000, 0x1000, 3, None) == INVALID
    assert b"one place" in lib.caddtree_last_error()


def test_scales_at_the_limit():
    lib, c, r = _lib.lib(), _c_cache(), ctypes.byref
    for scale in (2.0 ** 127 * 1.001, -3e38):
        a = _attention(scale=scale)
        assert lib.caddtree_window_attention(r(a), None, 0, None) == UNSUPPORTED
        assert lib.caddtree_cache_attention(r(c), r(a), None, 0, None) == UNSUPPORTED
        assert lib.caddtree_cache_score(r(c), r(a), None, 0x1000, 0x1000, 100, None) == UNSUPPORTED
    a = _attention(B=0, scale=2.0 ** 127)                 # taken: a call of nothing
    assert lib.caddtree_window_attention(r(a), None, 0, None) == _lib.OK


def test_windows_over_the_longest_sequences():
    """What the kernels subtract in a window's test stays in 32 bits, or the call is refused."""
    lib, c, r = _lib.lib(), _c_cache(), ctypes.byref
    one = dict(B=1, n_heads=2, n_kv_heads=2, window=5)
    for kw in (dict(T=2 ** 30, S=2 ** 30), dict(T=3, S=2 ** 30), dict(T=2 ** 30, S=2 ** 29 + 1)):
        a = _attention(**one, **kw)
        assert lib.caddtree_window_attention(r(a), None, 0, None) == UNSUPPORTED and b"2^31" in lib.caddtree_last_error(), kw
    for kw in (dict(T=2 ** 30, table_pages=1), dict(T=2 ** 29 + 1, table_pages=2 ** 24)):
        a = _attention(**one, **kw)
        assert lib.caddtree_cache_attention(r(c), r(a), None, 0, None) == UNSUPPORTED and b"2^31" in lib.caddtree_last_error(), kw


def test_lse_is_read_in_any_strides(rec, monkeypatch):
    """The scores' lse is an input: a transposed or repeated one is passed on with its strides."""
    f32, ops = torch.float32, rec.ops()
    for native in (False, True):
        monkeypatch.setattr(attention, "_native", lambda stream: (_lib.binding(), ops, 0, STREAM) if native else None)
        for lse, strides in ((_aligned((B, Hq, T), f32).transpose(1, 2), (Hq * T, 1, T)),
                             (_aligned((B, T, 1), f32).expand(B, T, Hq), (T, 1, 0)),
                             (_aligned((1, 1, 1), f32).expand(B, T, Hq), (0, 0, 0)),
                             (_aligned((B, 2 * T, Hq), f32)[:, ::2], (2 * T * Hq, 2 * Hq, 1))):
            rec.calls.clear()
            CALLS["score"][0](_cache(), dict(_state(), lse=lse))
            (_, args), = rec.calls
            a = dict(zip((f for f, _ in _lib.Attention._fields_), args[1]))
            assert a["lse"] == lse.data_ptr() and a["lse_strided"] == 1
            assert (a["lse_stride_b"], a["lse_stride_t"], a["lse_stride_h"]) == strides


def test_strides_of_lse():
    lib, c, r = _lib.lib(), _c_cache(), ctypes.byref
    for kw in (dict(lse_stride_b=-1), dict(lse_stride_t=-1), dict(lse_stride_h=-4)):
        a = _attention(lse_strided=1, **kw)
        assert lib.caddtree_cache_score(r(c), r(a), None, 0x1000, 0x1000, 100, None) == INVALID
    a = _attention(lse_strided=1, lse_stride_b=20, lse_stride_t=4, lse_stride_h=1)
    assert lib.caddtree_window_attention(r(a), None, 0, None) == INVALID        # (written there: contiguous)
    assert lib.caddtree_cache_attention(r(c), r(a), None, 0, None) == INVALID
