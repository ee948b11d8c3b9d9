"""What the calls on logits refuse (CPU, no GPU needed): the Python checks, the native calls against them, and the library's
own checks of a C caller's arguments.

Over forms of every argument a native call either passes the library exactly what the Python path passes it, or returns
None and leaves the call to the Python path; what the Python path refuses it never passes on.  Host tensors stand in for
device ones, and recording functions for the library's.
"""

import ctypes

import numpy as np
import pytest
import torch

from paper_2606_01813_amd import (_lib, adjust_logits, attention, distill, distill_grad, distill_workspace, verify_tree,
                                  verify_workspace)

STREAM = 0x1234
B, T, V, H, N, K, M = 2, 5, 70, 6, 3, 4, 4
BF, I32, F32 = torch.bfloat16, torch.int32, torch.float32
NAMES = ("adjust_logits", "verify_tree", "distill", "distill_grad")


def _flat(a):
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
        return _lib.binding().logits_ops(1, *(ctypes.cast(getattr(self, "caddtree_" + n), ctypes.c_void_p).value for n in NAMES))


@pytest.fixture
def rec(monkeypatch):
    r = _Recorder()
    monkeypatch.setattr(attention, "_on_device", lambda t, device: t.device.type == "cpu")
    monkeypatch.setattr(attention, "_device", lambda: 0)
    monkeypatch.setattr(attention, "_stream", lambda stream, device: STREAM)
    monkeypatch.setattr(attention, "_native", lambda stream: None)
    monkeypatch.setattr(_lib, "lib", lambda: r)
    return r


def _state():
    z = lambda *s, t=I32: torch.zeros(s, dtype=t)
    return {"logits": z(B, T, V, t=BF), "out": z(B, T, V, t=BF), "history": z(B, H), "history_len": z(B), "repetition": z(B, t=F32),
            "presence": z(B, t=F32), "frequency": z(B, t=F32), "bias_ids": z(B, N), "bias": z(B, N, t=F32), "allowed": z(B, T, 3),
            "token_ids": z(B, T - 1), "parent": z(B, T - 1), "count": z(B), "fill": -2.0, "accepted": z(B), "index": z(B, M),
            "tokens": z(B, M), "chosen": z(B, T), "weight": z(B, T, t=F32), "workspace": z(512, t=torch.uint8), "ids": z(B, T, K),
            "target": z(B, T, K, t=F32), "loss": z(B, T, t=F32), "grad": z(B, T, V, t=BF), "stats": z(B, T, 3, t=F32),
            "temperature": 2.0, "tail": True}


ADJUST = ("history", "history_len", "repetition", "presence", "frequency", "bias_ids", "bias", "allowed", "token_ids", "parent", "count", "fill")
CALLS = {
    "adjust": (lambda s: adjust_logits(s["logits"], s["out"], **{n: s[n] for n in ADJUST}), ("logits", "out") + ADJUST),
    "verify": (lambda s: verify_tree(s["logits"], s["token_ids"], s["parent"], s["count"], s["accepted"], s["index"], s["tokens"],
                                     weight=s["weight"], workspace=s["workspace"]),
               ("logits", "token_ids", "parent", "count", "accepted", "index", "tokens", "weight", "workspace")),
    "walk": (lambda s: verify_tree(None, s["token_ids"], s["parent"], s["count"], s["accepted"], s["index"], s["tokens"],
                                   chosen=s["chosen"]), ("chosen", "token_ids", "parent", "count", "index")),
    "distill": (lambda s: distill(s["logits"], s["ids"], s["target"], s["loss"], grad=s["grad"], stats=s["stats"], weight=s["weight"],
                                  temperature=s["temperature"], tail=s["tail"], workspace=s["workspace"]),
                ("logits", "ids", "target", "loss", "grad", "stats", "weight", "temperature", "tail", "workspace")),
    "grad": (lambda s: distill_grad(s["logits"], s["ids"], s["target"], s["stats"], s["grad"], weight=s["weight"],
                                    temperature=s["temperature"], tail=s["tail"]),
             ("logits", "ids", "target", "stats", "grad", "weight", "temperature", "tail")),
}


def _forms(x):
    """Other forms of an argument."""
    yield None
    yield "text"
    if not isinstance(x, torch.Tensor):
        yield from (0, 1, -1, 7, 1.5, 0.0, float("inf"), float("nan"), True, False, np.float64(3))
        return
    yield np.zeros(3)
    yield torch.nn.Parameter(x.clone(), requires_grad=False) if x.is_floating_point() else x.clone()
    if x.is_floating_point():
        yield x.clone().requires_grad_()
    for dt in (torch.int32, torch.int64, torch.float32, BF, torch.float16, torch.uint8, torch.uint32, torch.float64):
        yield torch.zeros(x.shape, dtype=dt)
    for d in range(x.dim()):
        for n in (0, 1, x.shape[d] - 1, x.shape[d] + 1):
            yield torch.zeros(x.shape[:d] + (n,) + x.shape[d + 1:], dtype=x.dtype)
        yield torch.zeros(x.shape[:d] + (2 * x.shape[d],) + x.shape[d + 1:], dtype=x.dtype)[(slice(None),) * d + (slice(None, None, 2),)]
        yield torch.zeros(x.shape[:d] + (1,) + x.shape[d + 1:], dtype=x.dtype).expand(x.shape)
    yield torch.zeros(tuple(x.shape) + (1,), dtype=x.dtype)
    yield torch.zeros(x.numel() + 1, dtype=x.dtype)[1:].view(x.shape)
    if x.dim() == 3:
        yield torch.zeros((x.shape[1], x.shape[0], x.shape[2]), dtype=x.dtype).transpose(0, 1)
        yield torch.zeros(x.shape[:2] + (x.shape[2] + 5,), dtype=x.dtype)[..., 2:-3]


@pytest.mark.parametrize("name", CALLS)
def test_native_calls_pass_on_what_the_python_path_does_or_leave_it_to_it(name, rec, monkeypatch):
    call, args = CALLS[name]
    ops, passed = rec.ops(), 0
    monkeypatch.setattr(_lib, "logits_ops", lambda: ops)

    def run(state, native):
        monkeypatch.setattr(attention, "_native", lambda stream: (_lib.binding(), None, 0, STREAM) if native else None)
        rec.calls.clear()
        try:
            call(state)
        except Exception as e:
            return type(e), repr(rec.calls)
        return None, repr(rec.calls)                              # (repr: a NaN is equal to itself)

    base = _state()
    assert run(base, False) == run(base, True) and rec.calls
    # the native call itself took the plain form (the Python path is not there to fall back on)
    with monkeypatch.context() as m:
        m.setattr(attention, "_tensor", lambda *a: pytest.fail("the Python checks were needed"))
        assert run(base, True)[0] is None
    for arg in args:
        for form in _forms(base[arg]):
            state = dict(base, **{arg: form})
            if arg in ("out", "grad") and form is None and name != "distill":
                continue                                          # made by the call: another place each time
            plain, native = run(state, False), run(state, True)
            assert plain == native, (arg, form if not isinstance(form, torch.Tensor) else (form.dtype, form.shape, form.stride()))
            passed += plain[0] is None
    assert passed > len(args)


REFUSED = [
    ("adjust", "logits", lambda s: s["logits"].double(), TypeError),
    ("adjust", "logits", lambda s: s["logits"][0], ValueError),
    ("adjust", "logits", lambda s: torch.zeros((B, V, T), dtype=BF).transpose(1, 2), ValueError),
    ("adjust", "logits", lambda s: s["logits"].requires_grad_(), ValueError),
    ("adjust", "out", lambda s: s["out"].float(), TypeError),
    ("adjust", "out", lambda s: s["out"][..., 1:], ValueError),
    ("adjust", "history", lambda s: s["history"].long(), TypeError),
    ("adjust", "history", lambda s: None, ValueError),
    ("adjust", "history_len", lambda s: s["history_len"].long(), TypeError),
    ("adjust", "repetition", lambda s: 1.3, TypeError),
    ("adjust", "bias", lambda s: s["bias"][:, 1:], ValueError),
    ("adjust", "bias_ids", lambda s: None, ValueError),
    ("adjust", "allowed", lambda s: s["allowed"][..., :2], ValueError),
    ("adjust", "allowed", lambda s: s["allowed"].long(), TypeError),
    ("adjust", "allowed", lambda s: torch.ones((B, T, V), dtype=torch.bool), TypeError),
    ("adjust", "parent", lambda s: None, ValueError),
    ("adjust", "parent", lambda s: s["parent"][:, 1:], ValueError),
    ("adjust", "count", lambda s: s["count"].long(), TypeError),
    ("verify", "logits", lambda s: None, ValueError),
    ("verify", "logits", lambda s: s["logits"].requires_grad_(), ValueError),
    ("verify", "token_ids", lambda s: torch.zeros((B, T), dtype=I32), ValueError),
    ("verify", "index", lambda s: s["index"].long(), TypeError),
    ("verify", "tokens", lambda s: s["tokens"][:, 1:], ValueError),
    ("verify", "weight", lambda s: s["weight"][:, 1:], ValueError),
    ("verify", "workspace", lambda s: 3, ValueError),
    ("walk", "chosen", lambda s: s["chosen"].long(), TypeError),
    ("walk", "chosen", lambda s: None, ValueError),
    ("distill", "logits", lambda s: s["logits"].requires_grad_(), ValueError),
    ("distill", "ids", lambda s: s["ids"].long(), TypeError),
    ("distill", "ids", lambda s: s["ids"][0], ValueError),
    ("distill", "target", lambda s: s["target"][..., 1:], ValueError),
    ("distill", "target", lambda s: s["target"].to(BF), TypeError),
    ("distill", "loss", lambda s: None, TypeError),
    ("distill", "loss", lambda s: s["loss"].to(BF), TypeError),
    ("distill", "grad", lambda s: s["grad"].float(), TypeError),
    ("distill", "stats", lambda s: torch.zeros((B, T, 2)), ValueError),
    ("distill", "temperature", lambda s: None, TypeError),
    ("grad", "stats", lambda s: None, TypeError),
    ("grad", "weight", lambda s: s["weight"].double(), TypeError),
]


@pytest.mark.parametrize("case", REFUSED, ids=[f"{c[0]}-{c[1]}-{i}" for i, c in enumerate(REFUSED)])
def test_refused_before_the_library_is_called(case, rec):
    name, arg, form, error = case
    s = _state()
    s[arg] = form(s)
    with pytest.raises(error):
        CALLS[name][0](s)
    assert not rec.calls


def test_gradients_are_refused_only_while_they_are_recorded(rec):
    for name in ("adjust", "verify", "distill", "grad"):
        s = _state()
        s["logits"].requires_grad_()
        with torch.no_grad():
            CALLS[name][0](s)
        assert rec.calls.pop()


def test_host_tensors_and_other_devices_are_refused(monkeypatch):
    monkeypatch.setattr(attention, "_device", lambda: 0)
    monkeypatch.setattr(attention, "_native", lambda stream: None)
    for name in CALLS:
        with pytest.raises(ValueError, match="cuda:0"):
            CALLS[name][0](_state())


def test_a_raw_stream_handle_needs_the_outputs(rec):
    s = _state()
    with pytest.raises(ValueError, match="out is required"):
        adjust_logits(s["logits"], stream=STREAM)
    with pytest.raises(ValueError, match="out is required"):
        distill_grad(s["logits"], s["ids"], s["target"], s["stats"], stream=STREAM)


def test_workspaces():
    x = torch.zeros((1, 3, 100), dtype=BF)
    for make in (verify_workspace, distill_workspace):
        assert make(x).dtype == torch.uint8 and make(x).numel() >= 1
        with pytest.raises(TypeError):
            make(x.double())


# ---------------------------------------------------------------- a C caller's arguments

INVALID, UNSUPPORTED, WORKSPACE = _lib.E_INVALID, _lib.E_UNSUPPORTED, _lib.E_WORKSPACE
AT = {n: 0x10000000 * (i + 1) for i, n in enumerate(
    ("logits", "out", "grad", "count", "history", "history_len", "repetition", "presence", "frequency", "bias_ids", "bias", "allowed",
     "token_ids", "parent", "accepted", "index", "tokens", "weight", "ids", "target", "loss", "stats", "chosen"))}


def _args(cls, **kw):
    a = cls()
    d = dict(dtype=1, B=2, T=5, V=70, H=6, n_bias=3, M=4, K=4, temperature=1.0, tail=0, allowed_stride_b=15, allowed_stride_t=3)
    d.update({n: (AT[n], 350, 70) if n in ("logits", "out", "grad") else AT[n] for n in AT})
    if cls is _lib.Verify:
        d["chosen"] = None
    d.update(kw)
    for f, _ in cls._fields_:
        if f in d:
            setattr(a, f, _lib.Rows(*d[f]) if isinstance(d[f], tuple) else d[f])
    return a


SIZES = [(dict(dtype=7), INVALID), (dict(dtype=-1), INVALID), (dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(B=2 ** 19 + 1), UNSUPPORTED),
         (dict(T=2 ** 19 + 1), UNSUPPORTED), (dict(V=0), INVALID), (dict(V=-5), INVALID), (dict(V=2 ** 20 + 1), UNSUPPORTED),
         (dict(logits=(AT["logits"] + 1, 350, 70)), INVALID), (dict(logits=(AT["logits"], -350, 70)), INVALID),
         (dict(logits=(AT["logits"], 350, -70)), INVALID), (dict(logits=(AT["logits"], 2 ** 41, 70)), UNSUPPORTED)]
GRAD = [(dict(grad=(AT["grad"], 350, 69)), INVALID), (dict(grad=(AT["grad"], 70, 70)), INVALID), (dict(grad=(AT["grad"], 0, 70)), INVALID),
        (dict(grad=(AT["grad"] + 1, 350, 70)), INVALID), (dict(grad=(AT["logits"] + 2, 350, 70)), INVALID),
        (dict(grad=(AT["logits"], 420, 70)), INVALID), (dict(grad=(AT["ids"], 350, 70)), INVALID), (dict(grad=(AT["weight"] - 4, 350, 70)), INVALID),
        (dict(logits=(AT["grad"], 350, 70), target=AT["grad"] + 64), INVALID)]


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(logits=(None, 350, 70)), INVALID), (dict(out=(None, 350, 70)), INVALID), (dict(H=-1), INVALID), (dict(H=2 ** 20), UNSUPPORTED),
    (dict(n_bias=-1), INVALID), (dict(n_bias=4096), UNSUPPORTED), (dict(bias=None), INVALID), (dict(bias_ids=None), INVALID),
    (dict(parent=None), INVALID), (dict(token_ids=None), INVALID), (dict(T=4098), UNSUPPORTED), (dict(allowed=AT["allowed"] + 2), INVALID),
    (dict(allowed_stride_b=-1), INVALID), (dict(allowed_stride_t=-1), INVALID), (dict(out=(AT["out"], 350, 69)), INVALID),
    (dict(out=(AT["out"], 349, 70)), INVALID), (dict(out=(AT["out"], 0, 70)), INVALID), (dict(out=(AT["logits"] + 2, 350, 70)), INVALID),
    (dict(out=(AT["logits"], 700, 70)), INVALID), (dict(out=(AT["history"], 350, 70)), INVALID), (dict(out=(AT["allowed"] + 8, 350, 70)), INVALID),
    (dict(out=(AT["parent"], 350, 70)), INVALID), (dict(fill=float("nan")), INVALID),
    (dict(T=2 ** 19, V=2 ** 20, parent=None, token_ids=None), UNSUPPORTED)])
def test_adjust_validation(kw, status):
    a = _args(_lib.Adjust, **kw)
    assert _lib.lib().caddtree_adjust_logits(ctypes.byref(a), None) == status, _lib.lib().caddtree_last_error()
    assert _lib.lib().caddtree_last_error()


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(logits=(None, 0, 0)), INVALID), (dict(chosen=AT["chosen"]), INVALID), (dict(T=0), INVALID), (dict(T=4098), UNSUPPORTED),
    (dict(M=0), INVALID), (dict(count=None), INVALID), (dict(token_ids=None), INVALID), (dict(parent=None), INVALID),
    (dict(accepted=None), INVALID), (dict(index=None), INVALID), (dict(tokens=None), INVALID), (dict(index=AT["tokens"]), INVALID),
    (dict(accepted=AT["count"]), INVALID), (dict(weight=AT["logits"] + 16), INVALID), (dict(weight=AT["parent"]), INVALID)])
def test_verify_validation(kw, status):
    a = _args(_lib.Verify, **kw)
    assert _lib.lib().caddtree_verify_tree(ctypes.byref(a), None, 0, None) == status, _lib.lib().caddtree_last_error()


@pytest.mark.parametrize("kw,status", SIZES + GRAD + [
    (dict(logits=(None, 350, 70)), INVALID), (dict(K=0), INVALID), (dict(K=257), UNSUPPORTED), (dict(temperature=0.0), INVALID),
    (dict(temperature=-1.0), INVALID), (dict(temperature=float("nan")), INVALID), (dict(temperature=float("inf")), INVALID),
    (dict(temperature=2.0 ** -21), INVALID), (dict(tail=2), INVALID), (dict(ids=None), INVALID), (dict(target=None), INVALID)])
def test_distill_validation(kw, status):
    lib, a = _lib.lib(), _args(_lib.Distill, **kw)
    assert lib.caddtree_distill(ctypes.byref(a), None, 0, None) == status, lib.caddtree_last_error()
    assert lib.caddtree_distill_grad(ctypes.byref(a), None) == status, lib.caddtree_last_error()


def test_other_refusals_and_calls_of_nothing():
    lib, r = _lib.lib(), ctypes.byref
    assert lib.caddtree_adjust_logits(None, None) == INVALID
    assert lib.caddtree_verify_tree(None, None, 0, None) == INVALID
    assert lib.caddtree_distill(None, None, 0, None) == INVALID and lib.caddtree_distill_grad(None, None) == INVALID
    assert lib.caddtree_verify_workspace_bytes(None) == 0 and lib.caddtree_distill_workspace_bytes(None) == 0
    assert lib.caddtree_verify_workspace_bytes(r(_args(_lib.Verify, B=-1))) == 0
    assert lib.caddtree_distill_workspace_bytes(r(_args(_lib.Distill, V=0))) == 0
    assert lib.caddtree_verify_tree(r(_args(_lib.Verify)), 0x1010, 100, None) == WORKSPACE
    assert lib.caddtree_distill(r(_args(_lib.Distill)), 0x1010, 100, None) == WORKSPACE
    assert lib.caddtree_distill(r(_args(_lib.Distill, loss=None)), None, 0, None) == INVALID
    assert lib.caddtree_distill(r(_args(_lib.Distill, loss=AT["stats"])), None, 0, None) == INVALID
    assert lib.caddtree_distill(r(_args(_lib.Distill, grad=(AT["loss"], 350, 70))), None, 0, None) == INVALID
    assert lib.caddtree_distill_grad(r(_args(_lib.Distill, stats=None)), None) == INVALID
    assert lib.caddtree_distill_grad(r(_args(_lib.Distill, grad=(None, 0, 0))), None) == INVALID
    assert lib.caddtree_distill_grad(r(_args(_lib.Distill, T=2 ** 19, V=2 ** 18, dtype=0)), None) == UNSUPPORTED   # 2^25 workgroups
    for kw in (dict(B=0), dict(T=0)):
        assert lib.caddtree_adjust_logits(r(_args(_lib.Adjust, parent=None, token_ids=None, **kw)), None) == _lib.OK
        assert lib.caddtree_distill(r(_args(_lib.Distill, **kw)), None, 0, None) == _lib.OK
        assert lib.caddtree_distill_grad(r(_args(_lib.Distill, **kw)), None) == _lib.OK
    assert lib.caddtree_verify_tree(r(_args(_lib.Verify, B=0)), None, 0, None) == _lib.OK
