"""What the calls on logits owe autograd, which does not see them (CPU, no GPU needed; host tensors and recording functions as in
test_logits_checks.py): no gradient is lost without a word, and nothing that a backward pass has saved changes unseen."""

import pytest
import torch

from paper_2606_01813_amd import _lib, attention
from tests.test_logits_checks import CALLS, STREAM, _state, rec  # noqa: F401  (a fixture)

FLOATS = [("adjust", n) for n in ("logits", "out", "repetition", "presence", "frequency", "bias")] + [("verify", "logits"), ("verify", "weight")] + \
    [("distill", n) for n in ("logits", "target", "loss", "grad", "stats", "weight")] + \
    [("grad", n) for n in ("logits", "target", "stats", "grad", "weight")]


@pytest.fixture(params=[False, True], ids=["python", "native"])
def calls(request, rec, monkeypatch):  # noqa: F811
    ops = rec.ops()
    monkeypatch.setattr(_lib, "logits_ops", lambda: ops)
    monkeypatch.setattr(attention, "_native", lambda stream: (_lib.binding(), None, 0, STREAM) if request.param else None)
    return rec.calls


@pytest.mark.parametrize("name,arg", FLOATS)
def test_a_tensor_that_requires_a_gradient_is_refused(name, arg, calls):
    s = _state()
    s[arg].requires_grad_()
    with pytest.raises(ValueError, match=f"{arg} requires a gradient"):
        CALLS[name][0](s)
    assert not calls
    with torch.no_grad():
        CALLS[name][0](s)
    assert calls.pop()


WRITTEN = {"adjust": ("out",), "verify": ("accepted", "index", "tokens", "weight"), "walk": ("accepted", "index", "tokens"),
           "distill": ("loss", "grad", "stats"), "grad": ("grad",)}


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_writes_has_another_version(name, calls):
    s = _state()
    before = {n: t._version for n, t in s.items() if isinstance(t, torch.Tensor)}
    CALLS[name][0](s)
    assert {n for n, v in before.items() if s[n]._version != v} == set(WRITTEN[name])
    for n in ("weight", "grad", "stats"):                          # (not given)
        s[n] = None if n not in CALLS[name][1] or name == "distill" else s[n]
    CALLS[name][0](s)
    with torch.inference_mode():
        s = _state()
        CALLS[name][0](s)
    CALLS[name][0](s)                                              # (inference tensors, outside)


@pytest.mark.parametrize("name", ["adjust", "distill", "grad"])
def test_a_backward_pass_through_an_overwritten_output_is_refused(name, calls):
    """A drafter whose last step saved its output, which a call then overwrites."""
    s = _state()
    w = torch.zeros(s["logits"].shape, dtype=torch.bfloat16, requires_grad=True)
    logits = 30 * torch.tanh(w)
    capped = torch.tanh(w)
    for out, ok in ((logits, True), (capped, False)):
        s["logits"] = s["grad"] = s["out"] = out.detach()
        CALLS[name][0](s)
        if ok:
            out.backward(torch.ones_like(out))
        else:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                out.backward(torch.ones_like(out))
