"""What the calls on logits owe autograd, which does not see them (CPU, no GPU needed; host tensors and recording functions as in
test_logits_checks.py): no gradient is lost without a word."""

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
