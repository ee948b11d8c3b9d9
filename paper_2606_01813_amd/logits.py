"""Operators on logits: what stands before and behind a draft tree, and what trains its drafter.

    adjust_logits(logits, logits, history=text, history_len=length, repetition=r, presence=p, frequency=f,
                  bias_ids=ids, bias=values, allowed=words, fill=-1e30)       # penalties, biases, a grammar's mask
    plan.build(logits, tree, workspace=ws)
    ...                                                                       # the target's logits [B, 1 + cap, V] at the tree
    adjust_logits(target, target, history=text, history_len=length, repetition=r, token_ids=tree.token_ids,
                  parent=tree.parent, count=tree.n_star)                      # ... with the tokens on each row's path
    verify_tree(target, tree.token_ids, tree.parent, tree.n_star, accepted, index, tokens, weight=on_path)
    cache.write(k, v, table, ctx_len, count=accepted, index=index)            # what verify_tree wrote are its arguments
    cache.score(q, table, ctx_len, lse, scores, weight=on_path, count=tree.n_star, depth=tree.depth)

    plan.reduce_topk(teacher_logits, ids, top, lse, lq)                       # a teacher's top tokens
    distill(student.detach(), ids, top, loss, grad=grad, weight=w)            # the drafter's loss and its gradient
    student.backward(grad)                                                    # ... through the drafter

Every call checks its tensors, then enqueues kernels on the stream (default: torch's current one) and returns.  Logits are
bf16, f16 or f32 [B, rows, V] with a unit last stride, in any strides.  include/caddtree.h states what is computed.
Autograd does not see these calls: ``distill`` writes the logits' gradient itself, and a tensor that requires one, be it the
logits, a bias, a teacher's logits or a weight, is refused while gradients are recorded.  What a call writes counts as changed in
place: where a layer saved its output for its backward pass (tanh, softmax), adjusting that output's detached form in place, or
writing the gradient over it, makes the backward pass raise an error; give the call an output of its own there.

As a plan's calls do, these go to the native binding first, which checks the tensors and calls the library; what it cannot
vouch for comes back as None and takes the Python checks here, which raise what is wrong.
"""

from __future__ import annotations

import ctypes
import math

from . import _lib
from . import attention as _at

__all__ = ["adjust_logits", "verify_tree", "verify_workspace", "distill", "distill_grad", "distill_workspace"]


def _torch():
    import torch
    return torch


def _dtype(name: str, t) -> int:
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor, got {type(t).__name__}")
    got = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}.get(t.dtype)
    if got is None:
        raise TypeError(f"{name} must be torch.bfloat16, torch.float16 or torch.float32, got {t.dtype}")
    return _lib.LOGIT_DTYPES[got]


def _no_gradient(name: str, t, instead: str) -> None:
    torch = _torch()
    if torch.is_grad_enabled() and isinstance(t, torch.Tensor) and t.requires_grad:
        raise ValueError(f"{name} requires a gradient, which autograd does not carry through this call: {instead}")


def _wrote(*tensors) -> None:
    """Tells autograd what a call wrote (None: not given): a backward pass that saved one of them is refused."""
    for t in tensors:
        if t is not None and not t.is_inference():
            _torch().autograd.graph.increment_version(t)


def _no_gradients(**others) -> None:
    for name, t in others.items():
        _no_gradient(name, t, f"call it under torch.no_grad(), or detach {name}")


def _rows(name: str, t, dtype, shape, device: int) -> _lib.Rows:
    """A [B, T, V] tensor with a unit last stride."""
    _at._tensor(name, t, dtype, device)
    if t.dim() != 3 or any(w is not None and w != g for w, g in zip(shape, t.shape)):
        raise ValueError(f"{name} must have shape {tuple('any' if w is None else w for w in shape)}, got {tuple(t.shape)}")
    _at._sizes(name, t)
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name} must have a unit last stride, got {t.stride()}")
    sb, st = (s if n > 1 else 0 for s, n in zip(t.stride(), t.shape[:2]))     # the stride of one element is free
    return _lib.Rows(t.data_ptr(), sb, st)


def _logits(a, t, device: int) -> None:
    a.dtype = _dtype("logits", t)
    a.logits = _rows("logits", t, t.dtype, (None,) * 3, device)
    a.B, a.T, a.V = t.shape


def adjust_logits(logits, out=None, *, history=None, history_len=None, repetition=None, presence=None, frequency=None,
                  bias_ids=None, bias=None, allowed=None, token_ids=None, parent=None, count=None,
                  fill: float = -math.inf, stream=None):
    """Penalties for the tokens of ``history`` (int32 [B, H], the first history_len[b] of each), biases and a mask on
    logits [B, T, V], into ``out`` (the logits themselves: in place; made of zeros if not given).  Returns out.

    A logit x of a token that occurred c > 0 times becomes x / repetition[b] (x repetition[b] if not positive), less
    frequency[b] c and presence[b] (float32 [B] each); bias[b, j] (float32 [B, n]) is added to token bias_ids[b, j]
    (int32); a token whose bit is not set in ``allowed`` (int32 or uint32 words [B, T, ceil(V / 32)], in any strides of
    its first two dimensions) becomes ``fill``: -inf (0 stands for it too, and so does what is past the logits' type, as
    -1e30 is in f16), or for the drafter's logits, of which a plan's calls want finite ones, a finite value.  Ids outside the vocabulary are padding; of a token listed twice the last
    bias counts.  With ``token_ids`` and ``parent`` (int32 [B, T - 1]) the rows are a tree's, row 0 its root and row i
    node i - 1, and a row's path counts as its history too.  ``count`` (int32 [B]): the rows of each sequence, in a
    tree its n_star; rows past it are left as they are."""
    out = _at._made(logits, out, stream)
    native = _at._native(stream)
    if native is not None and _lib.logits_ops() is not None:
        binding, _, device, raw = native
        if _at._done(binding.adjust_logits(_lib.logits_ops(), device, raw, logits, out, history, history_len, repetition, presence,
                                           frequency, bias_ids, bias, allowed, token_ids, parent, count, fill)):
            return out
    _no_gradients(logits=logits, out=out, repetition=repetition, presence=presence, frequency=frequency, bias=bias)
    torch = _torch()
    device = _at._device()
    a = _lib.Adjust()
    _logits(a, logits, device)
    a.out = _rows("out", out, logits.dtype, tuple(logits.shape), device)
    i32, f32 = torch.int32, torch.float32
    a.fill = float(fill)
    if history is not None:
        a.history, a.H = _at._array("history", history, i32, (a.B, None), device), history.shape[1]
    elif history_len is not None:
        raise ValueError("history_len is given without history")
    if history_len is not None:
        a.history_len = _at._array("history_len", history_len, i32, (a.B,), device)
    for name, t in (("repetition", repetition), ("presence", presence), ("frequency", frequency)):
        if t is not None:
            setattr(a, name, _at._array(name, t, f32, (a.B,), device))
    if (bias_ids is None) != (bias is None):
        raise ValueError("bias_ids and bias are given together")
    if bias is not None:
        a.bias_ids = _at._array("bias_ids", bias_ids, i32, (a.B, None), device)
        a.n_bias = bias_ids.shape[1]
        a.bias = _at._array("bias", bias, f32, (a.B, a.n_bias), device)
    if allowed is not None:
        if not isinstance(allowed, torch.Tensor) or allowed.dtype not in (i32, getattr(torch, "uint32", i32)):
            raise TypeError("allowed must be int32 or uint32 words")
        m = _rows("allowed", allowed, allowed.dtype, (a.B, a.T, (a.V + 31) // 32), device)
        a.allowed, a.allowed_stride_b, a.allowed_stride_t = m.data, m.stride_b, m.stride_t
    if (token_ids is None) != (parent is None):
        raise ValueError("a tree needs both token_ids and parent")
    if parent is not None:
        if a.T < 1:
            raise ValueError("a tree's logits need a row for its root")
        a.token_ids = _at._array("token_ids", token_ids, i32, (a.B, a.T - 1), device)
        a.parent = _at._array("parent", parent, i32, (a.B, a.T - 1), device)
    if count is not None:
        a.count = _at._array("count", count, i32, (a.B,), device)
        if parent is not None and a.T == 1:                # (the root alone: no nodes to count, and no arrays that say a tree)
            a.count = None
    _lib.check(_lib.lib().caddtree_adjust_logits(ctypes.byref(a), _at._stream(stream, device)))
    _wrote(out)
    return out


def verify_tree(logits, token_ids, parent, count, accepted, index, tokens, *, chosen=None, weight=None, workspace=None,
                stream=None) -> None:
    """The path of a built tree that the target agrees with: from the root on, the largest logit's token (of equals the
    lowest id; NaN and -inf are never chosen), then the child that carries it.

    logits [B, 1 + cap, V] are the target's at the root and the nodes, token_ids and parent (int32 [B, cap]) and count
    (int32 [B], n_star) the tree's.  Or ``chosen`` (int32 [B, 1 + cap]; logits None) holds the target's tokens, drawn
    by the caller.  Writes ``accepted`` (int32 [B]: rows on the path, the root's among them), ``index`` (int32 [B, M]:
    which, then -1), ``tokens`` (int32 [B, M]: each one's token, the last of them the bonus token, then -1; a row where
    nothing can be chosen has -1 as well) and ``weight`` (float32 [B, 1 + cap]: 1 on the path, else 0).  M, at most
    1 + L rows of a path, is the size of index."""
    native = _at._native(stream)
    if native is not None and _lib.logits_ops() is not None:
        binding, _, device, raw = native
        if _at._done(binding.verify_tree(_lib.logits_ops(), device, raw, logits, token_ids, parent, count, accepted, index, tokens,
                                         chosen, weight, workspace)):
            return
    _no_gradients(logits=logits, weight=weight)
    torch = _torch()
    device = _at._device()
    i32 = torch.int32
    if (logits is None) == (chosen is None):
        raise ValueError("either logits or chosen is given")
    a = _lib.Verify()
    if logits is not None:
        _logits(a, logits, device)
    else:
        a.chosen = _at._array("chosen", chosen, i32, (None, None), device)
        a.B, a.T = chosen.shape
        a.V = 1
    if a.T < 1:
        raise ValueError("a tree needs a row for its root")
    a.token_ids = _at._array("token_ids", token_ids, i32, (a.B, a.T - 1), device)
    a.parent = _at._array("parent", parent, i32, (a.B, a.T - 1), device)
    a.count = _at._array("count", count, i32, (a.B,), device)
    a.accepted = _at._array("accepted", accepted, i32, (a.B,), device)
    a.index = _at._array("index", index, i32, (a.B, None), device)
    a.M = index.shape[1]
    a.tokens = _at._array("tokens", tokens, i32, (a.B, a.M), device)
    if weight is not None:
        a.weight = _at._array("weight", weight, torch.float32, (a.B, a.T), device)
    ws, n = _at._workspace(workspace, device)
    _lib.check(_lib.lib().caddtree_verify_tree(ctypes.byref(a), ws, n, _at._stream(stream, device)))
    _wrote(accepted, index, tokens, weight)


def verify_workspace(logits):
    """A workspace for ``verify_tree`` of these logits (uint8; the contents do not matter)."""
    a = _lib.Verify()
    a.dtype = _dtype("logits", logits)
    _at._sizes("logits", logits)
    a.B, a.T, a.V = logits.shape
    return _torch().empty(max(int(_lib.lib().caddtree_verify_workspace_bytes(ctypes.byref(a))), 1), dtype=_torch().uint8,
                          device=logits.device)


def _distill(logits, ids, target, stats, grad, weight, temperature, tail, device: int):
    torch = _torch()
    a = _lib.Distill()
    _logits(a, logits, device)
    a.ids = _at._array("ids", ids, torch.int32, (a.B, a.T, None), device)
    a.K = ids.shape[2]
    a.target = _at._array("target", target, torch.float32, (a.B, a.T, a.K), device)
    if weight is not None:
        a.weight = _at._array("weight", weight, torch.float32, (a.B, a.T), device)
    if stats is not None:
        a.stats = _at._array("stats", stats, torch.float32, (a.B, a.T, 3), device)
    if grad is not None:
        a.grad = _rows("grad", grad, logits.dtype, tuple(logits.shape), device)
    a.temperature, a.tail = float(temperature), 1 if tail else 0
    return a


def distill(logits, ids, target, loss, *, grad=None, stats=None, weight=None, temperature: float = 1.0, tail: bool = False,
            workspace=None, stream=None) -> None:
    """The divergence of a student's logits [B, T, V] from a teacher's top tokens ``ids`` (int32 [B, T, K], as
    ``Plan.reduce_topk`` writes them; outside the vocabulary: padding), and its gradient.

    ``target`` (float32 [B, T, K]) are the teacher's logits, whose softmax at the temperature makes up its distribution;
    with ``tail`` its log-probabilities (reduce_topk's topk_lq), and what they leave is the probability of all other
    tokens.  Writes loss[b, t] = weight[b, t] KL(teacher || student at the temperature) (float32 [B, T]), ``grad`` (of
    the logits' shape and type: the gradient of loss.sum(); it may be the logits themselves) and ``stats`` (float32
    [B, T, 3], for ``distill_grad``).  Rows of weight 0 are not read: their loss, gradient and stats are 0."""
    native = _at._native(stream)
    if native is not None and _lib.logits_ops() is not None:
        binding, _, device, raw = native
        if _at._done(binding.distill(_lib.logits_ops(), device, raw, logits, ids, target, loss, grad, stats, weight, temperature, tail,
                                     workspace)):
            return
    _no_gradient("logits", logits, "pass logits.detach() and grad, then call logits.backward(grad)")
    _no_gradients(target=target, loss=loss, grad=grad, stats=stats, weight=weight)
    device = _at._device()
    a = _distill(logits, ids, target, stats, grad, weight, temperature, tail, device)
    a.loss = _at._array("loss", loss, _torch().float32, (a.B, a.T), device)
    ws, n = _at._workspace(workspace, device)
    _lib.check(_lib.lib().caddtree_distill(ctypes.byref(a), ws, n, _at._stream(stream, device)))
    _wrote(loss, grad, stats)


def distill_grad(logits, ids, target, stats, grad=None, *, weight=None, temperature: float = 1.0, tail: bool = False,
                 workspace=None, stream=None):
    """The gradient of ``distill`` by itself, from the ``stats`` that it wrote of the same logits, ids and temperature
    (weight: the gradient of its losses times their weights).  Into ``grad`` (made of zeros if not given; it may be the
    logits).  Returns grad.  A workspace is taken, as ``distill``'s arguments are, and not used."""
    grad = _at._made(logits, grad, stream)
    native = _at._native(stream)
    if native is not None and _lib.logits_ops() is not None:
        binding, _, device, raw = native
        if _at._done(binding.distill_grad(_lib.logits_ops(), device, raw, logits, ids, target, stats, grad, weight, temperature, tail)):
            return grad
    _no_gradient("logits", logits, "pass logits.detach(), then call logits.backward(grad)")
    _no_gradients(target=target, stats=stats, grad=grad, weight=weight)
    device = _at._device()
    if stats is None:
        raise TypeError("stats must be a torch tensor, got NoneType")
    a = _distill(logits, ids, target, stats, grad, weight, temperature, tail, device)
    _lib.check(_lib.lib().caddtree_distill_grad(ctypes.byref(a), _at._stream(stream, device)))
    _wrote(grad)
    return grad


def distill_workspace(logits):
    """A workspace for ``distill`` of these logits (uint8; the contents do not matter)."""
    a = _lib.Distill()
    a.dtype = _dtype("logits", logits)
    _at._sizes("logits", logits)
    a.B, a.T, a.V = logits.shape
    a.K, a.temperature = 1, 1.0
    return _torch().empty(max(int(_lib.lib().caddtree_distill_workspace_bytes(ctypes.byref(a))), 1), dtype=_torch().uint8,
                          device=logits.device)
