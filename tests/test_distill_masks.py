"""Distillation of logits far from 0 or from each other, against its definition in fp64 (tests/_distill_ref.py), on the GPU: finite
masks of any size, in a wavefront's first tokens, in later ones, in nearly all and in all; rows that are large throughout."""

import numpy as np
import pytest
import torch

from paper_2606_01813_amd import adjust_logits, distill, distill_grad, distill_workspace
from tests import _distill_ref as ref

pytestmark = pytest.mark.gpu

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32
STEP = {BF: 2.0 ** -7, F32: 2.0 ** -23}
# a row's vectors by the launch that takes them: 64 threads (two forms), 128, 256, 512, and in fp32 1024
LENGTHS = {F32: [900, 4001, 8003, 16001, 70001, 140001], BF: [1501, 8001, 16005, 30003, 140009]}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _close(got, want, tol, name):
    got = got.detach().double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want))
    if bad.any():
        at = tuple(int(i) for i in np.argwhere(bad)[0]) if bad.ndim else ()
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} off, first at {at}: got {got[at]!r}, want {want[at]!r} +- {tol[at]!r}")


def _every_form(x, ids, target, tau, tail, names, weight=None):
    """Loss with gradient, the loss alone and the gradient from the stats, in whole rows and in parts, a call each."""
    B, T, V = x.shape
    tau = float(np.float32(tau))                           # (a call's temperature is a float: 0.1 (1 + 1.5e-8))
    l, t, i = (a.detach().double().cpu().numpy() for a in (x, target, ids))
    w = np.ones((B, T)) if weight is None else weight.double().cpu().numpy()
    want = [[ref.distill(l[b, r], i[b, r].astype(int), t[b, r], w[b, r], tau, tail, x.dtype, again)
             for b in range(B) for r in range(T)] for again in (False, True)]
    for ws in (None, distill_workspace(x)):
        loss, stats, alone = (torch.full((B, T) + s, 9.0, device="cuda") for s in ((), (3,), ()))
        grad = torch.full_like(x, 9.0)
        kw = dict(temperature=tau, tail=tail, weight=weight)
        distill(x, ids, target, loss, grad=grad, stats=stats, workspace=ws, **kw)
        distill(x, ids, target, alone, workspace=ws, **kw)
        again = distill_grad(x, ids, target, stats, **kw)
        for n in range(B * T):
            b, r = divmod(n, T)
            at = (names[b], V, x.dtype, tau, tail, ws is not None)
            _close(loss[b, r], np.array(want[0][n][0]), np.array(want[0][n][3]), ("loss", at))
            _close(alone[b, r], np.array(want[0][n][0]), np.array(want[0][n][3]), ("loss alone", at))
            _close(stats[b, r], want[0][n][1], want[0][n][4], ("stats", at))
            _close(grad[b, r], want[0][n][2], want[0][n][5], ("grad", at))
            _close(again[b, r], want[1][n][2], want[1][n][5], ("grad from stats", at))
        y = x.clone()
        distill(y, ids, target, alone, grad=y, workspace=ws, **kw)
        assert torch.equal(y, grad) and torch.equal(alone, loss)
        y = x.clone()
        assert torch.equal(distill_grad(y, ids, target, stats, y, **kw), again)


def _teacher(gen, B, V, K, tail):
    ids = torch.stack([torch.randperm(V, generator=gen, device="cuda")[:K] for _ in range(B)]).view(B, 1, K).to(I32)
    target = torch.randn((B, 1, K + 1), generator=gen, device="cuda") * 1.5
    return ids, (torch.log_softmax(target, -1) if tail else target)[..., :K].contiguous()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [0.5, 1.0, 1.5])
@pytest.mark.parametrize("dtype,V", [(d, v) for d in LENGTHS for v in LENGTHS[d]])
def test_finite_masks(dtype, V, tau, tail):
    gen, rows, names = _gen(V), [], []
    K, window = 6, 512
    ids, target = _teacher(gen, 29, V, K, tail)
    for fill in (-1e4, -1e9, -1e10, -1e12, -1e20, -1e30, torch.finfo(dtype).min):
        for where in ("the first tokens", "a middle stretch", "all but a few", "all"):
            x = torch.randn(V, generator=gen, device="cuda") * 2
            n = len(rows)
            if where == "the first tokens":
                x[:window] = fill
            elif where == "a middle stretch":
                x[V // 3:V // 3 + 2 * window] = fill
            else:
                few = torch.cat((ids[n, 0, :K - 1].long(), torch.randint(V, (9,), generator=gen, device="cuda")))
                kept = x[few].clone()
                x[:] = fill
                if where == "all but a few":
                    x[few] = kept
            if where != "all but a few":                   # (one that is listed and masked: a large loss)
                x[ids[n, 0].long()] = torch.where(x[ids[n, 0].long()] == fill, x.max(), x[ids[n, 0].long()])
            rows.append(x)
            names.append((fill, where))
    x = torch.full((V,), -1e30, device="cuda")             # the student leaves the rest nothing
    x[ids[28, 0].long()] = torch.randn(K, generator=gen, device="cuda")
    x = torch.stack(rows + [x]).view(29, 1, V).to(dtype)
    _every_form(x, ids, target, tau, tail, names + ["nothing for the rest"])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("dtype,V", [(F32, 900), (F32, 8003), (F32, 70001), (BF, 8001), (BF, 140009)])
def test_rows_far_from_zero(dtype, V, tau, tail):
    """All of a row at one large value, or a step of its type from it, as a row is that a mask leaves nothing of."""
    gen = _gen(V + 1)
    values = [s * v for v in (2.0 ** 22, 2.0 ** 23, 2.0 ** 24, 1e8, 1e10, 1e12, 1e15, 1e20, 1e30, 3e38) for s in (1, -1)]
    x = torch.tensor(values, device="cuda").to(dtype).view(-1, 1, 1).repeat(1, 1, V)
    x[1::3, 0, 7::11] *= 1 - STEP[dtype]
    ids, target = _teacher(gen, len(values), V, 5, tail)
    _every_form(x, ids, target, tau, tail, values)


@pytest.mark.parametrize("V", [1000, 8001, 40000, 151936])
def test_logits_as_a_grammar_leaves_them(V):
    """adjust_logits with a finite fill, few tokens allowed, and then distilled in the same place."""
    gen, B, T, K = _gen(V + 2), 3, 4, 8
    x = torch.randn((B, T, V), generator=gen, device="cuda") * 2
    few = torch.randint(V, (B, T, 24), generator=gen, device="cuda")
    named = torch.zeros((B, T, (V + 31) // 32 * 32), dtype=torch.bool, device="cuda").scatter_(2, few, True)
    words = (named.view(B, T, -1, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(I32)
    ids = few[..., :K].to(I32).contiguous()
    for dtype in (BF, F32):
        for tau in (1.0, 1.5):
            for tail in (False, True):
                y = x.to(dtype)
                adjust_logits(y, y, allowed=words, fill=-1e30)
                target = torch.randn((B, T, K + 1), generator=gen, device="cuda")
                target = (torch.log_softmax(target, -1) if tail else target)[..., :K].contiguous()
                _every_form(y, ids, target, tau, tail, list(range(B)), weight=torch.rand((B, T), generator=gen, device="cuda") + 0.5)


@pytest.mark.parametrize("tau", [0.1, 0.25, 1.0, 3.0])
@pytest.mark.parametrize("dtype,V", [(F32, 40), (F32, 900), (F32, 4001), (F32, 16001), (F32, 70001), (F32, 140001), (BF, 1501), (BF, 8001),
                                     (BF, 140009), (F16, 33), (F16, 16005)])
def test_the_rest_far_below_the_listed_tokens(dtype, V, tau):
    """The rest's mass is its own sum, wherever the listed tokens lie and however far above the others they are."""
    gen = _gen(V + 3)
    gaps = [9.0, 30.0, 80.0, 86.0, 87.0, 88.0, 90.0, 100.0, 104.0, 120.0, 200.0, 300.0, 500.0, 700.0, 800.0, 2000.0]
    B, K = len(gaps), 5
    ids, target = _teacher(gen, B, V, K, True)
    x = torch.randn((B, 1, V), generator=gen, device="cuda") * tau          # (largest some 4 tau)
    for b, gap in enumerate(gaps):
        if b % 3 == 1:
            ids[b, 0, :2] = torch.tensor([0, V - 1], dtype=I32)
        listed = ids[b, 0].long()
        others = x[b, 0].index_fill(0, listed, -1e9).max()
        x[b, 0, listed] = others - torch.rand(K, generator=gen, device="cuda") * 3 * tau
        x[b, 0, listed[K - 1 if b % 2 else 0]] = others + gap * tau           # (one of them)
        if b % 4 == 3:
            x[b, 0, listed[1]] = others + (gap - 1) * tau
    weight = torch.rand((B, 1), generator=gen, device="cuda") * 64 + 0.5
    _every_form(x.to(dtype), ids, target, tau, True, gaps, weight)
    _every_form(x.to(dtype), ids, target, tau, False, gaps, weight)


def test_where_the_listed_token_lies_does_not_matter():
    """One listed token 88 above the rest, in each of a row's places: the same loss to the bound, in every form of the call."""
    V, n = 4096, 64
    x = torch.randn(V, generator=_gen(4), device="cuda").repeat(n, 1, 1)
    ids = (torch.arange(n, device="cuda") * (V // n)).to(I32).view(n, 1, 1)
    high = x[0].max() + 88
    first = x[0, 0, 0].clone()
    for b in range(n):                                     # (the same numbers in every row: place 0's and the listed one's change seats)
        x[b, 0, 0] = x[b, 0, ids[b, 0, 0].long()]
        x[b, 0, ids[b, 0, 0].long()] = high
    x[0, 0, 0] = high
    assert float(first) != float(high)
    target = torch.full((n, 1, 1), float(np.log(0.9)), device="cuda")
    _every_form(x, ids, target, 1.0, True, list(range(n)))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [2.0 ** -20, 2.0 ** -7, 2.0 ** 20])
@pytest.mark.parametrize("dtype,V", [(F32, 900), (F32, 8003), (F32, 70001), (BF, 16005), (F16, 8001)])
def test_the_smallest_and_largest_temperatures(dtype, V, tau, tail):
    gen, B = _gen(V + 5), 4
    x = (torch.randn((B, 1, V), generator=gen, device="cuda") * 3).to(dtype)
    x[1, 0, :600] = -1e4
    x[2, 0, ::3] = x[2, 0].max()                           # (many at the top)
    ids, target = _teacher(gen, B, V, 4, tail)
    x[3, 0, ids[3, 0].long()] = x[3, 0].max() + 1
    _every_form(x, ids, target, tau, tail, list(range(B)), torch.full((B, 1), min(1.0, tau), device="cuda"))   # (f16 ends at 65504)


@pytest.mark.parametrize("with_workspace", [False, True])
@pytest.mark.parametrize("V", [40, 4001, 16001, 70001, 140001])
def test_a_listed_nan_or_infinity_spreads_over_its_row(V, with_workspace):
    gen, B, K = _gen(V + 6), 4, 3
    x = torch.randn((B, 1, V), generator=gen, device="cuda")
    ids, target = _teacher(gen, B, V, K, True)
    at = ids[:, 0, 1].long()
    x[0, 0, at[0]], x[1, 0, at[1]] = float("nan"), float("inf")
    x[2] = -float("inf")
    x[2, 0, at[2]] = float("nan")                          # (and nothing else)
    x[3, 0, at[3]] = 1e30
    loss, stats, grad = torch.zeros((B, 1), device="cuda"), torch.zeros((B, 1, 3), device="cuda"), torch.zeros_like(x)
    for tail in (True, False):
        distill(x, ids, target, loss, grad=grad, stats=stats, tail=tail, workspace=distill_workspace(x) if with_workspace else None)
        for g in (grad, distill_grad(x, ids, target, stats, tail=tail)):
            assert torch.isnan(g[:3]).flatten(1).all(1).tolist() == [True] * 3 and bool(torch.isfinite(g[3]).all())
        assert torch.isnan(loss[:3, 0]).tolist() == [True] * 3 and bool(torch.isfinite(loss[3]))
