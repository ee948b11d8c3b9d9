"""Operators on logits against their definitions in fp64 (tests/_logits_ref.py), on the GPU: sizes around the kernels' steps,
every type, rows that start anywhere, masks and lists that leave nothing, in place, on other streams and in graphs."""

import numpy as np
import pytest
import torch

from paper_2606_01813_amd import (KVCache, Plan, adjust_logits, distill, distill_grad, distill_workspace, verify_tree,
                                  verify_workspace)
from tests import _logits_ref as ref

pytestmark = pytest.mark.gpu

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32
INF = float("inf")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(gen, B, T, V, dtype, pad=0, shift=0, scale=3.0):
    """[B, T, V] logits in rows V + pad elements apart, the first `shift` elements off the allocation's start."""
    flat = torch.randn(B * T * (V + pad) + shift, generator=gen, device="cuda") * scale
    return flat.to(dtype)[shift:].view(B, T, V + pad)[..., :V]


def _tree(gen, B, cap, V, kids=2.5):
    """Parents in breadth-first order, and tokens that differ among the children of a row where V allows it."""
    i = torch.arange(cap)
    parent = torch.minimum((i / kids).to(torch.int64), i) - 1
    tok = torch.stack([torch.randperm(max(V, cap), generator=torch.Generator().manual_seed(7 + b))[:cap] % V for b in range(B)])
    return tok.to(I32).cuda(), parent.to(I32).expand(B, -1).contiguous().cuda()


def _words(ok):
    """bool [..., V] as int32 words"""
    V = ok.shape[-1]
    n = (V + 31) // 32
    ok = torch.nn.functional.pad(ok, (0, n * 32 - V)).unflatten(-1, (n, 32)).to(torch.int64)
    w = (ok << torch.arange(32, device=ok.device)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(I32)


def _close(got, want, tol, name):
    got = ref.f64(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want)))
    if bad.any():
        at = tuple(int(i) for i in np.argwhere(bad)[0]) if bad.ndim else ()
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} off, first at {at}: got {got[at]!r}, want {want[at]!r} +- {tol[at]!r}")


# ---------------------------------------------------------------- adjust_logits

def _adjust_inputs(gen, B, T, V, H, N, mask, tree):
    kw = {}
    if H:
        tok = (torch.rand((B, H), generator=gen, device="cuda") ** 3 * (V + 2)).to(I32) - 1           # -1 and V: padding
        kw.update(history=tok, history_len=torch.tensor([H, H // 2, 0, 1, -3, H + 9][:B] + [H] * (B - 6), dtype=I32, device="cuda"),
                  repetition=torch.rand(B, generator=gen, device="cuda") + 0.7, presence=torch.rand(B, generator=gen, device="cuda"),
                  frequency=torch.rand(B, generator=gen, device="cuda") - 0.2)
    if N:
        kw.update(bias_ids=torch.randint(-1, V + 1, (B, N), generator=gen, device="cuda", dtype=I32),
                  bias=torch.randn((B, N), generator=gen, device="cuda") * 5)
    if mask:
        ok = torch.rand((B, T, V), generator=gen, device="cuda") < {"half": 0.5, "few": 0.02, "most": 0.99}[mask]
        ok[0, 0] = False                                                                               # a row with nothing left
        kw["allowed"] = _words(ok)
    if tree:
        kw["token_ids"], kw["parent"] = _tree(gen, B, T - 1, V)
    return kw


def _check_adjust(x, got, before, kw, name):
    want, tol = ref.adjust(ref.f64(x), x.dtype, **kw)
    got, before = ref.f64(got), ref.f64(before)
    for b in range(x.shape[0]):
        for t in range(x.shape[1]):
            if kw.get("count") is not None and t >= min(max(int(kw["count"][b]), 0), x.shape[1] - ("parent" in kw)) + ("parent" in kw):
                assert np.array_equal(got[b, t], before[b, t], equal_nan=True), (name, "a row past count was written", b, t)
                continue
            with np.errstate(invalid="ignore"):
                bad = ~((np.abs(got[b, t] - want[b, t]) <= tol[b, t]) | (got[b, t] == want[b, t]) | (np.isnan(got[b, t]) & np.isnan(want[b, t])))
            assert not bad.any(), (name, b, t, np.flatnonzero(bad)[:5], got[b, t][bad][:5], want[b, t][bad][:5])


@pytest.mark.parametrize("V", [1, 3, 8, 31, 33, 511, 4097, 8191, 8192, 8193, 20003])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
def test_adjust_sizes(V, dtype):
    gen = _gen(V)
    for T, H, N, mask, tree, pad, shift in [(1, 9, 0, "", False, 0, 0), (2, 40, 7, "half", False, 1, 1), (5, 0, 3, "most", True, 3, 2),
                                            (3, 300, 0, "few", True, 8, 0), (2, 0, 0, "", False, 5, 3)]:
        B = 3
        kw = _adjust_inputs(gen, B, T, V, H, N, mask, tree)
        x = _rows(gen, B, T, V, dtype, pad, shift)
        out = adjust_logits(x, **kw)
        torch.cuda.synchronize()
        _check_adjust(x, out, torch.zeros_like(out), kw, ("out of place", T, H, N, mask, tree))
        y = x.clone(memory_format=torch.contiguous_format) if pad == 0 else _rows(_gen(1), B, T, V, dtype, pad, shift).copy_(x)
        assert adjust_logits(y, y, **kw) is y
        _check_adjust(x, y, x, kw, ("in place", T, H, N, mask, tree))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_adjust_rows_past_count(tree, in_place):
    gen = _gen(5)
    B, T, V = 6, 37, 9001
    kw = _adjust_inputs(gen, B, T, V, 50, 20, "half", tree)
    kw["count"] = torch.tensor([0, 1, 16, 36, 90, -4], dtype=I32, device="cuda")
    x = _rows(gen, B, T, V, BF, pad=7)
    out = x.clone() if in_place else torch.full_like(x, 77.0)
    src = out if in_place else x
    before = out.clone()
    adjust_logits(src, out, **kw)
    _check_adjust(x, out, before, kw, "count")


@pytest.mark.parametrize("V", [5, 256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tree", [False, True])
def test_adjust_many_rows_of_a_short_vocabulary(V, dtype, tree):
    gen = _gen(V + 7)
    B, T = 5, 37
    kw = _adjust_inputs(gen, B, T, V, 90, 9, "most", tree)
    kw["count"] = torch.tensor([36, 17, 0, 100, 31], dtype=I32, device="cuda")
    x = _rows(gen, B, T, V, dtype, pad=1, shift=1)
    out = torch.full_like(x, 77.0)
    adjust_logits(x, out, **kw)
    _check_adjust(x, out, torch.full_like(x, 77.0), kw, "out of place")
    y = _rows(gen, B, T, V, dtype, pad=1, shift=1).copy_(x)
    adjust_logits(y, y, **kw)
    _check_adjust(x, y, x, kw, "in place")


def test_adjust_pad_between_rows_stays():
    gen = _gen(6)
    full = torch.randn((2, 3, 1030), generator=gen, device="cuda").to(BF)
    dst = torch.full((2, 3, 1030), 5.0, dtype=BF, device="cuda")
    ok = _words(torch.zeros((2, 3, 1003), dtype=torch.bool, device="cuda"))
    adjust_logits(full[..., 11:1014], dst[..., 11:1014], allowed=ok)
    assert bool((dst[..., 11:1014] == -INF).all()) and bool((dst[..., :11] == 5).all()) and bool((dst[..., 1014:] == 5).all())
    adjust_logits(full[..., 11:1014], full[..., 11:1014], allowed=ok)
    assert bool((full[..., 11:1014] == -INF).all()) and bool((full[..., :11] > -INF).all()) and bool((full[..., 1014:] > -INF).all())


@pytest.mark.parametrize("in_place", [False, True])
def test_adjust_special_values(in_place):
    """Infinities, NaN and the lowest value pass through; a masked place is -inf whatever it held."""
    V = 300
    special = torch.tensor([INF, -INF, float("nan"), torch.finfo(F32).min, torch.finfo(F32).max, 0.0, -0.0], device="cuda")
    x = special.repeat(V // 7 + 1)[:V].view(1, 1, V).contiguous()
    ok = torch.ones((1, 1, V), dtype=torch.bool, device="cuda")
    ok[..., 100:200] = False
    hist = torch.arange(0, 50, dtype=I32, device="cuda").view(1, -1)
    kw = dict(history=hist, repetition=torch.tensor([2.0], device="cuda"), allowed=_words(ok),
              bias_ids=torch.tensor([[60, 61, 62]], dtype=I32, device="cuda"), bias=torch.tensor([[-INF, 1.0, INF]], device="cuda"))
    y = x.clone()
    out = adjust_logits(y, y if in_place else None, **kw)
    want, tol = ref.adjust(ref.f64(x), F32, **kw)
    with np.errstate(invalid="ignore", over="ignore"):
        want = want.astype(np.float32).astype(np.float64)
    _close(out, want, tol, "special")


def test_adjust_counts_past_16_bits_and_many_biases():
    """A token that makes up a long history; every place of the largest list of biases, each token listed twice."""
    V, H = 5000, 200000
    hist = torch.full((1, H), 17, dtype=I32, device="cuda")
    hist[0, ::3] = 4999
    ids = (torch.arange(4095, device="cuda") % 2047).to(I32).view(1, -1)
    kw = dict(history=hist, frequency=torch.tensor([2.0 ** -10], device="cuda"), bias_ids=ids,
              bias=torch.randn((1, 4095), generator=_gen(3), device="cuda"))
    x = _rows(_gen(4), 1, 2, V, F32)
    _check_adjust(x, adjust_logits(x, **kw), x, kw, "long")
    y = x.clone()
    _check_adjust(x, adjust_logits(y, y, **kw), x, kw, "long, in place")


def test_adjust_paths():
    """A chain of 40 nodes of few tokens (the last 32 of a path count), a parent that is not below its node, tokens
    outside the vocabulary, a history that shares tokens with the path."""
    V, cap = 9000, 40
    par = torch.arange(-1, cap - 1, dtype=I32, device="cuda").view(1, -1).repeat(2, 1)
    par[1, 20] = 20
    par[1, 30] = 39
    tok = torch.tensor([3, 8999, 3, -1, 9000, 8191, 8192] * 6, dtype=I32, device="cuda")[:cap].view(1, -1).repeat(2, 1)
    hist = torch.tensor([[3, 5, 8192], [8999, 8999, 4]], dtype=I32, device="cuda")
    kw = dict(history=hist, repetition=torch.tensor([1.5, 0.5], device="cuda"), presence=torch.tensor([0.25, -1.0], device="cuda"),
              frequency=torch.tensor([0.5, 0.125], device="cuda"), token_ids=tok, parent=par,
              bias_ids=torch.tensor([[3, 8191], [8192, 8999]], dtype=I32, device="cuda"), bias=torch.tensor([[1.0, 2.0], [3.0, 4.0]], device="cuda"))
    x = _rows(_gen(8), 2, cap + 1, V, F16)
    _check_adjust(x, adjust_logits(x, **kw), x, kw, "path")
    y = x.clone()
    _check_adjust(x, adjust_logits(y, y, **kw), x, kw, "path, in place")


def test_adjust_the_largest_tree():
    """4096 nodes, more than are kept near, with paths that go through all parts of the tree."""
    V, cap = 300, 4096
    i = torch.arange(cap)
    par = torch.maximum(i - 170, torch.tensor(-1)).to(I32).view(1, -1).cuda()
    tok = torch.randint(V, (1, cap), generator=_gen(12), device="cuda", dtype=I32)
    kw = dict(repetition=torch.tensor([1.2], device="cuda"), frequency=torch.tensor([0.25], device="cuda"), token_ids=tok, parent=par,
              count=torch.tensor([4090], dtype=I32, device="cuda"))
    x = _rows(_gen(13), 1, cap + 1, V, BF)
    out = torch.full_like(x, 3.0)
    _check_adjust(x, adjust_logits(x, out, **kw), torch.full_like(x, 3.0), kw, "largest tree")
    y = x.clone()
    _check_adjust(x, adjust_logits(y, y, **kw), x, kw, "largest tree, in place")


@pytest.mark.parametrize("H", [3, 4, 2047, 2048, 2049, 4096, 6145])
def test_adjust_history_lengths(H):
    """Around what the workgroup takes at a time; every token from the same few."""
    V = 9000
    hist = (torch.arange(3 * H, device="cuda") * 7919 % 12 * 800).to(I32).view(3, H)
    kw = dict(history=hist, history_len=torch.tensor([H, H - 1, H - 3], dtype=I32, device="cuda"),
              frequency=torch.tensor([2.0 ** -6, 2.0 ** -5, 1.0], device="cuda"))
    x = _rows(_gen(14), 3, 3, V, F32)
    _check_adjust(x, adjust_logits(x, **kw), x, kw, "history")
    y = x.clone()
    _check_adjust(x, adjust_logits(y, y, **kw), x, kw, "history, in place")


def test_adjust_shared_masks_and_repeated_logits():
    """One mask for all rows (strides of 0), and rows of logits that are one row."""
    gen = _gen(9)
    B, T, V = 3, 4, 777
    x = _rows(gen, 1, 1, V, BF).expand(B, T, V)
    ok = torch.rand((1, 1, V), generator=gen, device="cuda") < 0.5
    words = _words(ok).expand(B, T, -1)
    out = adjust_logits(x, allowed=words)
    assert torch.equal(out, torch.where(ok.expand(B, T, V), x, torch.tensor(-INF, dtype=BF, device="cuda")))
    words = _words(torch.rand((B, 1, V), generator=gen, device="cuda") < 0.5).expand(-1, T, -1)
    _check_adjust(x, adjust_logits(x, allowed=words), x, dict(allowed=words), "by sequence")


@pytest.mark.parametrize("dtype", [BF, F16, F32])
def test_adjust_fill(dtype):
    """What a token that is not allowed gets: any value, rounded to the logits' type."""
    V = 700
    x = _rows(_gen(10), 2, 2, V, dtype)
    ok = torch.rand((2, 2, V), generator=_gen(11), device="cuda") < 0.5
    for fill in (-65504.0, -3.14159, 5.0, -0.0, 0.0):
        want = torch.where(ok, x, torch.tensor(fill if fill else -INF, device="cuda").to(dtype))     # (0: the default)
        assert torch.equal(adjust_logits(x, allowed=_words(ok), fill=fill), want)
        y = x.clone()
        assert torch.equal(adjust_logits(y, y, allowed=_words(ok), fill=fill), want)


# ---------------------------------------------------------------- verify_tree

def _outputs(B, T, M):
    z = lambda *s: torch.full(s, 99, dtype=I32, device="cuda")
    return z(B), z(B, M), z(B, M), torch.full((B, T), 99.0, device="cuda")


def _check_verify(got, want):
    for g, w, name in zip(got, want, ("accepted", "index", "tokens", "weight")):
        assert np.array_equal(g.cpu().numpy(), w), (name, g, w)


def _agree(x, tok, par, count, depth, high=60.0):
    """Makes the rows of a path of `depth[b]` nodes choose its tokens."""
    for b in range(x.shape[0]):
        n, row = min(max(int(count[b]), 0), x.shape[1] - 1), 0
        for _ in range(depth[b]):
            kids = [i for i in range(n) if int(par[b, i]) == row - 1]
            if not kids:
                break
            node = kids[(b + row) % len(kids)]
            x[b, row, int(tok[b, node])] = high
            row = node + 1


@pytest.mark.parametrize("V", [1, 5, 8, 64, 1023, 8192, 8200, 40009])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("with_workspace", [False, True])
def test_verify_sizes(V, dtype, with_workspace):
    gen = _gen(V)
    for B, cap, M, pad, shift in [(1, 1, 1, 0, 0), (4, 7, 3, 1, 1), (7, 40, 17, 3, 2), (2, 0, 4, 0, 1)]:
        x = _rows(gen, B, cap + 1, V, dtype, pad, shift)
        tok, par = _tree(gen, B, cap, V) if cap else (torch.zeros((B, 0), dtype=I32, device="cuda"),) * 2
        count = torch.tensor([cap, 0, cap // 2, 1, cap + 5, -2, cap][:B], dtype=I32, device="cuda")
        _agree(x, tok, par, count, [9, 2, 0, 1, 3, 5, 2][:B])
        acc, index, tokens, weight = _outputs(B, cap + 1, M)
        ws = verify_workspace(x) if with_workspace else None
        verify_tree(x, tok, par, count, acc, index, tokens, weight=weight, workspace=ws)
        want = ref.verify(tok.cpu().numpy(), par.cpu().numpy(), count.cpu().numpy(), M, logits=ref.f64(x))
        _check_verify((acc, index, tokens, weight), want)


@pytest.mark.parametrize("with_workspace", [False, True])
def test_verify_ties_and_special_values(with_workspace):
    """Equal logits go to the lowest id, wherever they stand; +inf wins, NaN and -inf are never chosen."""
    V, cap, B = 20000, 3, 8
    x = torch.full((B, cap + 1, V), -1.0, device="cuda")
    x[0, 0, [5, 4099, 19999]] = 3.0
    x[1, 0, [19999, 8191]] = 3.0
    x[2, 0, 77], x[2, 0, 78], x[2, 0, 79] = float("nan"), INF, float("nan")
    x[3, 0] = -INF
    x[4, 0] = float("nan")
    x[5, 0] = -INF
    x[5, 0, 12345] = torch.finfo(F32).min
    x[6, 0] = 0.0
    x[6, 0, 3] = -0.0                                                      # (equal to 0: the lowest id is 0)
    x[7, 0] = float("nan")
    x[7, 0, 4] = -INF
    tok = torch.tensor([[5, 8191, 78]] * B, dtype=I32, device="cuda")
    tok[6] = torch.tensor([0, 0, 0])                                       # twice among the children: the first node
    par = torch.full((B, cap), -1, dtype=I32, device="cuda")
    count = torch.full((B,), cap, dtype=I32, device="cuda")
    got = _outputs(B, cap + 1, 3)
    verify_tree(x, tok, par, count, *got[:3], weight=got[3], workspace=verify_workspace(x) if with_workspace else None)
    assert got[2][:, 0].tolist() == [5, 8191, 78, -1, -1, 12345, 0, -1]
    assert got[0].tolist() == [2, 2, 2, 1, 1, 1, 2, 1] and got[1][6].tolist() == [0, 1, -1]
    _check_verify(got, ref.verify(tok.cpu().numpy(), par.cpu().numpy(), count.cpu().numpy(), 3, logits=ref.f64(x)))


def test_verify_reads_only_its_path():
    """Rows off the path may hold anything; nodes past count carry no path, whatever their parents say."""
    B, cap, V = 2, 12, 5000
    gen = _gen(2)
    x = torch.full((B, cap + 1, V), float("nan"), device="cuda")
    tok, par = _tree(gen, B, cap, V)
    par[:, 9:] = -1
    count = torch.tensor([9, 9], dtype=I32, device="cuda")
    x[:, 0] = 0.0
    x[0, 0, int(tok[0, 1])] = 2.0
    x[0, 2] = 1.0
    x[1, 0, int(tok[1, 10])] = 2.0                                         # a node past count
    got = _outputs(B, cap + 1, 5)
    verify_tree(x, tok, par, count, *got[:3], weight=got[3])
    assert got[0].tolist() == [2, 1] and got[1][0, :2].tolist() == [0, 2]
    _check_verify(got, ref.verify(tok.cpu().numpy(), par.cpu().numpy(), count.cpu().numpy(), 5, logits=ref.f64(x)))


@pytest.mark.parametrize("with_workspace", [False, True])
@pytest.mark.parametrize("V", [64, 4200])
def test_verify_the_largest_tree(V, with_workspace):
    """A path to the last of 4096 nodes, most of them further than those kept near (of few tokens: siblings share them, and
    the first of them ends the path early)."""
    cap = 4096
    i = torch.arange(cap)
    par = torch.maximum(i - 500, torch.tensor(-1)).to(I32).view(1, -1).cuda()
    tok = (i * 31 % V).to(I32).view(1, -1).cuda()
    x = torch.randn((1, cap + 1, V), generator=_gen(4), device="cuda")
    row, path = cap, []
    while row > 0:
        path.append(row)
        row = int(par[0, row - 1]) + 1
    for r, after in zip([0] + path[::-1], path[::-1]):
        x[0, r, int(tok[0, after - 1])] = 50.0
    count = torch.tensor([cap], dtype=I32, device="cuda")
    got = _outputs(1, cap + 1, 12)
    verify_tree(x, tok, par, count, *got[:3], weight=got[3], workspace=verify_workspace(x) if with_workspace else None)
    _check_verify(got, ref.verify(tok.cpu().numpy(), par.cpu().numpy(), count.cpu().numpy(), 12, logits=ref.f64(x)))
    assert V < cap or got[1][0, :len(path) + 1].tolist() == [0] + path[::-1]


@pytest.mark.parametrize("V", [4099, 40011, 151936])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("with_workspace", [False, True])
def test_verify_ties_anywhere(V, dtype, with_workspace):
    """Of equals the lowest id, whichever lanes, vectors and parts of the row they stand in; -0 and 0 are equals."""
    gen = _gen(V)
    B = 40
    x = torch.full((B, 1, V), -5.0, dtype=dtype, device="cuda")
    first = []
    for b in range(B):
        n = [1, 2, 3, 50][b % 4]
        at = torch.randint(V * (b % 3) // 3, V, (n,), generator=gen, device="cuda")
        x[b, 0, at] = [2.5, 0.0, -0.0][b % 3]
        if b % 5 == 0:
            x[b, 0, at[0]] = -0.0 if b % 3 else 2.5
        if b % 7 == 3:
            at = torch.tensor([V - 1], device="cuda")                      # alone, past the last whole vector
            x[b, 0] = float("nan")
            x[b, 0, V - 1] = -7.0
        first.append(int(at.min()))
    none = torch.zeros((B, 0), dtype=I32, device="cuda")
    got = _outputs(B, 1, 1)
    verify_tree(x, none, none, torch.zeros(B, dtype=I32, device="cuda"), *got[:3], weight=got[3],
                workspace=verify_workspace(x) if with_workspace else None)
    assert got[2][:, 0].tolist() == first


def test_verify_chosen_tokens_of_the_largest_tree():
    cap = 4096
    i = torch.arange(cap)
    par = torch.maximum(i - 500, torch.tensor(-1)).to(I32).view(1, -1).cuda()
    tok = i.to(I32).view(1, -1).cuda()
    chosen = torch.full((1, cap + 1), -1, dtype=I32, device="cuda")
    row, path = cap, [cap]
    while row > 0:
        row, after = int(par[0, row - 1]) + 1, row
        chosen[0, row] = after - 1
        path.append(row)
    got = _outputs(1, cap + 1, 12)
    verify_tree(None, tok, par, torch.tensor([cap], dtype=I32, device="cuda"), *got[:3], chosen=chosen, weight=got[3])
    path = path[::-1]
    assert got[0].tolist() == [len(path)] and got[1][0, :len(path)].tolist() == path
    assert got[3].nonzero()[:, 1].tolist() == path


def test_verify_chosen_tokens():
    B, cap, V = 5, 100, 6
    gen = _gen(3)
    tok, par = _tree(gen, B, cap, V)
    chosen = torch.randint(-1, V, (B, cap + 1), generator=gen, device="cuda", dtype=I32)
    count = torch.tensor([100, 50, 0, 3, 99], dtype=I32, device="cuda")
    for M in (1, 2, 40):
        got = _outputs(B, cap + 1, M)
        verify_tree(None, tok, par, count, *got[:3], chosen=chosen, weight=got[3])
        _check_verify(got, ref.verify(tok.cpu().numpy(), par.cpu().numpy(), count.cpu().numpy(), M, chosen=chosen.cpu().numpy()))


def test_verify_a_chain_as_long_as_its_path():
    """Every node accepted, down to M rows; without the optional weight."""
    cap, V = 32, 4096
    par = torch.arange(-1, cap - 1, dtype=I32, device="cuda").view(1, -1)
    tok = torch.arange(10, 10 + cap, dtype=I32, device="cuda").view(1, -1)
    x = torch.zeros((1, cap + 1, V), dtype=BF, device="cuda")
    for i in range(cap):
        x[0, i, 10 + i] = 1.0
    count = torch.tensor([cap], dtype=I32, device="cuda")
    for M in (33, 40, 7):
        acc, index, tokens, _ = _outputs(1, cap + 1, M)
        verify_tree(x, tok, par, count, acc, index, tokens)
        n = min(M, 33)
        assert acc.tolist() == [n] and index[0].tolist() == list(range(n)) + [-1] * (M - n)
        assert tokens[0, :n].tolist() == [10 + i if i < cap else 0 for i in range(n)]


# ---------------------------------------------------------------- distill, distill_grad

def _teacher(gen, B, T, V, K, tail, junk=True):
    ids = torch.stack([torch.randperm(max(V, K), generator=gen, device="cuda")[:K] for _ in range(B * T)]).view(B, T, K)
    ids = torch.where(ids < V, ids, -1).to(I32)
    target = torch.randn((B, T, K), generator=gen, device="cuda") * 2
    if tail:
        target = torch.log_softmax(torch.cat((target, torch.randn((B, T, 1), generator=gen, device="cuda")), -1), -1)[..., :K].contiguous()
    if junk and K > 2:
        ids[0, 0, 1] = V + 3
        target[0, 0, 1] = float("nan")                                     # (padding: not read into anything)
        ids[0, -1, 2] = ids[0, -1, 0]                                      # a token listed twice
        target[-1, 0, 0] = -INF
    return ids, target


def _check_distill(x, ids, target, weight, tau, tail, loss=None, stats=None, grad=None, again=False):
    l, t, i = ref.f64(x), ref.f64(target), ids.cpu().numpy()
    w = np.ones(ids.shape[:2]) if weight is None else ref.f64(weight)
    for b in range(x.shape[0]):
        for r in range(x.shape[1]):
            want = ref.distill(l[b, r], i[b, r], t[b, r], w[b, r], tau, tail, x.dtype, again)
            at = (b, r, x.shape, x.dtype, tau, tail)
            if loss is not None:
                _close(loss[b, r], np.array(want[0]), np.array(want[3]), ("loss", at))
            if stats is not None:
                _close(stats[b, r], want[1], want[4], ("stats", at))
            if grad is not None:
                _close(grad[b, r], want[2], want[5], ("grad", at))


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 500, 4096, 4099, 16389, 70001])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("with_workspace", [False, True])
def test_distill_sizes(V, dtype, with_workspace):
    gen = _gen(V)
    for B, T, K, tail, tau, pad, shift in [(1, 1, 1, False, 1.0, 0, 0), (2, 3, 8, True, 1.0, 1, 1), (3, 2, 16, False, 2.5, 8, 0),
                                           (1, 2, 256, True, 1.0, 3, 3), (1, 2, 100, False, 0.5, 0, 2)]:
        x = _rows(gen, B, T, V, dtype, pad, shift)
        ids, target = _teacher(gen, B, T, V, K, tail)
        w = torch.randn((B, T), generator=gen, device="cuda")
        w[-1, -1] = 0.0 if B * T > 1 else -1.5
        loss, stats = torch.full((B, T), 9.0, device="cuda"), torch.full((B, T, 3), 9.0, device="cuda")
        room = torch.full((B, T, V + pad), 9.0, dtype=dtype, device="cuda")
        grad = room[..., :V]
        ws = distill_workspace(x) if with_workspace else None
        distill(x, ids, target, loss, grad=grad, stats=stats, weight=w, temperature=tau, tail=tail, workspace=ws)
        _check_distill(x, ids, target, w, tau, tail, loss, stats, grad)
        assert bool((room[..., V:] == 9).all())
        alone = torch.full((B, T), 9.0, device="cuda")
        distill(x, ids, target, alone, weight=w, temperature=tau, tail=tail, workspace=ws)
        _check_distill(x, ids, target, w, tau, tail, alone)
        g = distill_grad(x, ids, target, stats, weight=w, temperature=tau, tail=tail)
        _check_distill(x, ids, target, w, tau, tail, grad=g, again=True)
        y = x.clone()                                                      # the gradient over the logits
        distill(y, ids, target, alone, grad=y, weight=w, temperature=tau, tail=tail, workspace=ws)
        assert torch.equal(y, grad) and torch.equal(alone, loss)
        y = x.clone()
        assert torch.equal(distill_grad(y, ids, target, stats, y, weight=w, temperature=tau, tail=tail), g)


@pytest.mark.parametrize("vectors", [64, 128, 256, 512, 1024, 2048, 4096, 32768])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("more", [0, 1, 9])
def test_distill_rows_around_the_launches_limits(vectors, dtype, more):
    """Rows of just so many vectors of 16 bytes, and of a few elements more."""
    gen = _gen(vectors + more)
    V = vectors * (16 // dtype.itemsize) + more
    B, T, K, tau = (1, 2, 5, 0.7) if vectors > 4096 else (2, 3, 5, 0.7)
    used = float(np.float32(tau))                                          # (a call's temperature is a float: 0.7 (1 - 1.7e-8))
    x = _rows(gen, B, T, V, dtype, 1, 1)
    ids, target = _teacher(gen, B, T, V, K, False)
    ids[0, 0, 0] = V - 1
    loss, stats = torch.full((B, T), 9.0, device="cuda"), torch.full((B, T, 3), 9.0, device="cuda")
    grad = torch.full_like(x, 9.0)
    distill(x, ids, target, loss, grad=grad, stats=stats, temperature=tau)
    _check_distill(x, ids, target, None, used, False, loss, stats, grad)
    alone = torch.full((B, T), 9.0, device="cuda")
    distill(x, ids, target, alone, temperature=tau)
    _check_distill(x, ids, target, None, used, False, alone)
    _check_distill(x, ids, target, None, used, False, grad=distill_grad(x, ids, target, stats, temperature=tau), again=True)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_against_differences(tail):
    """The gradient against differences of the definition in fp64 and, in fp32, of the library's own loss."""
    gen = _gen(11)
    V, K, tau, h = 40, 6, 1.7, 1e-5
    x = _rows(gen, 1, 1, V, F32)
    ids, target = _teacher(gen, 1, 1, V, K, tail, junk=False)
    loss, grad = torch.zeros((1, 1), device="cuda"), torch.zeros_like(x)
    distill(x, ids, target, loss, grad=grad, temperature=tau, tail=tail)
    l, i, t = ref.f64(x)[0, 0], ids[0, 0].cpu().numpy(), ref.f64(target)[0, 0]
    of = lambda l: ref.distill(l, i, t, 1.0, tau, tail, F32)[0]
    for v in range(V):
        e = np.zeros(V)
        e[v] = h
        slope = (of(l + e) - of(l - e)) / (2 * h)
        # the second-order rest is h^2 / 6 of a third derivative below 1 / tau^3, the subtraction's rounding 2^-52 loss / h
        assert abs(float(grad[0, 0, v]) - slope) < 1e-9 + 3e-6 * abs(slope) + 3e-7
    step = 2.0 ** -6
    for v in (0, int(ids[0, 0, 0]), V - 1):
        moved = [torch.zeros((1, 1), device="cuda") for _ in range(2)]
        for s, out in zip((1, -1), moved):
            y = x.clone()
            y[0, 0, v] += s * step
            distill(y, ids, target, out, temperature=tau, tail=tail)
        slope = (float(moved[0]) - float(moved[1])) / (2 * step)
        # a loss below 16 is off by some 2^-21, over 2^-5; the third derivative (below 1 / tau^3) times step^2 / 6
        assert abs(float(grad[0, 0, v]) - slope) < 2 * 2.0 ** -21 / (2 * step) + step ** 2 / 6 + 1e-5


def test_distill_sharp_rows():
    """The rest's mass is the student's own sum over what is not listed, also where that is 1e-9 of all."""
    V, K = 5000, 4
    x = torch.full((1, 1, V), -30.0, device="cuda")
    ids = torch.tensor([[[7, 4096, 4999, 100]]], dtype=I32, device="cuda")
    x[0, 0, ids[0, 0].long()] = torch.tensor([0.0, -1.0, -2.0, -3.0], device="cuda")
    target = torch.log(torch.tensor([[[0.5, 0.2, 0.1, 0.1]]], device="cuda"))
    loss, stats, grad = torch.zeros((1, 1), device="cuda"), torch.zeros((1, 1, 3), device="cuda"), torch.zeros_like(x)
    distill(x, ids, target, loss, grad=grad, stats=stats, tail=True)
    _check_distill(x, ids, target, None, 1.0, True, loss, stats, grad)
    assert float(stats[0, 0, 2]) < 1e-8


@pytest.mark.parametrize("with_workspace", [False, True])
def test_distill_masks_and_special_values(with_workspace):
    V, K, B = 9000, 4, 10
    gen = _gen(12)
    x = _rows(gen, B, 1, V, F32)
    ids, target = _teacher(gen, B, 1, V, K, False, junk=False)
    low = torch.finfo(F32).min
    free = (set(range(V)) - set(ids.flatten().tolist())).pop()
    x[0, 0, free] = -INF                                                   # a masked token
    x[1, 0, int(ids[1, 0, 0])] = -INF                                      # ... that the teacher lists: an infinite loss
    x[2] = -INF                                                            # a row of nothing else
    x[3] = low                                                             # the type's lowest value as a mask, everywhere
    x[4, 0, :V // 2] = low
    x[5, 0, free] = float("nan")
    x[6, 0, free] = INF
    target[7] = -INF                                                       # a teacher that lists nothing
    ids[8] = -1
    x[9] = 3.0e38                                                          # differences of 0, products that would overflow
    loss, stats, grad = torch.zeros((B, 1), device="cuda"), torch.zeros((B, 1, 3), device="cuda"), torch.zeros_like(x)
    ws = distill_workspace(x) if with_workspace else None
    for tail in (False, True):
        distill(x, ids, target, loss, grad=grad, stats=stats, tail=tail, temperature=0.5, workspace=ws)
        g2 = distill_grad(x, ids, target, stats, tail=tail, temperature=0.5)
        fine = [0, 3, 4, 7, 8, 9]
        pick = lambda t: t[fine].contiguous()
        _check_distill(pick(x), pick(ids), pick(target), None, 0.5, tail, pick(loss), pick(stats), pick(grad))
        _check_distill(pick(x), pick(ids), pick(target), None, 0.5, tail, grad=pick(g2), again=True)
        assert float(loss[1]) == INF and bool(torch.isfinite(grad[1]).all()) and bool(torch.isfinite(g2[1]).all())
        assert float(loss[2]) == INF and stats[2, 0].tolist() == [-INF, 0.0, 0.0]
        for g in (grad, g2):
            on = torch.zeros(V, dtype=torch.bool, device="cuda").index_fill_(0, ids[2, 0].long(), True)
            assert bool((g[2, 0][~on] == 0).all()) and bool((g[2, 0][on] < 0).all())
        for r in (5, 6):
            assert bool(torch.isnan(loss[r]).all()) and bool(torch.isnan(grad[r]).all()) and bool(torch.isnan(g2[r]).all()), r
        if not tail:
            assert float(loss[7]) == 0 and float(loss[8]) == 0 and bool((grad[7:9] == 0).all())


@pytest.mark.parametrize("with_workspace", [False, True])
def test_distill_rows_of_no_weight_are_not_read(with_workspace):
    B, T, V, K = 2, 5, 3001, 8
    gen = _gen(13)
    x = _rows(gen, B, T, V, BF)
    ids, target = _teacher(gen, B, T, V, K, False)
    w = torch.ones((B, T), device="cuda")
    w[0, 1], w[1, 4] = 0.0, -0.0
    x[0, 1], x[1, 4], target[1, 4] = float("nan"), INF, float("nan")
    loss, stats, grad = torch.ones((B, T), device="cuda"), torch.ones((B, T, 3), device="cuda"), torch.ones_like(x)
    distill(x, ids, target, loss, grad=grad, stats=stats, weight=w, workspace=distill_workspace(x) if with_workspace else None)
    _check_distill(x, ids, target, w, 1.0, False, loss, stats, grad)
    assert float(loss[0, 1]) == 0 and bool((grad[1, 4] == 0).all())
    assert bool((distill_grad(x, ids, target, stats, weight=w)[0, 1] == 0).all())


def test_distill_large_vocabulary():
    V = 1 << 20
    x = _rows(_gen(14), 1, 2, V, BF)
    ids, target = _teacher(_gen(15), 1, 2, V, 8, True)
    loss, stats, grad = torch.zeros((1, 2), device="cuda"), torch.zeros((1, 2, 3), device="cuda"), torch.zeros_like(x)
    distill(x, ids, target, loss, grad=grad, stats=stats, tail=True)
    _check_distill(x, ids, target, None, 1.0, True, loss, stats, grad)
    _check_distill(x, ids, target, None, 1.0, True, grad=distill_grad(x, ids, target, stats, tail=True), again=True)


# ---------------------------------------------------------------- all of them

def test_offsets_past_32_bits():
    """Rows that lie further apart than 2^32 elements."""
    V, apart = 1000, (1 << 32) + 24
    room = torch.zeros(apart + V, dtype=BF, device="cuda")
    x = room.as_strided((2, 1, V), (apart, apart, 1))
    x.copy_(_rows(_gen(16), 2, 1, V, BF))
    ids, target = _teacher(_gen(17), 2, 1, V, 8, False)
    loss, grad = torch.zeros((2, 1), device="cuda"), torch.zeros((2, 1, V), dtype=BF, device="cuda")
    distill(x, ids, target, loss, grad=grad)
    _check_distill(x, ids, target, None, 1.0, False, loss, None, grad)
    kw = dict(history=torch.randint(V, (2, 30), generator=_gen(18), device="cuda", dtype=I32), repetition=torch.tensor([2.0, 3.0], device="cuda"))
    before = x.clone()
    _check_adjust(before, adjust_logits(x, **kw), before, kw, "far")
    _check_adjust(before, adjust_logits(x, x, **kw), before, kw, "far, in place")
    got = _outputs(2, 1, 2)
    none = torch.zeros((2, 0), dtype=I32, device="cuda")
    verify_tree(x, none, none, torch.zeros(2, dtype=I32, device="cuda"), *got[:3], weight=got[3])
    assert got[2][:, 0].tolist() == x[:, 0].float().argmax(-1).tolist()


def test_more_rows_than_a_grid_has_places_in_its_second_dimension():
    T, V = 70001, 9
    x = _rows(_gen(19), 1, T, V, BF)
    ok = torch.rand((1, T, V), generator=_gen(20), device="cuda") < 0.5
    want = torch.where(ok, x, torch.tensor(-INF, dtype=BF, device="cuda"))
    assert torch.equal(adjust_logits(x, allowed=_words(ok)), want)
    y = x.clone()
    assert torch.equal(adjust_logits(y, y, allowed=_words(ok)), want)
    ids, target = torch.zeros((1, T, 1), dtype=I32, device="cuda"), torch.zeros((1, T, 1), device="cuda")
    loss, stats, grad = torch.zeros((1, T), device="cuda"), torch.zeros((1, T, 3), device="cuda"), torch.zeros_like(x)
    distill(x, ids, target, loss, grad=grad, stats=stats)
    cut = lambda t: t[:, -3:].contiguous()
    _check_distill(cut(x), cut(ids), cut(target), None, 1.0, False, cut(loss), cut(stats), cut(grad))
    _check_distill(cut(x), cut(ids), cut(target), None, 1.0, False, grad=cut(distill_grad(x, ids, target, stats)), again=True)


def test_more_sequences_than_a_grid_has_places_in_its_second_dimension():
    B, V = 70001, 9
    x = _rows(_gen(19), B, 1, V, BF)
    ok = torch.rand((B, 1, V), generator=_gen(20), device="cuda") < 0.5
    want = torch.where(ok, x, torch.tensor(-INF, dtype=BF, device="cuda"))
    assert torch.equal(adjust_logits(x, allowed=_words(ok)), want)
    y = x.clone()
    assert torch.equal(adjust_logits(y, y, allowed=_words(ok)), want)
    y[:, 0, 4] = 70.0
    tok, par = torch.full((B, 0), 4, dtype=I32, device="cuda"), torch.full((B, 0), -1, dtype=I32, device="cuda")
    acc, index, tokens, weight = _outputs(B, 1, 2)
    verify_tree(y, tok, par, torch.zeros(B, dtype=I32, device="cuda"), acc, index, tokens, weight=weight)
    assert bool((acc == 1).all()) and bool((tokens == torch.tensor([4, -1], device="cuda")).all())
    ids, target = torch.zeros((B, 1, 1), dtype=I32, device="cuda"), torch.zeros((B, 1, 1), device="cuda")
    loss, stats, grad = torch.zeros((B, 1), device="cuda"), torch.zeros((B, 1, 3), device="cuda"), torch.zeros_like(x)
    distill(x, ids, target, loss, grad=grad, stats=stats)
    again = distill_grad(x, ids, target, stats)
    alone = torch.zeros((B, 1), device="cuda")
    distill(x, ids, target, alone)
    for cut in (lambda t: t[:2], lambda t: t[32767:32770], lambda t: t[-3:]):
        _check_distill(cut(x), cut(ids), cut(target), None, 1.0, False, cut(loss), cut(stats), cut(grad))
        _check_distill(cut(x), cut(ids), cut(target), None, 1.0, False, cut(alone))
        _check_distill(cut(x), cut(ids), cut(target), None, 1.0, False, grad=cut(again), again=True)


def test_empty_calls():
    z = lambda *s, t=F32: torch.zeros(s, dtype=t, device="cuda")
    assert adjust_logits(z(0, 3, 8)).shape == (0, 3, 8) and adjust_logits(z(2, 0, 8)).shape == (2, 0, 8)
    verify_tree(z(0, 3, 8), z(0, 2, t=I32), z(0, 2, t=I32), z(0, t=I32), z(0, t=I32), z(0, 4, t=I32), z(0, 4, t=I32))
    distill(z(0, 3, 8), z(0, 3, 2, t=I32), z(0, 3, 2), z(0, 3))
    assert distill_grad(z(2, 0, 8), z(2, 0, 2, t=I32), z(2, 0, 2), z(2, 0, 3)).shape == (2, 0, 8)
    x = z(2, 1, 8) + 1
    out = adjust_logits(x, history=z(2, 0, t=I32), repetition=z(2) + 2, bias_ids=z(2, 0, t=I32), bias=z(2, 0))
    assert torch.equal(out, x)


def _pipeline(state, stream=None):
    """Adjust, verify, distill and its separate gradient, once."""
    s = state
    adjust_logits(s["x"], s["adj"], **s["kw"], stream=stream)
    verify_tree(s["adj"], s["tok"], s["par"], s["kw"]["count"], s["acc"], s["index"], s["tokens"], weight=s["on"], workspace=s["vws"], stream=stream)
    distill(s["x"], s["ids"], s["target"], s["loss"], grad=s["grad"], stats=s["stats"], weight=s["on"], tail=True, workspace=s["dws"],
            stream=stream)
    distill_grad(s["x"], s["ids"], s["target"], s["stats"], s["grad2"], tail=True, stream=stream)
    return [s[n] for n in ("adj", "acc", "index", "tokens", "on", "loss", "grad", "stats", "grad2")]


def _pipeline_state(seed, B=3, T=18, V=33001, dtype=BF):
    gen = _gen(seed)
    tok, par = _tree(gen, B, T - 1, V)
    kw = _adjust_inputs(gen, B, T, V, 100, 12, "most", False)
    kw.update(token_ids=tok, parent=par, count=torch.tensor([T - 1, 5, 0][:B], dtype=I32, device="cuda"))
    x = _rows(gen, B, T, V, dtype, pad=3)
    _agree(x, tok, par, kw["count"], [3, 2, 1])
    ids, target = _teacher(gen, B, T, V, 8, True)
    acc, index, tokens, on = _outputs(B, T, 9)
    z = lambda *s: torch.zeros(s, device="cuda")
    return dict(x=x, adj=torch.zeros((B, T, V), dtype=dtype, device="cuda"), kw=kw, tok=tok, par=par, acc=acc, index=index, tokens=tokens, on=on,
                ids=ids, target=target, loss=z(B, T), stats=z(B, T, 3), grad=torch.zeros((B, T, V), dtype=dtype, device="cuda"),
                grad2=torch.zeros((B, T, V), dtype=dtype, device="cuda"), vws=verify_workspace(x), dws=distill_workspace(x))


def test_results_repeat_and_other_streams():
    state = _pipeline_state(21)
    want = [t.clone() for t in _pipeline(state)]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for stream in (None, other, None):
        for n in ("adj", "loss", "grad", "stats", "grad2"):
            state[n].zero_()
        other.wait_stream(torch.cuda.current_stream())
        got = _pipeline(state, stream)
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g.view(torch.uint8), w.view(torch.uint8))


def test_two_streams_at_once():
    states = [_pipeline_state(22), _pipeline_state(23)]
    want = [[t.clone() for t in _pipeline(s)] for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, st in zip(states, streams):
            _pipeline(s, st)
    torch.cuda.synchronize()
    for s, ws in zip(states, want):
        for g, w in zip([s[n] for n in ("adj", "acc", "index", "tokens", "on", "loss", "grad", "stats", "grad2")], ws):
            assert torch.equal(g.view(torch.uint8), w.view(torch.uint8))


def test_graph_replays_with_new_inputs():
    state, fresh = _pipeline_state(24), _pipeline_state(25)
    want = [t.clone() for t in _pipeline(fresh)]
    _pipeline(state)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = _pipeline(state)
    torch.cuda.synchronize()
    first = None
    for n in range(4):
        if n == 2:
            for name in ("x", "tok", "par", "ids", "target"):
                state[name].copy_(fresh[name])
            for name, t in state["kw"].items():
                t.copy_(fresh["kw"][name])
        graph.replay()
        torch.cuda.synchronize()
        _ = (state["x"].float().sum(), fresh["x"].exp())                   # the program's own work in between
        torch.cuda.synchronize()
        if n < 2:
            first = first or [t.clone() for t in outs]
            assert all(torch.equal(g.view(torch.uint8), w.view(torch.uint8)) for g, w in zip(outs, first))
        else:
            # (rows past count of the adjusted logits keep what the first inputs left there)
            live = torch.arange(18, device="cuda") <= fresh["kw"]["count"][:, None]
            assert torch.equal(outs[0][live].view(torch.uint8), want[0][live].view(torch.uint8))
            for g, w in zip(outs[1:], want[1:]):
                assert torch.equal(g.view(torch.uint8), w.view(torch.uint8))


def test_a_verified_round():
    """The calls as a program uses them: the drafter's logits adjusted, a tree built, the target's logits adjusted along its
    paths and verified, what was accepted written to the cache, and the drafter taught by the target's top tokens."""
    B, L, V, K, cap, heads, D = 4, 6, 8001, 8, 24, 2, 64
    gen = _gen(31)
    plan = Plan(L=L, V=V, K=K, cap=cap, t_draft=1.0, t_verify=[1.0 + 0.002 * n for n in range(cap + 1)], dtype="f32", mask="bits")
    text = torch.randint(V, (B, 50), generator=gen, device="cuda", dtype=I32)
    length = torch.tensor([50, 31, 1, 0], dtype=I32, device="cuda")
    rep, freq = torch.full((B,), 1.3, device="cuda"), torch.full((B,), 0.2, device="cuda")
    draft = _rows(gen, B, L, V, F32)
    plain = draft.clone()
    ok = torch.rand((B, L, V), generator=gen, device="cuda") < 0.9
    kw = dict(history=text, history_len=length, repetition=rep, frequency=freq, allowed=_words(ok))
    adjust_logits(draft, draft, fill=-1e30, **kw)                          # (a plan takes finite logits)
    _check_adjust(plain, torch.where(draft == -1e30, -INF, draft), plain, kw, "draft")
    tree, ws = plan.new_outputs(B, topk=True), plan.new_workspace(B)
    plan.build(draft, tree, workspace=ws)
    target = _rows(gen, B, cap + 1, V, F32)
    _agree(target, tree.token_ids, tree.parent, tree.n_star, [4, 2, 0, 6], high=80.0)
    raw = target.clone()
    kw = dict(history=text, history_len=length, repetition=rep, frequency=freq, token_ids=tree.token_ids, parent=tree.parent, count=tree.n_star)
    adjust_logits(target, target, **kw)
    _check_adjust(raw, target, raw, kw, "target")
    acc, index, tokens, on = _outputs(B, cap + 1, L + 1)
    verify_tree(target, tree.token_ids, tree.parent, tree.n_star, acc, index, tokens, weight=on, workspace=verify_workspace(target))
    want = ref.verify(tree.token_ids.cpu().numpy(), tree.parent.cpu().numpy(), tree.n_star.cpu().numpy(), L + 1, logits=ref.f64(target))
    _check_verify((acc, index, tokens, on), want)
    cache = KVCache(heads, D, num_pages=B)
    table = torch.arange(B, dtype=I32, device="cuda").view(B, 1)
    k = torch.ones((B, cap + 1, heads, D), dtype=BF, device="cuda") * torch.arange(1, cap + 2, device="cuda").view(1, -1, 1, 1)
    start = torch.zeros(B, dtype=torch.int64, device="cuda")
    cache.write(k, k, table, start, count=acc, index=index)
    got, same = torch.zeros_like(k[:, :L + 1]), torch.zeros_like(k[:, :L + 1])
    cache.read(table, start + acc, got, same)
    for b in range(B):
        n = int(acc[b])
        rows = torch.tensor([index[b, j].item() + 1.0 for j in range(n)])
        # 4 bits: codes a and 1.5 a are the furthest apart, so a value between them is off by at most 0.25 a of 1.25 a
        assert torch.all((got[b, :n, 0, 0].float().cpu() - rows).abs() <= rows / 5)
    plan.reduce_topk(raw[:, :L].contiguous(), tree.topk_ids, tree.topk_logit, tree.lse, tree.topk_lq)
    student = plain.clone().requires_grad_()
    loss, grad = torch.zeros((B, L), device="cuda"), torch.zeros_like(plain)
    distill(student.detach(), tree.topk_ids, tree.topk_lq, loss, grad=grad, tail=True)
    (student * 1.0).backward(grad)
    assert torch.equal(student.grad, grad)
    _check_distill(plain, tree.topk_ids, tree.topk_lq, None, 1.0, True, loss, None, grad)
