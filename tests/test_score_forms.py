"""Accumulated attention weight over many pages, many queries and tables with holes (GPU), against 64 bits.

A wavefront of the score kernel takes several pages where a call has 16384 pages and kv heads or more, and more than 512
queries come in chunks; the sizes here reach both, alone and together.

Bounds: a weight's exponent is off by at most ds (as in _attention_ref) and 2^-18 of it by exp2 and the sum with lse in
fp32; a score is a sum in fp32 of at most a quarter of the rows in a lane and a few more."""

import pytest
import torch

from paper_2606_01813_amd import KVCache
from tests._parity import say
from tests.test_attention import BF, F16, Filled, i32, i64, make

pytestmark = pytest.mark.gpu

FORMS = [
    # B, T, Hq, Hkv, D, pages, ctx, count, window, sinks, weights, holes
    (4, 1, 16, 8, 64, 515, [32955, 20001, 1, 0], None, 0, 0, "ones", False),              # 2 pages a wavefront, at most 16 rows
    (4, 3, 8, 8, 64, 1030, [65920, 40000, 64, 65857], [3, 2, 1, 3], 0, 0, "some", False),  # 4 pages
    (4, 5, 32, 8, 64, 515, [32955, 20001, 63, 0], None, 0, 0, "some", False),              # 2 pages, more rows
    (4, 9, 16, 8, 64, 1030, [65900, 40000, 64, 65857], [9, 2, 1, 0], 0, 0, "some", False),
    (2, 2, 8, 8, 128, 1500, [96000, 70007], None, 70000, 70, "ones", False),               # a window over most of them
    (2, 513, 4, 2, 64, 7, [400, 130], None, 0, 0, "some", False),                          # a second chunk of one query
    (2, 1100, 3, 1, 128, 5, [257, 320], [1100, 700], 200, 3, "some", False),
    (1, 1100, 2, 2, 64, 4, [200], None, 0, 0, "gap", False),                               # a chunk without a weight
    (1, 1100, 2, 2, 64, 4, [200], None, 0, 0, "none", False),
    (3, 600, 16, 8, 64, 700, [44800, 30000, 5], [600, 513, 512], 0, 0, "few", False),      # several pages and chunks
    (4, 1100, 8, 8, 64, 1030, [65920, 1, 50000, 0], None, 40000, 5, "gap", False),
    (2, 2, 4, 2, 64, 9, [570, 300], None, 0, 0, "ones", True),
    (2, 40, 4, 2, 128, 9, [570, 300], None, 100, 70, "some", True),
    (4, 1, 16, 8, 64, 515, [32955, 20001, 100, 0], None, 0, 0, "ones", True),
    (4, 600, 8, 8, 64, 515, [32955, 20001, 100, 0], None, 0, 0, "few", True),
]


def weights(kind, B, T):
    g = torch.Generator().manual_seed(11)
    w = torch.rand((B, T), generator=g)
    if kind == "ones":
        return None
    if kind == "none":
        return torch.where(w < 0.5, 0.0, -w)
    keep = {"some": 0.4, "few": 0.02, "gap": 0.05}[kind]
    w = torch.where(torch.rand((B, T), generator=g) < keep, 0.25 + w, torch.where(w < 0.5, 0.0, -1.0))
    w[:, T // 3] = 1.0
    if kind == "gap":
        w[:, 512:1024] = 0.0
    return w


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("case", FORMS, ids=[str(i) for i in range(len(FORMS))])
def test_score_forms(case, dtype):
    B, T, Hq, Hkv, D, pages, ctx, count, window, sinks, kind, holed = case
    say(f"[attention] score {case} {dtype}")
    G, scale, slots = Hq // Hkv, D ** -0.5, pages * 64
    n = B * pages + 2
    cache = KVCache(Hkv, D, n, dtype="bf16" if dtype == BF else "f16")
    cache.pages.fill_(255)
    table = torch.randperm(n, generator=torch.Generator().manual_seed(3))[:B * pages].to(torch.int32).view(B, pages).cuda()
    k = torch.empty((B, slots, Hkv, D), dtype=dtype, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    cache.write(k, k, table, i64([0] * B), count=i32(ctx))
    keys = torch.zeros_like(k)
    cache.read(table, i64(ctx), keys, torch.zeros_like(k))
    there = torch.arange(slots, device="cuda") < i64(ctx)[:, None]
    if holed:
        gone = torch.rand((B, pages), generator=torch.Generator().manual_seed(5)).cuda() < 0.3
        table = torch.where(gone, torch.where(torch.rand((B, pages), generator=torch.Generator().manual_seed(6)).cuda() < 0.5, -1, n),
                            table).to(torch.int32)
        there &= ~gone.repeat_interleave(64, 1)
    q = make((B, T, Hq, D), dtype, 5)
    num = count or [T] * B
    for b in range(B):
        q[b, num[b]:] = float("nan")
    w = weights(kind, B, T)
    old = torch.rand((B, Hkv, slots), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    lse = torch.full((B, T, Hq), float("nan"), device="cuda")
    want, tol = old.double(), torch.zeros((B, Hkv, slots), dtype=torch.float64, device="cuda")
    at = torch.arange(slots, device="cuda")
    for b in range(B):
        picked = [i for i in range(num[b]) if w is None or w[b, i] > 0]
        if not picked:
            continue
        pos = ctx[b] + torch.tensor(picked, device="cuda")
        seen = there[b] & ((pos[:, None] - at < window) | (at < sinks)) if window else there[b].expand(len(picked), -1)
        share = torch.ones(len(picked), dtype=torch.float64, device="cuda") if w is None else w[b, picked].double().cuda()
        for h in range(Hq):
            x, y = q[b, picked, h].double(), keys[b, :, h // G].double()
            s = (x @ y.t()) * scale
            lse[b, picked, h] = torch.logsumexp(torch.where(seen, s, -float("inf")), 1).float()
            p = torch.where(seen, share[:, None] * torch.exp(s - lse[b, picked, h].double()[:, None]), 0.0)
            ds = D * 2.0 ** -24 * scale * (x.abs() @ y.abs().t())
            want[b, h // G] += p.sum(0)
            tol[b, h // G] += (p * (ds + 2.0 ** -18)).sum(0)
    tol += 2.0 ** -24 * (T * G / 4 + 16) * want
    new = torch.full_like(old, 7.0)
    kw = dict(weight=None if w is None else w.cuda(), count=None if count is None else i32(count), window=window, sinks=sinks)
    cache.score(q, table, i64(ctx), lse, old, new, **kw)
    again = old.clone()
    cache.score(q, table, i64(ctx), lse, again, **kw)               # in place
    torch.cuda.synchronize()
    assert torch.equal(new, again)
    assert torch.equal(new[~there[:, None].expand_as(new)], old[~there[:, None].expand_as(old)])
    off = (new.double() - want).abs()
    assert torch.all(off <= tol), float((off / tol.clamp(min=1e-30)).max())


@pytest.mark.parametrize("T", [3, 40])
def test_lse_in_any_strides(T):
    f = Filled(2, 4, 64, [300, 70], BF)
    q = make((2, T, 4, 64), BF, 5)
    lse = torch.zeros((2, T, 4), device="cuda")
    f.cache.attention(q, f.table, i64(f.ctx), lse=lse)
    zero = torch.zeros((2, 4, f.table.shape[1] * 64), device="cuda")

    def score(x):
        got = torch.full_like(zero, 7.0)
        f.cache.score(q, f.table, i64(f.ctx), x, zero, got)
        torch.cuda.synchronize()
        return got

    want = score(lse)
    wide = torch.full((2, 2 * T, 9), float("nan"), device="cuda")
    wide[:, ::2, 3:7] = lse
    for x in (lse.transpose(1, 2).contiguous().transpose(1, 2), lse.permute(2, 1, 0).contiguous().permute(2, 1, 0), wide[:, ::2, 3:7]):
        assert not x.is_contiguous() and torch.equal(score(x), want)
    same = lse[:, :1, :1]
    assert torch.equal(score(same.expand(2, T, 4)), score(same.expand(2, T, 4).contiguous()))
