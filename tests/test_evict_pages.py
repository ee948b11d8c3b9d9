"""Eviction from tables with pages outside the cache, which hold no key (GPU): what is kept has keys, and attention over
it is attention over the same keys as before."""

import pytest
import torch

from paper_2606_01813_amd import KVCache
from tests import _attention_ref as ref
from tests.test_attention import BF, F16, check, evict, i32, i64, make

pytestmark = pytest.mark.gpu


class Holed:
    """Sequences of random tokens; `gone` are (sequence, page) of the table that name no page.  Memory that is not
    theirs holds scale bytes of 255, which read as NaN."""

    def __init__(self, Hkv, D, ctx, gone, budget, dtype=BF):
        B, room = len(ctx), max(1, -(-max(ctx) // 64))
        self.ctx, self.D, self.dtype = ctx, D, dtype
        n = B * (room + max(1, -(-budget // 64)) + 1)
        self.cache = KVCache(Hkv, D, n, dtype="bf16" if dtype == BF else "f16")
        self.cache.pages.fill_(255)
        self.table = torch.randperm(n, generator=torch.Generator().manual_seed(3))[:B * room].to(torch.int32).view(B, room).cuda()
        k, v = make((B, room * 64, Hkv, D), dtype, 1), make((B, room * 64, Hkv, D), dtype, 2)
        self.cache.write(k, v, self.table, i64([0] * B), count=i32(ctx))
        self.k, self.v = torch.zeros_like(k), torch.zeros_like(v)
        self.cache.read(self.table, i64(ctx), self.k, self.v)
        holes = [-1, n, -2 ** 31, 2 ** 31 - 1]
        for j, (b, p) in enumerate(gone):
            if p < room:
                self.table[b, p] = holes[j % 4]
        missing = set(gone)
        self.slots = [[t for t in range(ctx[b]) if (b, t // 64) not in missing] for b in range(B)]


def wanted(scores, slots, n, budget, sinks, recent):
    if len(slots) <= budget:
        return slots
    forced = [p for p in slots if p < sinks or p >= n - recent]
    rest = [p for p in slots if sinks <= p < n - recent]
    rest.sort(key=lambda p: (-float(scores[p]), p))
    return sorted(forced + rest[:budget - len(forced)])


HOLES = [
    # Hkv, D, ctx, gone, budget, sinks, recent
    (2, 64, [400, 190, 64], [(0, 0), (0, 4), (1, 2), (2, 0)], 500, 4, 8),                 # all fit
    (2, 128, [400, 190, 64], [(0, 0), (0, 4), (1, 2)], 100, 70, 20),                       # sinks and recent ones among the holes
    (1, 64, [400, 300], [(0, 1), (0, 2), (0, 3), (1, 0), (1, 1), (1, 2), (1, 3), (1, 4)], 200, 0, 0),   # fewer keys than the budget
    (1, 64, [5000, 4097], [(0, 3), (0, 70), (1, 64)], 1000, 100, 30),                      # (one: the last page, of one slot)
    (2, 64, [9000, 16384], [(b, p) for b in (0, 1) for p in range(0, 256, 3)], 4000, 5, 100),
    # rows in parts: all fit, a hole that is a whole part, fewer keys than the budget
    (2, 64, [20000, 100], [(0, 0), (0, 200), (1, 1), (0, 312)], 25000, 4, 8),
    (2, 64, [30000, 16385], [(0, p) for p in range(128, 256)] + [(1, 0), (1, 256)], 8000, 500, 1000),
    (1, 64, [40000, 33000], [(0, p) for p in range(2, 600)] + [(1, 5)], 30000, 10, 10),
    (1, 128, [40000], [(0, p) for p in range(0, 625, 2)], 300, 100, 200),                  # nothing but sinks and recent ones
]


@pytest.mark.parametrize("ties", [False, True], ids=["spread", "ties"])
@pytest.mark.parametrize("case", HOLES, ids=[str(i) for i in range(len(HOLES))])
def test_slots_without_a_key_are_not_kept(case, ties):
    Hkv, D, ctx, gone, budget, sinks, recent = case
    f = Holed(Hkv, D, ctx, gone, budget)
    B = len(ctx)
    x = torch.rand((B, Hkv, f.table.shape[1] * 64), generator=torch.Generator().manual_seed(9))
    if ties:
        x = (x * 3).floor()
    new_table, new_len, new_scores, kept = evict(f, x.cuda(), budget, sinks, recent)
    rk, rv = (torch.full((B, max(budget, 1), Hkv, D), 7.0, dtype=BF, device="cuda") for _ in range(2))
    f.cache.read(new_table, new_len, rk, rv)
    for b in range(B):
        m = min(len(f.slots[b]), budget)
        assert int(new_len[b]) == m
        for h in range(Hkv):
            want = wanted(x[b, h], f.slots[b], ctx[b], budget, sinks, recent)
            assert len(want) == m and kept[b, h].tolist() == want + [-1] * (budget - m), (b, h)
            assert torch.equal(new_scores[b, h, :m].cpu(), x[b, h, want]) and torch.all(new_scores[b, h, m:] == 0.0)
            at = torch.tensor(want, dtype=torch.int64, device="cuda")
            assert torch.equal(rk[b, :m, h], f.k[b, at, h]) and torch.equal(rv[b, :m, h], f.v[b, at, h])
        assert torch.all(rk[b, m:] == 7.0)


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("T", [1, 30])
def test_attention_over_what_was_kept(T, dtype):
    """All slots with a key fit: attention and scores are over the same keys before and after."""
    f = Holed(2, 64, [300, 190, 64], [(0, 0), (0, 3), (1, 1), (2, 0)], 256, dtype)
    q = make((3, T, 4, 64), dtype, 5)
    x = torch.zeros((3, 2, f.table.shape[1] * 64), device="cuda")
    new_table, new_len, _, _ = evict(f, x, 256, 2, 5)
    assert new_len.tolist() == [len(s) for s in f.slots] == [300 - 2 * 64, 190 - 64, 0]
    k, v = (t.double().cpu().numpy() for t in (f.k, f.v))
    want = []
    for b, slots in enumerate(f.slots):
        for i in range(T):
            want.append((b, i) + ref.attend(q[b, i].double().cpu().numpy(), k[b, slots], v[b, slots], [True] * len(slots), 0.125,
                                            ref.ROUNDOFF[dtype]))
    for table, lengths in ((f.table, i64(f.ctx)), (new_table, new_len)):
        out, lse = torch.full_like(q, 7.0), torch.full((3, T, 4), 7.0, device="cuda")
        f.cache.attention(q, table, lengths, out=out, lse=lse)
        check(want, out, lse)
        got = torch.zeros((3, 2, table.shape[1] * 64), device="cuda")
        f.cache.score(q, table, lengths, lse, got)
        total = got.sum(-1)                               # each query's two heads of a kv head: weights that sum to 1
        assert torch.all((total[:2] - 2 * T).abs() < 1e-4 * T) and torch.all(total[2] == 0.0)
