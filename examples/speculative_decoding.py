"""Speculative decoding with draft trees over a 4-bit cache, on a toy target of one attention layer.

    python examples/speculative_decoding.py --rounds 24

Prompt: ``window_attention`` and ``KVCache.write``.  Each round: a draft tree (``Plan.build``), the target's
attention over cache and tree (``KVCache.attention``), the longest path of the tree that the target agrees with,
its tokens into the cache (``KVCache.write`` with an index) and the cached tokens' attention weight
(``KVCache.score``).  A sequence near its cache's end is cut to the tokens that were attended to most
(``KVCache.evict``).  Everything between two rounds stays on the device.

The target prefers one successor of every token by more than its attention can change, so the text it writes is
known; the drafter guesses that successor, or a wrong one, with its logits.
"""

import argparse
import os
import sys
from dataclasses import dataclass

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2606_01813_amd import KVCache, Plan, attention_workspace, window_attention

PAGE = 64


class Target:
    """One attention layer with random weights; its head adds 12 to the logit of the token's successor."""

    def __init__(self, vocab, heads, kv_heads, head_dim, gen):
        def weight(*shape):
            return (torch.randn(shape, generator=gen, device="cuda") / shape[0] ** 0.5).to(torch.bfloat16)
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.embed = weight(vocab, 256) * vocab ** 0.5
        self.wq, self.wk, self.wv = weight(256, heads * head_dim), weight(256, kv_heads * head_dim), weight(256, kv_heads * head_dim)
        self.head = weight(heads * head_dim, vocab)
        self.after = torch.randperm(vocab, generator=gen, device="cuda")

    def qkv(self, tokens):
        x = self.embed[tokens]
        cut = lambda y, n: y.view(*tokens.shape, n, self.head_dim)
        return cut(x @ self.wq, self.heads), cut(x @ self.wk, self.kv_heads), cut(x @ self.wv, self.kv_heads)

    def choose(self, tokens, attended):
        logits = (attended.flatten(-2) @ self.head).float()
        logits.scatter_add_(-1, self.after[tokens].unsqueeze(-1), torch.full((*tokens.shape, 1), 12.0, device="cuda"))
        return logits.argmax(-1)


def draft(target, last, L, gen):
    """The drafter's logits of the next L tokens: the successors', but for a quarter of the places a wrong token's first."""
    B, V = last.shape[0], target.after.numel()
    logits = torch.randn((B, L, V), generator=gen, device="cuda")
    token = last
    for i in range(L):
        token = target.after[token]
        logits[:, i].scatter_(1, token[:, None], 9.0)
        wrong = torch.randint(V, (B, 1), generator=gen, device="cuda")
        slip = torch.rand((B, 1), generator=gen, device="cuda") < 0.25
        at = logits[:, i].gather(1, wrong)
        logits[:, i].scatter_(1, wrong, torch.where(slip & (wrong != token[:, None]), 10.0, at))
    return logits.to(torch.bfloat16)


def accepted(tree, tokens, chosen, L):
    """Per sequence: which rows (root and nodes) are on the path that the target agrees with, in order and how many."""
    B, cap = tree.parent.shape
    nodes = torch.arange(cap, device="cuda") < tree.n_star[:, None]
    parent = torch.where(nodes, tree.parent, -1).to(torch.int64) + 1          # as rows
    agrees = nodes & (tokens[:, 1:] == chosen.gather(1, parent))
    on = torch.zeros((B, cap + 1), dtype=torch.bool, device="cuda")
    on[:, 0] = True
    for _ in range(L):
        on[:, 1:] = agrees & on.gather(1, parent)
    rows = torch.arange(cap + 1, device="cuda")
    depth = torch.cat([torch.zeros((B, 1), dtype=torch.int32, device="cuda"), tree.depth], 1)
    order = torch.where(on, depth.to(torch.int64) * (cap + 1) + rows, 1 << 40).argsort(1)[:, :L + 1]
    return on, order, on.sum(1).to(torch.int32)


@dataclass
class Run:
    text: torch.Tensor          # [B, tokens] int64: prompt and what was written
    length: torch.Tensor        # [B] its length
    accepted: torch.Tensor      # [rounds, B] tokens of each round
    cached: torch.Tensor        # [rounds, B] cached tokens after each round
    evictions: int
    target: Target
    cache: KVCache
    table: torch.Tensor
    ctx_len: torch.Tensor


def run(B=4, prompt=300, rounds=24, L=8, cap=24, slots=512, budget=320, window=0, seed=0) -> Run:
    """Evicts every sequence of the batch down to `budget` when one could outgrow its `slots` in the next round."""
    gen = torch.Generator("cuda").manual_seed(seed)
    target = Target(4096, 16, 4, 128, gen)
    plan = Plan(L=L, V=4096, K=4, cap=cap, t_draft=1.0, t_verify=[1.0 + 0.002 * n for n in range(cap + 1)], dtype="bf16", mask="bits")
    tree, ws = plan.new_outputs(B), plan.new_workspace(B)
    pages = slots // PAGE
    cache = KVCache(target.kv_heads, target.head_dim, num_pages=2 * B * pages)
    table, spare = torch.arange(2 * B * pages, dtype=torch.int32, device="cuda").view(2, B, pages).unbind(0)
    scores = torch.zeros((B, target.kv_heads, slots), device="cuda")
    spare_scores = torch.zeros_like(scores)
    kept = torch.zeros((B, target.kv_heads, budget), dtype=torch.int32, device="cuda")

    text = torch.zeros((B, prompt + rounds * (L + 1) + 1), dtype=torch.int64, device="cuda")
    text[:, :prompt] = torch.randint(4096, (B, prompt), generator=gen, device="cuda")
    q, k, v = target.qkv(text[:, :prompt])
    out = window_attention(q, k, v, window=window, sinks=4, workspace=attention_workspace(q, k))
    ctx_len = torch.zeros(B, dtype=torch.int64, device="cuda")
    cache.write(k, v, table, ctx_len)
    ctx_len += prompt
    last = target.choose(text[:, prompt - 1:prompt], out[:, -1:])[:, 0]       # (the bonus token: chosen, not yet cached)
    text[:, prompt] = last
    length = ctx_len + 1

    T = cap + 1
    lse = torch.zeros((B, T, target.heads), device="cuda")
    attended = torch.zeros((B, T, target.heads, target.head_dim), dtype=torch.bfloat16, device="cuda")
    attn_ws, most, evictions, took, cached = None, prompt, 0, [], []
    for _ in range(rounds):
        if most + L + 1 > slots:                                              # (an upper bound, known without asking the device)
            new_len = torch.empty_like(ctx_len)
            cache.evict(table, ctx_len, scores, spare, new_len, spare_scores, kept, budget=budget, sinks=4, recent=64)
            table, spare, scores, spare_scores, ctx_len = spare, table, spare_scores, scores, new_len
            most, evictions = budget, evictions + 1
        plan.build(draft(target, last, L, gen), tree, workspace=ws)
        tokens = torch.cat([last[:, None], tree.token_ids.to(torch.int64)], 1)
        live = torch.arange(T, device="cuda") <= tree.n_star[:, None]
        tokens = torch.where(live, tokens, 0)
        q, k, v = target.qkv(tokens)
        if attn_ws is None:
            attn_ws = attention_workspace(q, cache=cache, page_table=table)
        cache.attention(q, table, ctx_len, k, v, mask=tree.mask, depth=tree.depth, count=tree.n_star, window=window, sinks=4,
                        out=attended, lse=lse, workspace=attn_ws)
        chosen = target.choose(tokens, attended)
        on, order, count = accepted(tree, tokens, chosen, L)
        cache.score(q, table, ctx_len, lse, scores, weight=on.float(), count=tree.n_star, depth=tree.depth, window=window, sinks=4)
        cache.write(k, v, table, ctx_len, count=count, index=order.to(torch.int32))
        ctx_len = ctx_len + count
        new = chosen.gather(1, order)                                         # each accepted row's choice: the next row, or the bonus
        at = torch.arange(L + 1, device="cuda")
        text.scatter_(1, torch.where(at < count[:, None], length[:, None] + at, text.shape[1] - 1), new)
        length = length + count
        last = new.gather(1, count[:, None].to(torch.int64) - 1)[:, 0]
        most += L + 1
        took.append(count)
        cached.append(ctx_len)
    return Run(text, length, torch.stack(took), torch.stack(cached), evictions, target, cache, table, ctx_len)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--rounds", type=int, default=24)
    p.add_argument("--window", type=int, default=0)
    a = p.parse_args()
    r = run(B=a.batch, rounds=a.rounds, window=a.window)
    print(f"{a.batch} sequences, {a.rounds} rounds: {r.accepted.float().mean():.2f} tokens a round, "
          f"{r.evictions} evictions, cached {r.cached[-1].tolist()} of {r.length.tolist()} tokens")


if __name__ == "__main__":
    main()
