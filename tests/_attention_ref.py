"""Attention, the 4-bit cache and its eviction from their definitions, in fp64 on the CPU.  Test
infrastructure: it shares no code with the library.

Error bounds that the tests use.  With u the unit roundoff of the 16-bit type (2^-8 for bf16, 2^-11 for
f16) a result is rounded once (u |out|), and each weight once before its product with v (u A with A =
sum_j p_j |v_j|).  A score is a sum of D exact products in fp32: off by at most ds = D 2^-24 scale
sum_d |q_d k_d|, which shifts a weight by a factor of 1 + ds and the normaliser likewise (2 ds A); the
exponentials, the running sums and the division add less than 2^-14 A.
"""

import math

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
ROUNDOFF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
EXPONENTS = {torch.bfloat16: (-125, 125), torch.float16: (-13, 13)}


def attend(q, k, v, seen, scale, u):
    """q [Hq, D], k, v [n, Hkv, D] (fp64 arrays), seen [n]: out [Hq, D], lse [Hq] and how far they may be off."""
    Hq, D = q.shape
    G = Hq // k.shape[1]
    out, lse, tol, ltol = np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros((Hq, D)), np.zeros(Hq)
    idx = np.flatnonzero(seen)
    if len(idx) == 0:
        return out, lse, tol, ltol
    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(Hq):
            kk, vv = k[idx, h // G], v[idx, h // G]
            s = scale * (kk @ q[h])
            m = s.max()
            p = np.exp(s - m)
            lse[h] = m + np.log(p.sum())
            p = p / p.sum()
            out[h] = p @ vv
            A = p @ np.abs(vv)
            ds = D * 2.0 ** -24 * abs(scale) * (np.abs(kk) @ np.abs(q[h])).max()
            tol[h] = u * np.abs(out[h]) + (u + 2 * ds + 2.0 ** -14) * A + 2.0 ** -24
            ltol[h] = ds + 2.0 ** -18 * (1 + abs(lse[h]))
    return out, lse, tol, ltol


def in_window(pos_q, pos_k, window, sinks):
    return np.ones_like(pos_k, dtype=bool) if window == 0 else (pos_q - pos_k < window) | (pos_k < sinks)


def window_reference(q, k, v, window, sinks, causal, scale, q_len, k_len):
    """q, k, v as [B, T, H, D] tensors; yields (b, i, out, lse, tol, ltol) for every query there is."""
    u = ROUNDOFF[q.dtype]
    q, k, v = (x.double().cpu().numpy() for x in (q, k, v))
    for b in range(q.shape[0]):
        nq, nk = int(q_len[b]), int(k_len[b])
        pos = np.arange(nk)
        for i in range(nq):
            p = nk - nq + i
            seen = in_window(p, pos, window, sinks)
            if causal:
                seen = seen & (pos <= p)
            yield (b, i) + attend(q[b, i], k[b, :nk], v[b, :nk], seen, scale, u)


def cache_reference(q, ck, cv, ctx, k, v, order, ancestors, depth, count, window, sinks, scale):
    """q [B, T, Hq, D]; ck, cv: per sequence the cached tokens [ctx, Hkv, D] as fp64 arrays (NaN scale blocks
    included), missing[b]: slots whose page is not there are left out by the caller.  k, v [B, T, Hkv, D] or
    None.  ancestors[b][i]: the new keys that query i of a tree sees."""
    u = ROUNDOFF[q.dtype]
    q = q.double().cpu().numpy()
    for b in range(q.shape[0]):
        n = int(count[b]) + (order == "tree")
        n = min(n, q.shape[1])
        slots, kk, vv = ck[b][0], ck[b][1], cv[b][1]
        pos = slots
        step = [0 if order == "tree" and j == 0 else int(depth[b][j - 1]) if order == "tree" else j for j in range(n)]
        if k is not None:
            kk = np.concatenate([kk, k[b, :n].double().cpu().numpy()])
            vv = np.concatenate([vv, v[b, :n].double().cpu().numpy()])
            pos = np.concatenate([pos, ctx[b] + np.array(step, dtype=np.int64)])
        for i in range(n):
            seen = in_window(ctx[b] + step[i], pos, window, sinks)
            if k is not None:
                new = np.ones(n, dtype=bool)
                if order == "chain":
                    new = np.arange(n) <= i
                elif order == "tree":
                    new = np.isin(np.arange(n), list(ancestors[b][i]))
                seen = seen & np.concatenate([np.ones(len(slots), dtype=bool), new])
            yield (b, i) + attend(q[b, i], kk, vv, seen, scale, u)


def quantise(x):
    """A [..., D] tensor of a 16-bit type: the 4-bit values as fp64, block by block and value by value."""
    lo, hi = EXPONENTS[x.dtype]
    a = np.ascontiguousarray(x.double().cpu().numpy())
    out = np.empty_like(a)
    flat, res = a.reshape(-1, 32), out.reshape(-1, 32)
    for r in range(flat.shape[0]):
        blk = flat[r]
        if not np.all(np.isfinite(blk)):
            res[r] = np.nan
            continue
        m = np.abs(blk).max()
        e = lo if m == 0 else math.floor(math.log2(m))
        if m > 0:
            while 2.0 ** e > m:
                e -= 1
            while 2.0 ** (e + 1) <= m:
                e += 1
            e = e - 2 + (1 if m > 1.75 * 2.0 ** e else 0)
        scale = 2.0 ** min(max(e, lo), hi)
        for c in range(32):
            off = np.abs(abs(blk[c]) / scale - GRID)
            best = np.flatnonzero(off == off.min())
            g = best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1]
            res[r, c] = math.copysign(GRID[g] * scale, blk[c])
    return out


def evict(scores, n, budget, sinks, recent):
    """The slots a kv head keeps, by sorting them all."""
    if n <= budget:
        return list(range(n))
    forced = set(range(sinks)) | set(range(n - recent, n))
    rest = [p for p in range(n) if p not in forced]
    rest.sort(key=lambda p: (1, 0.0, p) if math.isnan(scores[p]) else (0, -float(scores[p]), p))
    return sorted(forced | set(rest[:budget - len(forced)]))
