"""The operators on logits from their definitions, in fp64 on the CPU, row by row.  Test infrastructure: it shares no code
with the library.

Error bounds.  h = 2^-24 is half a step of fp32, u that of the logits' type (a result is rounded to it once).
Adjusting: a quotient (a product with a rounded inverse, 2 h) or product, a fused product and difference, a difference and a
sum, each off by h of its result, which is at most S = |x| max(r, 1 / r) + f c + p + |bias|: 5 h S in all (f c is not rounded,
c < 2^24).
Distilling: with d = (l_v - m) / tau <= 0 a term is the hardware's 2^x (off by a step, 2 h) of l c - r, rounded once, with
c = log2(e) / tau rounded to fp32 (h |d|) and a reference r at most 8 below the largest in 2^x: the rounding is h (|d| + 8 ln 2).
Far from the numbers' middle it is 2^((l - m) c): three roundings of d.  Both are below t_v = h (3 |d| + 8), relative to the
term; without the reference's distance, as the gradient has it, t'_v = h (3 |d| + 2).  Up to eight terms are summed in fp32 (at
most 7 h) before the sum goes on in fp64; a sum moves to the row's largest by a 2^x with an argument below 1/2 (3 h), as a
listed token's term is formed.  So R, the sum over what is not listed, is off by dR = sum e_v (t_v + 7 h) + 3 h R, and Z over all
by dR + 3 h (Z - R); eR and eZ are these relative to R and Z.  All sums over the list are fp64.
    stats: the largest is exact, the sums are rounded once more (h).
    loss: |w| [(P + rho) eZ + rho eR] and one rounding.
    gradient: of a listed token (eZ + 3 h) q M, of another t'_v + 5 h (the reference, the coefficient and the product), and eZ
    and eR, of both of its parts; then u of the result.
A second call starts from sums in fp32: h more for each.  Results below the smallest normal fp32 number may be flushed; f16 has
steps of 2^-24 below 2^-14.
"""

import math

import numpy as np
import torch

H = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -125, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -125}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def path_of(parent, row):
    """Nodes from row's own up to the root's child, the last 32 of a longer path."""
    node, got = row - 1, []
    while node >= 0 and len(got) < 32:
        got.append(node)
        node = parent[node] if parent[node] < node else -1
    return got


def adjust(x, dtype, *, history=None, history_len=None, repetition=None, presence=None, frequency=None, bias_ids=None, bias=None,
           allowed=None, token_ids=None, parent=None, count=None):
    """(out, how far it may be off) for x [B, T, V] in fp64; rows past count are NaN in out."""
    B, T, V = x.shape
    out, tol = np.full(x.shape, np.nan), np.zeros(x.shape)
    num = lambda a: None if a is None else a.cpu().numpy()
    history, history_len, bias_ids, token_ids, parent, count = map(num, (history, history_len, bias_ids, token_ids, parent, count))
    words = None if allowed is None else allowed.cpu().numpy().astype(np.int64) & 0xffffffff
    per = lambda t, b, default: default if t is None else float(t[b])
    for b in range(B):
        rows = T if count is None else (min(max(int(count[b]), 0), T - (parent is not None)) + (parent is not None))
        r, p, f = per(repetition, b, 1.0), per(presence, b, 0.0), per(frequency, b, 0.0)
        bv = {}
        if bias_ids is not None:
            for i, v in zip(bias_ids[b], bias[b].tolist()):
                if 0 <= i < V:
                    bv[int(i)] = v
        for t in range(rows):
            c = np.zeros(V)
            if history is not None:
                n = history.shape[1] if history_len is None else min(max(int(history_len[b]), 0), history.shape[1])
                for tok in history[b, :n]:
                    if 0 <= tok < V:
                        c[tok] += 1
            if parent is not None:
                for node in path_of(parent[b], t):
                    if 0 <= token_ids[b, node] < V:
                        c[token_ids[b, node]] += 1
            y = x[b, t].copy()
            size = np.zeros(V)
            on = c > 0
            with np.errstate(invalid="ignore"):
                y[on] = np.where(y[on] > 0, y[on] / r, y[on] * r) - f * c[on] - p
                size[on] = np.abs(x[b, t][on]) * max(abs(r), 1 / abs(r)) + abs(f) * c[on] + abs(p)
                for i, v in bv.items():
                    size[i] = (size[i] if on[i] else abs(x[b, t, i])) + abs(v)
                    y[i] += v
            if words is not None:
                v = np.arange(V)
                y[(words[b, t, v // 32] >> (v % 32)) & 1 == 0] = -np.inf
            out[b, t] = y
            with np.errstate(invalid="ignore"):
                tol[b, t] = np.where(size > 0, np.nan_to_num(5 * H * size + U[dtype] * np.abs(y), nan=0.0, posinf=0.0), 0.0)
                if dtype == torch.float16:
                    tol[b, t] += np.where(size > 0, TINY[dtype], 0.0)
    return out, tol


def verify(token_ids, parent, count, M, logits=None, chosen=None):
    """accepted, index, tokens and the path's weight, from logits [B, T, V] or chosen [B, T] (numpy)."""
    B, T = (logits if logits is not None else chosen).shape[:2]
    acc = np.zeros(B, np.int32)
    index, tokens = np.full((B, M), -1, np.int32), np.full((B, M), -1, np.int32)
    weight = np.zeros((B, T), np.float32)
    for b in range(B):
        row, n = 0, min(max(int(count[b]), 0), T - 1)
        while True:
            if chosen is not None:
                t = int(chosen[b, row])
            else:
                x = np.where(np.isnan(logits[b, row]), -np.inf, logits[b, row])
                t = int(x.argmax()) if x.max() > -np.inf else -1
            index[b, acc[b]], tokens[b, acc[b]], weight[b, row] = row, t, 1.0
            acc[b] += 1
            kids = [i for i in range(n) if parent[b, i] == row - 1 and i >= row and token_ids[b, i] == t]
            if acc[b] == M or t < 0 or not kids:
                break
            row = kids[0] + 1
    return acc, index, tokens, weight


def _exp(x):
    return math.exp(x) if x > -math.inf else 0.0


def distill(l, ids, target, w, tau, tail, dtype, again=False):
    """One row: loss, stats [3], gradient [V] and how far each may be off.  again: the gradient starts from stats in fp32."""
    V = len(l)
    zero = (0.0, np.zeros(3), np.zeros(V), 0.0, np.zeros(3), np.zeros(V))
    if w == 0:
        return zero
    keep = (ids >= 0) & (ids < V)
    ids, t = ids[keep], target[keep]
    if tail:
        p, logp = np.exp(t), t
        rho = max(0.0, 1.0 - p.sum())
    else:
        rho, top = 0.0, t.max() if len(t) else 0.0
        if top == -np.inf:
            p, logp = np.zeros(len(t)), t
        else:
            logp = (t - top) / tau
            logp = logp - math.log(np.exp(logp).sum()) if len(t) else logp
            p = np.exp(logp)
    on = np.zeros(V, bool)
    on[ids] = True
    m = l.max()
    d = (l - m) / tau if m > -np.inf else np.full(V, -np.inf)
    with np.errstate(under="ignore"):
        e = np.exp(d)
    term = np.where(d > -np.inf, H * (3 * np.abs(np.where(d > -np.inf, d, 0.0)) + 2), 0.0)
    Z, R = e.sum(), e[~on].sum()
    dR = (e * (term + 13 * H))[~on].sum() + 3 * H * R + TINY[torch.float32] * V
    dZ = dR + 3 * H * (Z - R)
    eZ, eR = (dZ / Z if Z > 0 else 0.0), (dR / R if R > 0 else 0.0)
    loss, M = 0.0, p.sum() + rho
    teacher = np.zeros(V)
    for pk, lk, i in zip(p, logp, ids):
        teacher[i] += pk
        if pk > 0:
            loss += pk * (lk - (d[i] - math.log(Z) if d[i] > -np.inf else -np.inf))
    if rho > 0 and R > 0:
        loss += rho * (math.log(rho) - math.log(R / Z))
    q = e / Z if Z > 0 else e
    g = w / tau * (q * M - teacher)
    loose = eZ + (H if again else 0)
    tol = np.abs(w) / tau * q * M * (loose + 3 * H)
    if R > 0:
        other = rho * e / R
        g = np.where(on, g, w / tau * (q * M - other))
        more = eR + (H if again else 0) + 5 * H + term
        tol = np.where(on, tol, np.abs(w) / tau * (q * M * (loose + 5 * H + term) + other * more))
    tol = tol + U[dtype] * np.abs(g) + TINY[dtype] * max(1.0, abs(w) / tau)
    loss_tol = abs(w) * (M * eZ + rho * eR + 1e-12 * (1 + abs(loss))) + H * abs(w * loss) if np.isfinite(loss) else 0.0
    stats = np.array([m, Z, R])
    with np.errstate(over="ignore"):
        loss = float(np.float32(w * loss)) if abs(w * loss) > np.finfo(np.float32).max else w * loss     # (past fp32's range: infinite)
    return loss, stats, g, loss_tol, np.array([0.0, dZ + H * Z, dR + H * R]), tol
