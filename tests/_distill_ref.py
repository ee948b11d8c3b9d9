"""Distillation's loss, gradient and stats from the definition in fp64 on the CPU, in logarithms, for rows whose logits lie far
from 0 or far from each other.  Test infrastructure: it shares no code with the library, nor with _logits_ref.py.

S = sum of exp((l_v - r) / tau) over the tokens not listed, r the largest of these, R = S exp((r - m) / tau) with m the row's
largest, Z = R + the listed tokens' terms.  Where R is not a number of fp64 the student gives the rest nothing, and its term is
left out of the loss.

Error bounds (h = 2^-24, u half a step of the logits' type).  With d = (l_v - r) / tau, a term is 2^x, to a step (2 h), of an
argument that is c = log2(e) / tau rounded (h |d|) times the distance, less a reference at most 8 below the largest of the sum it
is in, rounded once (h (|d| + 8 ln 2)); far from 0 three roundings of d.  Both are below t_v = h (3 |d| + 8).  Eight terms at most
are summed in fp32 (7 h), a sum moves by two such powers with arguments below 1/2 (3 h each).  What is below the smallest normal
number, of 1 at the largest, may be left out.  So eR = sum e_v t_v / S + 13 h + V 2^-126.  A listed token's term is off by 3 h, and
so is R where it moves to the row's largest: eZ = (R (eR + 3 h) + 3 h (Z - R)) / Z.
    stats: the largest is exact, the sums are rounded once (h); a logarithm is off by h of itself and eR / ln 2.
    loss: |w| (M eZ + rho eR), fp64's own roundings of its terms, and one rounding.
    gradient of a listed token: q M (eZ + 3 h); of another t_v + 5 h (the reference, the coefficient, the product), and eZ and eR of
    its two parts, 3 h where q moves; then u.
A second call starts from R and Z in fp32 (h each), or from R's logarithm (h |ln R|), and its reference is within 2^-1 of R and so
up to log2 V from the largest term: 18 ln 2 h more in the argument's rounding.
"""

import math

import numpy as np
import torch

H = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}
NONE = 1074 * math.log(2)                                  # exp(-NONE): the smallest number of fp64


def distill(l, ids, target, w, tau, tail, dtype, again=False):
    """One row of finite logits, or -inf: (loss, stats [3], gradient [V], and how far each may be off)."""
    V = len(l)
    keep = (ids >= 0) & (ids < V)
    ids, t = ids[keep], target[keep]
    top = t.max() if len(t) else 0.0
    logp = t if tail else (t - top) / tau - math.log(np.exp((t - top) / tau).sum())
    p = np.exp(logp)
    rho = max(0.0, 1.0 - math.fsum(p)) if tail else 0.0
    M = math.fsum(p) + rho
    on = np.zeros(V, bool)
    on[ids] = True
    m, r = l.max(), (l[~on].max() if not on.all() else -np.inf)
    S = eR = R = 0.0
    e, term, lnR = np.zeros(V), np.zeros(V), -np.inf
    if r > -np.inf:
        d = np.where(on, -np.inf, (np.where(on, r, l) - r) / tau)
        with np.errstate(under="ignore"):
            e = np.exp(d)
        far = np.where(np.isfinite(d), np.abs(np.where(np.isfinite(d), d, 0.0)), 0.0)
        term = H * (3 * np.minimum(far, 200.0) + 8)        # (a term further off than that is 0 on both sides)
        S = float(e.sum())
        eR = float((e * term).sum() / S) + 13 * H + V * 2.0 ** -126
        lnR = math.log(S) + (r - m) / tau
        R = math.exp(lnR) if lnR > -NONE else 0.0
    dl = np.where(on, (np.where(on, l, m) - m) / tau, 0.0)  # of the listed
    with np.errstate(under="ignore"):
        q = np.where(on, np.exp(dl), 0.0)
    Z = R + float(q.sum())
    eZ = (R * (eR + 3 * H) + 3 * H * (Z - R)) / Z
    lnZ = math.log(Z)
    loss, size, teacher = 0.0, 0.0, np.zeros(V)
    for pk, lk, i in zip(p, logp, ids):
        teacher[i] += pk
        if pk > 0:
            loss += pk * (lk - (dl[i] - lnZ))
            size += pk * (abs(lk) + abs(dl[i]) + lnZ)
    if rho > 0 and R > 0:
        loss += rho * (math.log(rho) - (lnR - lnZ))
        size += rho * (abs(math.log(rho)) + abs(lnR) + lnZ) + 2.0 ** -52 * (abs(lnR) + abs(math.log(rho)) + 1)   # (rho: 1 - P)
    loss_tol = abs(w) * (M * eZ + rho * eR + 2.0 ** -46 * size) + H * abs(w * loss)
    more = (1 + 18 * math.log(2)) * H if again else 0.0
    moreR = more + (H * abs(lnR) if again and 0 < R < 2.0 ** -126 else 0.0)
    g = w / tau * (q / Z * M - teacher)
    tol = abs(w) / tau * q / Z * M * (eZ + 3 * H + (H if again else 0))
    if R > 0:
        a, b = e * math.exp(lnR - lnZ) / S * M, rho * e / S
        g = np.where(on, g, w / tau * (a - b))
        tol = np.where(on, tol, abs(w) / tau * (a * (eZ + 8 * H + term + more) + b * (eR + 5 * H + term + moreR)))
    with np.errstate(over="ignore"):
        loss = float(np.float32(w * loss)) if abs(w * loss) > np.finfo(np.float32).max else w * loss
    tol = tol + U[dtype] * np.abs(g) + TINY[dtype] * max(1.0, abs(w) / tau)
    stats, off = np.array([m, Z, R]), np.array([0.0, (eZ + H) * Z, (eR + 4 * H) * R])
    if 0 < R < 2.0 ** -126:
        stats[2], off[2] = lnR / math.log(2), H * abs(lnR) / math.log(2) + eR / math.log(2)
    return loss, stats, g, loss_tol, off, tol
