"""Attention rows in float64 and how far a kernel may be from them.

``rows`` takes q [R, d], K and V [L, d] and what each row sees [R, L].  Its bounds follow
from the roundings a kernel makes, each at most half a step:

* a logit is a float32 sum of d products, within (d + 8) 2^-24 sum |q_i k_i| / sqrt(d), and
  an exponential is within 2^-22: every weight is off by a factor 1 + dl;
* over bf16 values a weight is rounded to bf16 (2^-8 of it), and o is divided by the sum of
  the rounded weights, so with weights p_j (1 + e_j), |e_j| <= e, o moves by at most
  e sum p_j |v_j - o| (to first order; 1 + 2^-6 covers the rest);
* float32 sums over n keys are within (n + 64) 2^-24 sum p_j |v_j|;
* o is rounded once to its type (bf16 2^-8, float32 2^-24 of it).
"""
import math

import torch


def rows(q, K, V, seen, bf16):
    q, K, V = q.double(), K.double(), V.double()
    d = q.shape[1]
    w = q @ K.t() / math.sqrt(d)
    w = torch.where(seen, w, torch.full_like(w, -math.inf))
    lse = torch.logsumexp(w, 1)
    p = torch.where(seen, torch.exp(w - lse.clamp(min=-1e300)[:, None]), torch.zeros_like(w))
    o = p @ V
    T = p @ V.abs()
    S = torch.zeros_like(o)
    for r in range(q.shape[0]):
        S[r] = p[r] @ (V - o[r]).abs()
    size = torch.where(seen, q.abs() @ K.abs().t() / math.sqrt(d), torch.zeros_like(w))
    dl = (1.5 * (d + 8) * 2.0 ** -24 * (size.amax(1) if K.shape[0] else size.sum(1)) + 2.0 ** -22)[:, None]
    n = seen.sum(1)[:, None]
    e, out = (2.0 ** -8, 2.0 ** -8) if bf16 else (0.0, 2.0 ** -24)
    tol = (e + 2 * dl) * S * (1 + 2.0 ** -6) + (n + 64) * 2.0 ** -24 * T
    tol = tol + out * (o.abs() + tol) + 1e-30
    tol_lse = 2 * dl[:, 0] + (n[:, 0] + 64) * 2.0 ** -24 + 2.0 ** -22 * lse.abs()
    return o, lse, tol, tol_lse


def check(name, o, lse, q, K, V, seen):
    """o [R, d] and lse [R] of a kernel against the rows."""
    want, wl, tol, tl = rows(q, K, V, seen, q.dtype == torch.bfloat16)
    none = ~seen.any(1)
    assert torch.equal(torch.isneginf(lse), none), name
    assert not o[none].any(), name
    off = ((o.double() - want).abs() / tol)[~none]
    offl = ((lse.double() - wl).abs() / tl)[~none]
    worst = off.max().item() if off.numel() else 0.0
    worst_l = offl.max().item() if offl.numel() else 0.0
    print(name, "o %.2f lse %.2f of the bound" % (worst, worst_l), flush=True)
    assert worst <= 1 and worst_l <= 1, name


def ancestors(parents):
    """[t, t]: token i sees token j (itself and its ancestors), and depths."""
    t = len(parents)
    see, depth = torch.zeros((t, t), dtype=torch.bool), []
    for i, up in enumerate(parents):
        see[i, i] = True
        ok = -1 < up < i
        if ok:
            see[i] |= see[up]
        depth.append(depth[up] + 1 if ok else 0)
    return see, depth


def tree_seen(n, t, parents, window, n_sink):
    """[t, n]: what the t drafted tokens of a unit of n slots see (t may exceed n)."""
    see, depth = ancestors(parents[:t])
    base = n - t
    slot = torch.arange(n)
    pos = torch.tensor([j if j < base else base + depth[j - base] for j in range(n)], dtype=torch.long)
    out = torch.zeros((t, n), dtype=torch.bool)
    for i in range(t):
        out[i] = slot < base
        for j in range(t):
            if see[i, j] and 0 <= base + j < n:
                out[i, base + j] = True
        if window:
            out[i] &= (pos < n_sink) | (pos > base + depth[i] - window)
    return out


def sink_seen(n, nq, window, n_sink):
    pos = torch.arange(n - nq, n)[:, None]
    j = torch.arange(n)
    seen = j <= pos
    if window:
        seen &= (j < n_sink) | (j > pos - window)
    return seen
