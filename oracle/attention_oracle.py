"""float64 statement of attention over a key/value cache with a sliding window and always-visible first positions, of
the attention weight the entries receive, and of the eviction by it (numpy; test infrastructure only).

An entry at position p is visible to a query at position s if p <= s and (window == 0 or s - p < window or p < n_sink).
"""
from __future__ import annotations

import numpy as np


def visible(p, s, window: int, n_sink: int):
    """[queries, entries] truth table from entry positions p and query positions s."""
    p, s = np.asarray(p, np.int64)[None, :], np.asarray(s, np.int64)[:, None]
    ok = p <= s
    if window:
        ok = ok & ((s - p < window) | (p < n_sink))
    return ok


def attend(q, k, v, p, s, window: int, n_sink: int, scale: float):
    """One head: q [T, D] at positions s, k, v [n, D] at positions p (float64).

    Returns out [T, D], lse [T], w [T, n] (softmax weights, 0 where hidden), reach [T, D] = sum_j w_j |v_j| and
    size [T] = the largest sum_c |q_c k_jc| * |scale| over visible entries (what rounding errors scale with)."""
    ok = visible(p, s, window, n_sink)
    out, reach = np.zeros(q.shape), np.zeros(q.shape)
    lse, w, size = np.full(len(q), -np.inf), np.zeros((len(q), len(k))), np.zeros(len(q))
    for i in range(len(q)):
        see = np.nonzero(ok[i])[0]
        if len(see) == 0:
            continue
        x = k[see] @ q[i] * scale
        top = x.max()
        e = np.exp(x - top)
        lse[i] = top + np.log(e.sum())
        w[i, see] = e / e.sum()
        out[i] = w[i, see] @ v[see]
        reach[i] = w[i, see] @ np.abs(v[see])
        size[i] = (np.abs(k[see]) @ np.abs(q[i])).max() * abs(scale)
    return out, lse, w, reach, size


def evict(weight, p, last: int, budget: int, n_sink: int, n_recent: int):
    """One head with n entries: source slot of every slot 0 .. budget-1 (-1: nothing).

    Kept: protected positions, then the largest weights (NaN below every number), ties to the lower slot.  Kept slots
    below the budget stay; the others go to the freed slots, both in ascending order."""
    n = len(weight)
    src = np.full(budget, -1, np.int64)
    if n <= budget:
        src[:n] = np.arange(n)
        return src
    def order(j):
        held = p[j] < n_sink or p[j] > last - n_recent
        x = float(weight[j])
        return (0 if held else 1, 0.0 if held else (np.inf if np.isnan(x) else -x), (not held) and np.isnan(x), j)
    kept = sorted(sorted(range(n), key=order)[:budget])
    stay = [j for j in kept if j < budget]
    src[stay] = stay
    freed = [j for j in range(budget) if src[j] < 0]
    for slot, j in zip(freed, [j for j in kept if j >= budget]):
        src[slot] = j
    return src
