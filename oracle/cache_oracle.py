"""Float64 CPU oracle for serving from a paged cache (admit, append, attend, evict).

TEST INFRASTRUCTURE ONLY, like compactor_oracle: it shares no code with the library, and each function is
written so that it can be checked against the definition by eye.  Everything is per head (eviction: per pool of
heads), on plain arrays indexed by logical slot; `there[s]` says whether the page of slot s exists.
"""
from __future__ import annotations

import numpy as np

__all__ = ["sees", "attend", "append", "rank_keys", "evict_keep", "evict_moves"]


def sees(count: int, new: int, T: int) -> list:
    """Slots that the queries of T rows see when the last `new` tokens of `count` are theirs: row t < new the
    first count - (new - 1 - t) slots, a padding row none."""
    return [max(0, count - (new - 1 - t)) if t < new else 0 for t in range(T)]


def attend(q, k, v, see, there, scale, cap):
    """One query row: q [d], the first `see` slots of k, v [n, d] that are there.
    -> (out [d], lse, p [n])."""
    n = k.shape[0]
    p = np.zeros(n)
    at = np.flatnonzero(there[:see])
    if len(at) == 0:
        return np.zeros(v.shape[1]), -np.inf, p
    x = scale * (k[at] @ q)
    if cap > 0:
        x = cap * np.tanh(x / cap)
    m = x.max()
    e = np.exp(x - m)
    p[at] = e / e.sum()
    return p[at] @ v[at], m + np.log(e.sum()), p


def append(count: int, seen: int, new: int, capacity: int):
    """-> ([(row, slot, position)], new count, new seen)"""
    rows = [(t, count + t, seen + t) for t in range(new) if count + t < capacity]
    return rows, min(count + new, capacity), seen + new


def rank_keys(mass, pos, there, seen: int, sink: int, recent: int):
    """What the slots of a head are ranked by, largest first: (class, mass), class 3 protected, 2 a number, 1 NaN, 0 a
    page that is not there."""
    keys = []
    for m, p, t in zip(mass, pos, there):
        if not t:
            keys.append((0, 0.0))
        elif p < sink or p >= seen - recent:
            keys.append((3, 0.0))
        elif np.isnan(m):
            keys.append((1, 0.0))
        else:
            keys.append((2, float(m)))
    return keys


def evict_keep(keys, budget: int):
    """keys: one list per head of the pool.  -> the slots that stay, ascending, per head."""
    flat = [(k, h, s) for h, head in enumerate(keys) for s, k in enumerate(head)]
    flat.sort(key=lambda x: (-x[0][0], -x[0][1], x[1], x[2]))
    stay = [[] for _ in keys]
    for _, h, s in flat[:max(0, budget)]:
        stay[h].append(s)
    return [sorted(x) for x in stay]


def evict_moves(stay, count: int):
    """-> [(to, from)]: retained slots from the new count on go to the slots below it that were given up."""
    left = len(stay)
    kept = set(stay)
    return list(zip([s for s in range(min(left, count)) if s not in kept], [s for s in stay if s >= left]))
