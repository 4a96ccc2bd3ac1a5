"""Plain oracle for the pages of caches (reserve, fork, release, compact), entry by entry on Python lists.  TEST INFRASTRUCTURE ONLY, like
cache_oracle.  tables [request][entry], refs [page], counts [request][list of heads] of 0 .. len(table) * page."""
from __future__ import annotations

__all__ = ["reserve", "fork", "release", "compact"]


def reserve(tables, refs, counts, new, page, own_all):
    """Changes tables and refs. -> (pairs, lacking)"""
    named, wants = {}, []
    for b, table in enumerate(tables):
        top, low = max(counts[b]), min(counts[b])
        holds, need = -(-top // page), min(-(-(top + new[b]) // page), len(table))
        first = 0 if own_all else low // page if new[b] > 0 else holds
        for i in range(first, need):
            p = table[i]
            if not 0 <= p < len(refs):
                if i >= holds:
                    wants.append((b, i, None))
            elif refs[p] > 1:
                named.setdefault(p, []).append((b, i))
                wants.append((b, i, p))
    keep = {entries[-1] for p, entries in named.items() if len(entries) == refs[p]}
    wants = [w for w in wants if w[:2] not in keep]
    free = [p for p, r in enumerate(refs) if r == 0]
    if len(free) < len(wants):
        return [], len(wants) - len(free)
    pairs = []
    for (b, i, old), p in zip(wants, free):
        tables[b][i] = p
        refs[p] = 1
        if old is not None:
            refs[old] -= 1
            pairs.append((old, p))
    return pairs, 0


def fork(tables, refs, state, parents):
    """state: lists per request that go along."""
    was = [list(t) for t in tables], [[list(x) for x in s] for s in state]
    for b, p in enumerate(parents):
        if not 0 <= p < len(tables):
            continue
        for i, page in enumerate(was[0][p]):
            old = tables[b][i]
            tables[b][i] = page
            if 0 <= page < len(refs):
                refs[page] += 1
            if 0 <= old < len(refs):
                refs[old] -= 1
        for s, w in zip(state, was[1]):
            s[b][:] = w[p]


def release(tables, refs, state, page, finished):
    """state: counts first."""
    for b, table in enumerate(tables):
        if finished[b]:
            for s in state:
                s[b][:] = [0] * len(s[b])
        for i in range(-(-max(state[0][b]) // page), len(table)):
            if 0 <= table[i] < len(refs):
                refs[table[i]] -= 1
                table[i] = -1


def compact(tables, refs):
    """-> (pairs, pages in use)"""
    used = [p for p, r in enumerate(refs) if r > 0]
    n = len(used)
    free = [p for p in range(n) if refs[p] <= 0]
    pairs = list(zip([p for p in reversed(used) if p >= n], free))
    to = dict(pairs)
    for table in tables:
        table[:] = [to.get(p, p) for p in table]
    for a, z in pairs:
        refs[a], refs[z] = 0, refs[a]
    return pairs, n
