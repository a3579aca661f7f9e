"""A paged cache's management in plain Python: refs, tables and lens as lists of integers, the pool as a NumPy array
[planes][pages][...]. Each call returns the bits that it adds to the status."""
from __future__ import annotations

BAD_INDEX, EXHAUSTED, BUSY = 1, 2, 4


def held(n, page):
    return -(-max(n, 0) // page)


def free_pages(refs):
    return [p for p, r in enumerate(refs) if r <= 0]


def grow(refs, tables, lens, new_lens, page):
    status, free = 0, free_pages(refs)
    for s, new in enumerate(new_lens):
        have, want = held(lens[s], page), held(new, page)
        if want > have and (want > len(tables[s]) or want - have > len(free)):
            status |= EXHAUSTED
            continue
        for e in range(have, want):
            tables[s][e] = free.pop(0)
            refs[tables[s][e]] = 1
        lens[s] = max(lens[s], new)
    return status


def fork(pool, refs, tables, lens, parents, children, page):
    status, free = 0, free_pages(refs)
    was_lens, was = list(lens), [list(t) for t in tables]
    seen = set()
    for p, c in zip(parents, children):
        ok_child = 0 <= c < len(lens)
        twice = c in seen
        if ok_child:
            seen.add(c)
        if not ok_child or not 0 <= p < len(lens):
            status |= BAD_INDEX
            continue
        if was_lens[c] > 0 or twice:
            status |= BUSY
            continue
        n = max(was_lens[p], 0)
        full = n // page
        last = None
        if n % page:
            last = was[p][full] if full < len(was[p]) else -1
            if not 0 <= last < len(refs):
                status |= BAD_INDEX
                continue
            if not free:
                status |= EXHAUSTED
                continue
        for e in range(min(full, len(was[p]))):
            tables[c][e] = was[p][e]
            if 0 <= was[p][e] < len(refs):
                refs[was[p][e]] += 1
            else:
                status |= BAD_INDEX
        if last is not None:
            to = free.pop(0)
            tables[c][full] = to
            refs[to] = 1
            pool[:, to] = pool[:, last]
        lens[c] = n
    return status


def free(refs, tables, lens, slots, page):
    status = 0
    for s in slots:
        if not 0 <= s < len(lens):
            status |= BAD_INDEX
            continue
        for e in range(min(held(lens[s], page), len(tables[s]))):
            if 0 <= tables[s][e] < len(refs):
                refs[tables[s][e]] -= 1
            else:
                status |= BAD_INDEX
        lens[s] = 0
    return status


def compact(pool, refs, tables, lens, page):
    """Returns (status, refs, tables, used)."""
    used = [p for p, r in enumerate(refs) if r > 0]
    u = len(used)
    to = dict(zip([p for p in used if p >= u], [p for p in range(u) if refs[p] <= 0]))
    out_refs, out_tables, status = list(refs), [list(t) for t in tables], 0
    for a, b in to.items():
        pool[:, b] = pool[:, a]
        out_refs[b], out_refs[a] = refs[a], 0
    for s, n in enumerate(lens):
        for e in range(min(held(n, page), len(tables[s]))):
            if not 0 <= tables[s][e] < len(refs):
                status |= BAD_INDEX
            else:
                out_tables[s][e] = to.get(tables[s][e], tables[s][e])
    return status, out_refs, out_tables, u
