"""Oracle of the calls on the cache's pages: rows of a table forked with copy-on-write, a pool compacted.

TEST INFRASTRUCTURE ONLY (see kvprm_oracle). Tables are lists of lists (a row's held pages), and a call
returns what it does to them and which pages are copied.
"""
from __future__ import annotations

PAGE = 16


def fork(rows, lengths, parent, room, refs, to_pages):
    """rows: held pages of each row. Returns (status, new rows, new lengths, new refs, copies [(source, to)],
    fresh pages needed, pages there were)."""
    refs = list(refs)
    before = list(refs)
    bad = (2, None, None, None, None, 0, 0)
    for row in rows:
        for p in row:
            if not 0 <= p < len(refs):
                return bad
            refs[p] -= 1
    if any(r < 0 for r in refs):
        return bad
    seen, plans = set(), []
    for i, p in enumerate(parent):
        if p >= len(rows) or room[i] < 0:
            return bad
        n = lengths[p] if p >= 0 else 0
        if p >= 0 and not 0 <= n <= PAGE * len(rows[p]):
            return bad
        want = -(-(n + room[i]) // PAGE)
        if want > to_pages:
            return bad
        kept, copy = (list(rows[p][:n // PAGE]) if p >= 0 else []), None
        if n % PAGE:
            last = rows[p][n // PAGE]
            if p not in seen and before[last] == 1:
                kept.append(last)
            else:
                copy = last
        seen.add(p)
        for q in kept:
            refs[q] += 1
        plans.append((n, kept, want, copy))
    sources = {c for _, _, _, c in plans if c is not None}
    free = [q for q in range(len(refs)) if refs[q] == 0 and q not in sources]
    need = sum(want - len(kept) for _, kept, want, _ in plans)
    if need > len(free):
        return 1, None, None, None, None, need, len(free)
    fresh, out, copies = iter(free), [], []
    for n, kept, want, copy in plans:
        new = [next(fresh) for _ in range(want - len(kept))]
        for q in new:
            refs[q] += 1
        if copy is not None:
            copies.append((copy, new[0]))
        out.append(kept + new)
    return 0, out, [n for n, _, _, _ in plans], refs, copies, need, len(free)


def compact(rows, refs):
    """Returns (status, new rows, new refs, moved: every page's new id or -1, copies [(source, to)])."""
    if any(r < 0 for r in refs) or any(not 0 <= p < len(refs) or refs[p] <= 0 for row in rows for p in row):
        return 2, None, None, None, None
    live = [p for p, r in enumerate(refs) if r > 0]
    holes = [p for p in range(len(live)) if refs[p] == 0]
    far = [p for p in live if p >= len(live)]
    copies = list(zip(far, holes))
    moved = [p if r > 0 else -1 for p, r in enumerate(refs)]
    for src, to in copies:
        moved[src] = to
    new = [0] * len(refs)
    for p in live:
        new[moved[p]] = refs[p]
    return 0, [[moved[p] for p in row] for row in rows], new, moved, copies
