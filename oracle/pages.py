"""Blocks of the paged cache shared, freed and moved (oracle).

Test infrastructure: see the package docstring.  Not in the paper ("parity unpinned").
Arrays are changed in place; every function returns the device flags that the call
raises.  `pools` are arrays indexed by block first (caches, scales, mean keys).
"""
from __future__ import annotations

import numpy as np

BS = 16
BAD_TABLE, BAD_CTXLEN, CACHE_FULL, BAD_ROW = 1, 2, 4, 16


def _range_ok(free, n_ids):
    return 0 <= free[0] <= free[1] <= n_ids


def fork(src, dst, tables, ctx, shared, ids, free, P: int, pools=()):
    """See ent_cache_fork."""
    R, maxb = tables.shape
    if not _range_ok(free, len(ids)):
        return BAD_TABLE | (BAD_ROW if _fork_rows(src, dst, R)[1] else 0) | _fork_lens(src, dst, ctx, R, maxb)
    go, bad = _fork_rows(src, dst, R)
    flags = (BAD_ROW if bad else 0) | _fork_lens(src, dst, ctx, R, maxb)
    at, end = int(free[0]), int(free[1])
    for i in go:
        s, d = int(src[i]), int(dst[i])
        n = int(ctx[s])
        if not 0 <= n <= maxb * BS:
            continue
        if n % BS and at == end:
            flags |= CACHE_FULL
            break
        full = n // BS
        for j in range(full):
            p = int(tables[s, j])
            tables[d, j] = p
            if 0 <= p < P:
                shared[p] += 1
            else:
                flags |= BAD_TABLE
        if n % BS:
            p, new = int(tables[s, full]), int(ids[at])
            at += 1
            ok, there = 0 <= new < P, 0 <= p < P
            tables[d, full] = new if ok else -1
            if ok and there:
                for x in pools:
                    x[new] = x[p]
            else:
                flags |= BAD_TABLE
        ctx[d] = n
    free[0] = at
    return flags


def _fork_rows(src, dst, R):
    """Forks whose rows are good, and whether some are not."""
    from_, seen, go = {int(s) for s in src}, set(), []
    for i, (s, d) in enumerate(zip(src, dst)):
        s, d = int(s), int(d)
        if 0 <= s < R and 0 <= d < R and d not in seen and d not in from_:
            go.append(i)
        seen.add(d)
    return go, len(go) < len(src)


def _fork_lens(src, dst, ctx, R, maxb):
    return BAD_CTXLEN if any(not 0 <= int(ctx[int(src[i])]) <= maxb * BS
                             for i in _fork_rows(src, dst, R)[0]) else 0


def release(rows, tables, ctx, shared, ids, free, P: int):
    """See ent_cache_release (shared may be None)."""
    R, maxb = tables.shape
    if not _range_ok(free, len(ids)):
        return BAD_TABLE
    flags, held = 0, {}
    seen = set()
    for r in rows:
        r = int(r)
        if not 0 <= r < R or r in seen:
            flags |= BAD_ROW
            continue
        seen.add(r)
        n = int(ctx[r])
        if not 0 <= n <= maxb * BS:
            flags |= BAD_CTXLEN
            continue
        for j in range(-(-n // BS)):
            p = int(tables[r, j])
            if 0 <= p < P:
                held[p] = held.get(p, 0) + 1
            else:
                flags |= BAD_TABLE
        ctx[r] = 0
    gone = []
    for p, k in sorted(held.items()):
        others = 0 if shared is None else int(shared[p])
        if k > others + 1:
            flags |= BAD_TABLE
        if k > others:
            gone.append(p)
        if shared is not None:
            shared[p] = max(others - k, 0) if k <= others else 0
    if len(gone) > free[0]:
        flags |= CACHE_FULL
        gone = gone[len(gone) - int(free[0]):]
    free[0] -= len(gone)
    ids[free[0]:free[0] + len(gone)] = gone
    return flags


def compact(tables, ctx, shared, ids, free, P: int, pools=()):
    """See ent_cache_compact: (flags, blocks in use)."""
    R, maxb = tables.shape
    flags, held = 0, {}
    rows = []
    for r in range(R):
        n = int(ctx[r])
        if not 0 <= n <= maxb * BS:
            flags |= BAD_CTXLEN
            continue
        rows.append((r, -(-n // BS)))
        for j in range(rows[-1][1]):
            p = int(tables[r, j])
            if 0 <= p < P:
                held[p] = held.get(p, 0) + 1
            else:
                flags |= BAD_TABLE
    U = len(held)
    place = dict(zip(sorted(p for p in held if p >= U), (p for p in range(U) if p not in held)))
    for a, b in place.items():
        for x in pools:
            x[b] = x[a]
    if shared is not None:
        shared[:] = 0
        for p, n in held.items():
            shared[place.get(p, p)] = n - 1
    for r, nb in rows:
        for j in range(nb):
            tables[r, j] = place.get(int(tables[r, j]), tables[r, j])
    first = len(ids) - (P - U)
    ids[first:] = np.arange(U, P)
    free[0], free[1] = first, len(ids)
    return flags, U
