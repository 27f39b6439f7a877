"""Steps with drafted tokens in fp64 on the CPU (test infrastructure only): the
plan of a tree, verification by the rule that include/moe_offload.h states for
moe_verify_drafts, and keeping accepted entries."""
from __future__ import annotations

import numpy as np

MOST = 1024   # tokens of a sequence that take part


def tree(parents, first: int, words: int):
    """(pos, seen [n, n] bool) of one sequence's tree; seen as a token's words have it."""
    n = len(parents)
    pos, seen = np.full(n, -1), np.zeros((n, n), dtype=bool)
    depth = np.zeros(n, dtype=int)
    for i in range(min(n, 32 * words)):
        p = parents[i]
        if 0 <= p < i:
            depth[i] = depth[p] + 1
            seen[i] = seen[p]
        seen[i, i] = True
        pos[i] = first + depth[i]
    return pos, seen


def words_of(seen, words: int):
    """Bits of seen [n, m] as int32 [n, words]."""
    n = seen.shape[0]
    bits = np.zeros((n, 32 * words), dtype=bool)
    m = min(seen.shape[1], 32 * words)
    bits[:, :m] = seen[:, :m]
    return (bits.reshape(n, words, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)


def positive(x):
    """x where it is above 0, NaN kept."""
    return np.where(x <= 0, 0.0, x)


def verify(p, ids, parents, u, q=None):
    """(path, next) of one sequence: p [n, vocab], q the same or None, in fp64."""
    n, vocab = p.shape
    if n == 0:
        return [], -1
    u = np.fmax(np.asarray(u, dtype=np.float64), 0.0)
    path = [0]
    while True:
        at = path[-1]
        row, share, left, gone = p[at], 0.0, 1.0, []
        accepted = None
        for c in range(at + 1, min(n, MOST)):
            if parents[c] != at:
                continue
            x = ids[c]
            inside = 0 <= x < vocab
            if q is not None:
                if gone:
                    left = positive(row - share * q[at]).sum()
                weight = positive(row[x] - share * q[at, x]) if inside else 0.0
                guess = q[at, x] if inside else 0.0
                if u[c] * left * guess < weight:
                    accepted = c
                    break
                share += left
            else:
                weight = positive(row[x]) if inside and x not in gone else 0.0
                if u[c] * left < weight:
                    accepted = c
                    break
                left = positive(left - weight)
            gone.append(x)
        if accepted is None:
            break
        path.append(accepted)
    if q is not None:
        rest = positive(row - share * q[at]) if gone else positive(row)   # a row of q that drew nothing may hold anything
    else:
        rest = positive(row).copy()
        rest[[x for x in gone if 0 <= x < vocab]] = 0.0
    if rest.sum() == 0:
        rest = positive(row)
    total = rest.sum()
    if not (0 < total < np.inf):
        return path, -1
    over = np.flatnonzero((np.cumsum(rest) > u[0] * total) & (rest > 0))
    return path, int(over[0]) if over.size else int(np.flatnonzero(rest > 0)[-1])


def keep(pool, pages, base: int, n: int, path, count: int, P: int, D: int):
    """The pool's bytes with entries base + path[k] at places base + k, one
    sequence; entries are copied one after another, in order."""
    from . import attention as oa
    records = {}

    def entry(place):
        col = place // P
        page = pages[col] if place >= 0 and col < len(pages) else -1
        return (page, place % P) if 0 <= page < pool.shape[0] else None

    def parts(page, head):
        if (page, head) not in records:
            records[page, head] = [np.array(x) for x in oa.unpack_record(pool[page, head], P, D)]
        return records[page, head]

    for k in range(max(0, min(count, n))):
        if not k <= path[k] < n:
            continue
        source, to = entry(base + path[k]), entry(base + k)
        if source is None or to is None:
            continue
        for head in range(pool.shape[1]):
            for a, b in zip(parts(source[0], head), parts(to[0], head)):
                b[to[1]] = a[source[1]]
    for (page, head), rec in records.items():
        pool[page, head] = oa.record(*rec)
    return pool
