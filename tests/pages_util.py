"""The upkeep of the cache's pages one page and one token at a time."""
import numpy as np


def left(n, page, window):
    """The first page that the window of token n needs."""
    return max(0, n - window + 1) // page if window else 0


def holds(j, n, held, page, window=0, sinks=0):
    return j < -(-n // page) and (j < -(-sinks // page) or j >= left(held, page, window))


def needs_lost(n, held, page, window=0, sinks=0):
    """Whether n tokens need a page that a request held at `held` tokens has let go of."""
    many = max(n, held) + page
    return any(holds(j, n, n, page, window, sinks) and not holds(j, many, held, page, window, sinks)
               for j in range(-(-n // page)))


def free_plain(seq, new, table, free, head, page, shared=None, window=0, sinks=0, held=None):
    """avtp_cache_free: (free, head, shared)."""
    free, gone = free.copy(), []
    shared = None if shared is None else shared.copy()
    for r in range(len(seq)):
        h = 0 if held is None else int(held[r])
        for j in range(-(-int(seq[r]) // page)):
            if holds(j, seq[r], h, page, window, sinks) and not (
                    new[r] > 0 and holds(j, new[r], new[r], page, window, sinks)):
                p = int(table[r, j])
                if shared is not None and shared[p] > 0:
                    shared[p] -= 1
                else:
                    gone.append(p)
    head -= len(gone)
    free[head:head + len(gone)] = gone
    return free, head, shared


def fork_plain(parent, child, seq, table, free, head, page, shared, length=None, window=0, sinks=0, held=None):
    """avtp_cache_fork: (table, seq, head, shared, src, dst, held)."""
    table, seq, shared = table.copy(), seq.copy(), shared.copy()
    held = None if held is None else held.copy()
    src, dst = np.full(len(parent), -1, np.int32), np.full(len(parent), -1, np.int32)
    for i, (p, c) in enumerate(zip(parent, child)):
        n = int(seq[p] if length is None else length[i])
        for j in range(n // page):
            if holds(j, n, 0 if held is None else held[p], page, window, sinks):
                table[c, j] = table[p, j]
                shared[table[p, j]] += 1
        if n % page:
            src[i], dst[i] = table[p, n // page], free[head]
            table[c, n // page] = free[head]
            head += 1
        seq[c] = n
        if held is not None:
            held[c] = min(held[p], n)
    return table, seq, head, shared, src, dst, held


def compact_plain(pool, keep_cu, keep, table, dst_table, page, base=None):
    """avtp_cache_compact on one pool [n_pages, page, ...], token by token: the pool."""
    pool = pool.copy()
    for r in range(len(keep_cu) - 1):
        for j, i in enumerate(range(int(keep_cu[r]), int(keep_cu[r + 1]))):
            p = int(keep[i]) - (0 if base is None else int(base[r]))
            pool[dst_table[r, j // page], j % page] = pool[table[r, p // page], p % page]
    return pool
