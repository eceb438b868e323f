"""The plain forms of the cache's upkeep from call to call, without a GPU: forks of prefixes, cuts and ends in a window."""
import numpy as np
import pytest

from tests.pages_util import fork_plain, free_plain, holds, needs_lost


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5), (9, 0), (9, 33), (1, 0), (1, 20), (300, 4), (25, 60)])
@pytest.mark.parametrize("page", [1, 7, 16])
def test_forks_of_prefixes_keep_every_page_accounted_for(page, window, sinks):
    """A random run of new tokens, forks of every prefix whose pages are held, cuts and ends: a page's holders are the
    rows that hold it, pages without holders, and no others, are in the free list, and no held length is longer than
    its row."""
    rng = np.random.default_rng(page + window + sinks)
    R, columns = 6, -(-260 // page) + 1
    n_pages = R * columns
    table, seq, held = np.full((R, columns), -1, np.int64), np.zeros(R, np.int64), np.zeros(R, np.int64)
    free, head, shared = rng.permutation(n_pages), 0, np.zeros(n_pages, np.int64)

    def length(r):
        return int(rng.choice([n for n in range(int(seq[r]) + 1) if not needs_lost(n, held[r], page, window, sinks)]))

    def books():
        holders = np.zeros(n_pages, np.int64)
        for r in range(R):
            for j in range(-(-int(seq[r]) // page)):
                if holds(j, seq[r], held[r], page, window, sinks):
                    holders[table[r, j]] += 1
        assert np.array_equal(np.maximum(holders - 1, 0), shared)
        assert sorted(free[head:]) == sorted(np.flatnonzero(holders == 0))
        assert (held <= seq).all()

    for step in range(60):
        for r in range(R):  # new tokens, to rows whose last page is theirs alone
            n = int(rng.integers(0, 30))
            if seq[r] + n > 250 or (seq[r] % page and shared[table[r, seq[r] // page]]):
                continue
            for j in range(-(-int(seq[r]) // page), -(-(int(seq[r]) + n) // page)):
                table[r, j], head = free[head], head + 1
            seq[r] += n
        books()
        parents, empty = [r for r in range(R) if seq[r] > 0], [r for r in range(R) if seq[r] == 0]
        if parents and empty:
            p = [int(rng.choice(parents)) for _ in empty]
            n = [length(r) for r in p] if step % 2 else None
            table, seq, head, shared, _, _, held = fork_plain(p, empty, seq, table, free, head, page, shared, n, window,
                                                              sinks, held)
            books()
        new = np.where(rng.random(R) < 0.2, 0, seq)
        for r in range(R):
            n = length(r)
            if rng.random() < 0.2 and not (n % page and shared[table[r, n // page]]):
                new[r] = n
        free, head, shared = free_plain(seq, new, table, free, head, page, shared, window, sinks, held)
        seq, held = new, new.copy()
        books()


def test_which_lengths_need_a_page_let_go_of():
    """Pages of 16, a window of 40, 20 sinks (two pages), held at 100: pages 2 on page are gone up to page 2."""
    lost = [n for n in range(111) if needs_lost(n, 100, 16, 40, 20)]
    # page (100 - 40 + 1) // 16 = 3 is the first held behind the sinks', so page 2 is gone: needed by lengths that
    # reach into it and whose own window has not left it, (n - 39) // 16 < 3
    assert lost == list(range(33, 87))
    assert not any(needs_lost(n, 100, 16, 40, 48) for n in range(111))  # the sinks' three pages: nothing is gone
    assert not any(needs_lost(n, 100, 16, 0, 0) for n in range(111))
