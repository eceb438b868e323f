"""What one call of the cache's upkeep leaves is what the next one takes: lengths, held lengths and pages from call to
call, on the GPU, against the plain forms one page and one token at a time."""
import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.cache_util import pool
from tests.gpu_util import ensure_built
from tests.pages_util import fork_plain, free_plain, holds, needs_lost
from tests.test_gpu_cache_pages import BAD_IN_PLACE, Compacted, Forked, Freed, i32, ints, refused, status

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


# ---------------------------------------------------------------- forks of prefixes in a window
class Books:
    """A table's numbers on the device and in the plain forms, call after call."""

    def __init__(self, f):
        f.call()
        self.f, self.d = f, f.dev
        self.seq, self.table, self.free, self.shared, self.held = (
            np.array(x) for x in (f.seq, f.table, f.free, f.shared, f.held))
        self.head = f.head
        self.more = dict(page_size=f.page, n_pages=f.n_pages, free_pages=self.d["free"], free_head=self.d["head"],
                         shared=self.d["shared"], window=f.window, sinks=f.sinks, held_len=self.d["held"],
                         free_head_out=self.d["head"])

    def fork(self, parent, child, length=None):
        f, d = self.f, self.d
        c = avtp.CacheForkCall(i32(parent), i32(child), d["seq"], d["table"],
                               fork_len=None if length is None else i32(length), **self.more).run()
        self.table, self.seq, self.head, self.shared, src, dst, self.held = fork_plain(
            parent, child, self.seq, self.table, self.free, self.head, f.page, self.shared, length, f.window, f.sinks,
            self.held)
        assert status(c) == avtp.OK
        assert np.array_equal(ints(c.copy_src), src) and np.array_equal(ints(c.copy_dst), dst)
        self.agree()

    def go_on(self, new):
        f, d = self.f, self.d
        c = avtp.CacheFreeCall(d["seq"], i32(new), d["table"], seq_len_out=d["seq"], held_len_out=d["held"],
                               **self.more).run()
        self.free, self.head, self.shared = free_plain(self.seq, new, self.table, self.free, self.head, f.page, self.shared,
                                                       f.window, f.sinks, self.held)
        self.seq, self.held = np.array(new), np.array(new)
        assert status(c) == avtp.OK
        self.agree()

    def agree(self):
        d = self.d
        for name in ("seq", "table", "shared", "held", "free"):
            assert np.array_equal(ints(d[name]), getattr(self, name)), name
        assert int(d["head"]) == self.head and (self.held <= self.seq).all()
        holders = np.zeros(self.f.n_pages, dtype=np.int64)
        for r, n in enumerate(self.seq):
            for j in range(-(-int(n) // self.f.page)):
                if holds(j, n, self.held[r], self.f.page, self.f.window, self.f.sinks):
                    holders[self.table[r, j]] += 1
        assert np.array_equal(np.maximum(holders - 1, 0), self.shared)


PREFIXES = {  # parents' lengths, held lengths, the prefix of the first, window, sinks
    "window_not_full": ([100, 50], [100, 50], 60, 1024, 0),
    "one_token": ([100, 50], [100, 50], 1, 1024, 4),
    "nothing": ([100, 50], [100, 50], 0, 1024, 4),
    "within_a_page": ([100, 50], [100, 50], 99, 30, 0),
    "behind_what_is_held": ([120, 50], [100, 50], 110, 30, 20),
}


@pytest.mark.parametrize("page", [1, 7, 16])
@pytest.mark.parametrize("name", PREFIXES)
def test_a_forked_prefix_goes_on_is_forked_and_ends(name, page):
    seq, held, n, window, sinks = PREFIXES[name]
    if needs_lost(n, held[0], page, window, sinks):
        n = next(m for m in range(n, seq[0] + 1) if not needs_lost(m, held[0], page, window, sinks))
    b = Books(Forked(seq, [], [], page, rows=5, window=window, sinks=sinks, held=held, spare=20))
    b.fork([0], [2], [n])
    b.go_on([seq[0], seq[1], n, 0, 0])  # a step of the batch with the child in it
    b.fork([2], [3], [n])
    b.fork([3], [4])                    # a child as a parent, ahead of any step
    b.go_on([0, seq[1], n, 0, n])       # and its end
    b.go_on([0, seq[1], 0, 0, n])
    b.go_on([0, 0, 0, 0, 0])
    assert (b.shared == 0).all()


# ---------------------------------------------------------------- lengths whose pages are all held
LENGTHS = [(40, 20), (40, 33), (9, 60), (1, 0), (1, 17), (30, 110), (200, 5)]  # window, sinks


@pytest.mark.parametrize("page", [1, 7, 16])
@pytest.mark.parametrize("window,sinks", LENGTHS)
def test_free_takes_every_length_whose_pages_are_held(window, sinks, page):
    seq, held = 110, 100
    lost = [n for n in range(seq + 1) if needs_lost(n, held, page, window, sinks)]
    fine = [n for n in range(seq + 1) if n not in lost]
    f = Freed([seq] * len(fine), fine, page, window=window, sinks=sinks, held=[held] * len(fine))
    f.check(f.call().run())
    for n in lost[:1] + lost[-1:]:
        refused(Freed([seq, 50], [n, 50], page, window=window, sinks=sinks, held=[held, 0]))


@pytest.mark.parametrize("page", [1, 7, 16])
@pytest.mark.parametrize("window,sinks", LENGTHS)
def test_fork_takes_every_length_whose_pages_are_held(window, sinks, page):
    seq, held = 110, 100
    lost = [n for n in range(seq + 1) if needs_lost(n, held, page, window, sinks)]
    fine = [n for n in range(seq + 1) if n not in lost]
    at = dict(window=window, sinks=sinks, held=[held])
    f = Forked([seq], [0] * len(fine), list(range(1, len(fine) + 1)), page, length=fine, **at)
    f.check(f.call().run())
    for n in lost[:1] + lost[-1:]:
        c = Forked([seq], [0], [1], page, length=[n], **at).call().run()
        assert status(c) == avtp.ERR_DEVICE_INPUT and int(c.free_head_out) == -1


def test_a_prompt_kept_as_sinks_is_forked_and_a_request_cut_back_to_it():
    b = Books(Forked([500, 300], [], [], 16, rows=5, window=64, sinks=40, held=[500, 300], spare=10))
    b.fork([0, 1], [2, 3], [40, 48])
    b.go_on([32, 300, 40, 48, 0])
    b.fork([0], [4], [32])
    b.go_on([0, 48, 40, 0, 32])
    b.go_on([0, 0, 0, 0, 0])
    assert (b.shared == 0).all()


# ---------------------------------------------------------------- compaction in place, then the pages behind it
def refused_ones(name):
    """A request with a fault, one that is moved and one of which nothing is kept; and what the call is told more."""
    keep = list(range(3, 90, 3)) + [99]
    c, more = Compacted([100, 60, 40], [keep, 20, 0], 16, other=False), {}
    if name in BAD_IN_PLACE:
        BAD_IN_PLACE[name](c)
    elif name == "shared":
        shared = np.zeros(c.n_pages, dtype=np.int32)
        shared[c.table[0, 1]] = 1
        more = dict(shared=i32(shared))
    elif name == "let_go":
        c = Compacted([100, 60, 40], [list(range(1, 16)) + list(range(70, 80)), [1, 40], 0], 16, other=False)
        more = dict(window=32, sinks=16, held_len=i32([100, 60, 40]))
    return c, more


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("name", list(BAD_IN_PLACE) + ["shared", "let_go"])
def test_a_request_that_is_not_moved_keeps_its_length_and_its_pages(name, captured):
    """The lengths that a compaction gives go to the free without a look at the status between them."""
    c, more = refused_ones(name)
    kept = c.call(len_out=torch.full((3,), -7, dtype=torch.int32, device="cuda"), **more)
    free = np.arange(-40, 0)
    seq, lst, head = i32(c.seq), i32(free), i32([30])
    given = avtp.CacheFreeCall(seq, kept.len_out, kept._keep[3], page_size=16, n_pages=c.n_pages, free_pages=lst,
                               free_head=head, **{k: v for k, v in more.items() if k != "shared"})
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept.run()
            given.run()
        graph.replay()
        torch.cuda.synchronize()
    else:
        kept.run()
        given.run()
    n = [100, int(c.cu[2] - c.cu[1]), 0]
    assert status(kept) == avtp.ERR_DEVICE_INPUT and ints(kept.len_out).tolist() == n
    want, h, _ = free_plain(c.seq, n, c.table, free, 30, 16, None, *(
        (32, 16, [100, 60, 40]) if name == "let_go" else ()))
    assert status(given) == avtp.OK and np.array_equal(ints(lst), want) and int(given.free_head_out) == h
    assert c.same(c.want(rows=[1]))


@pytest.mark.parametrize("R", [40, 400, 1100])
def test_lengths_of_many_requests_of_which_some_are_not_moved(R):
    rng = np.random.default_rng(R)
    c = Compacted([20 + i % 9 for i in range(R)], [int(k) for k in rng.integers(0, 8, R)], 4, other=False, seed=R)
    n = np.diff(c.cu)
    wrong = [r for r in range(R) if n[r] > 1 and r % 3 == 0]
    for r in wrong:
        c.idx[c.cu[r + 1] - 1] = c.idx[c.cu[r]]
    call = c.call().run()
    want = np.where(np.isin(np.arange(R), wrong), c.seq, n)
    assert status(call) == avtp.ERR_DEVICE_INPUT and np.array_equal(ints(call.len_out), want)
    assert c.same(c.want(rows=[r for r in range(R) if r not in wrong]))


# ---------------------------------------------------------------- tokens that stay where they are
def test_kept_tokens_that_stay_are_looked_at_too():
    """On a page let go of, or outside the pool, a token cannot be kept, moved or not."""
    more = dict(window=32, sinks=16, held_len=i32([100, 60]))
    c = Compacted([100, 60], [list(range(21)), [1, 40]], 16, other=False)
    call = c.call(**more).run()
    assert status(call) == avtp.ERR_DEVICE_INPUT and ints(call.len_out).tolist() == [100, 2] and c.same(c.want(rows=[1]))
    c = Compacted([100, 60], [list(range(16)), [1, 40]], 16, other=False)
    call = c.call(**more).run()
    assert status(call) == avtp.OK and ints(call.len_out).tolist() == [16, 2] and c.same(c.want(rows=[1]))
    for page in (-1, 10 ** 6):
        c = Compacted([100, 60], [list(range(40)) + [60, 99], 20], 16, other=False)
        c.table[0, 1] = page
        call = c.call().run()
        assert status(call) == avtp.ERR_DEVICE_INPUT and ints(call.len_out).tolist() == [100, 20]
        assert c.same(c.want(rows=[1]))


# ---------------------------------------------------------------- pages that are let go of twice
def twice(f, a, b):
    f.table[b] = f.table[a]
    return f


REPEATED = {
    "two_rows": lambda: twice(Freed([100, 90], [0, 0], 16), (0, 2), (1, 4)),
    "one_row": lambda: twice(Freed([100, 90], [100, 0], 16), (1, 0), (1, 5)),
    "behind_cuts": lambda: twice(Freed([100, 90], [30, 40], 16), (0, 3), (1, 3)),
    "two_windows": lambda: twice(Freed([300, 290], [300, 290], 16, window=40, sinks=5, held=[200, 0]), (0, 10), (1, 4)),
    "many_rows": lambda: twice(Freed([17] * 2500, [0] * 2500, 16), (0, 1), (2499, 0)),
    "many_pages": lambda: twice(Freed([1200000, 40], [0, 0], 16), (0, 70000), (0, 3)),
}


@pytest.mark.parametrize("name", REPEATED)
def test_without_counts_a_page_let_go_of_twice_is_refused(name):
    refused(REPEATED[name]())


def test_without_counts_a_page_that_another_row_keeps_is_let_go_of_once():
    f = twice(Freed([100, 90], [0, 90], 16), (0, 2), (1, 4))
    f.check(f.call().run())


POOLS = [12288, 12289, 3 * 12288, 16 * 12288 + 1, 32 * 12288, 32 * 12288 + 1, 32 * 12288 * 16, 32 * 12288 * 16 + 1]


@pytest.mark.parametrize("n_pages", POOLS)
@pytest.mark.parametrize("case", [([100, 90, 5], [0, 40, 5]), ([9000] * 40, [0, 9000] * 20), ([17] * 2500, [0] * 2500)])
def test_repeated_pages_of_large_pools(n_pages, case):
    """Pages all over pools of as many pages as a cluster of one CTA, or of sixteen, has words or bits for, and of one more.
    (The second case has 22520 pages in use.)"""
    f = Freed(*case, 16)
    n_pages = max(n_pages, f.n_pages)
    ids = np.sort(np.random.default_rng(n_pages).choice(n_pages, f.n_pages, replace=False))
    ids[0], ids[-1] = 0, n_pages - 1
    f.table[f.table >= 0] = ids[f.table[f.table >= 0]]
    f.n_pages = n_pages
    f.check(f.call().run())
    last = -(-case[0][0] // 16) - 1
    f.table[0, last] = f.table[0, 0]
    refused(f)
    f.table[0, last] = n_pages
    refused(f)


# ---------------------------------------------------------------- kept tokens that end in a page of several holders
@pytest.mark.parametrize("n,ok", [(40, False), (33, False), (47, False), (32, True), (48, True), (60, True), (100, True)])
def test_kept_tokens_may_not_end_inside_a_page_that_others_hold(n, ok):
    """A request's next token would be written over theirs; the free refuses such a length, with its whole batch."""
    c = Compacted([100, 60], [list(range(n)), 20], 16, other=False)
    shared = np.zeros(c.n_pages, dtype=np.int32)
    shared[c.table[0, :3]] = 1
    call = c.call(shared=i32(shared)).run()
    want = [n if ok else 100, 20]
    assert status(call) == (avtp.OK if ok else avtp.ERR_DEVICE_INPUT) and ints(call.len_out).tolist() == want
    assert c.same(c.want(rows=[1]))
    free = np.arange(-40, 0)
    counts, lst = i32(shared), i32(free)
    given = avtp.CacheFreeCall(i32(c.seq), call.len_out, i32(c.table), page_size=16, n_pages=c.n_pages, free_pages=lst,
                               free_head=i32([30]), shared=counts).run()
    f, h, s = free_plain(c.seq, want, c.table, free, 30, 16, shared)
    assert status(given) == avtp.OK and np.array_equal(ints(lst), f) and int(given.free_head_out) == h
    assert np.array_equal(ints(counts), s)


# ---------------------------------------------------------------- together
def may_stay(r, keep, seq, table, shared, held, page, window, sinks):
    """Whether avtp_cache_compact moves these tokens together in place."""
    def held_page(p):
        return holds(p // page, seq[r], held[r], page, window, sinks)

    n = len(keep)
    if not all(held_page(p) for p in keep):
        return False
    if any(j != p and (not held_page(j) or shared[table[r, j // page]] > 0) for j, p in enumerate(keep)):
        return False
    return not (n < seq[r] and n % page and shared[table[r, n // page]] > 0)


@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 5), (40, 40), (500, 16), (9, 70)])
@pytest.mark.parametrize("page", [4, 16])
def test_a_run_with_prefixes_cuts_and_compactions(page, window, sinks):
    """Steps of a serving program, every number on the device and no look at a status between the calls: new tokens, forks
    of prefixes, selections in place (some of them refused), cuts and ends. The books agree with the plain forms', and
    every token that is held is found where the table says."""
    rng = np.random.default_rng(page + window + sinks)
    R, most = 10, 300
    columns = -(-(most + 40) // page)
    n_pages = R * columns + 8
    k, v = pool(n_pages, page, 1, 64, fill=0.0)
    cache = avtp.PagedCache(k, v)
    table = i32(np.full((R, columns), -1))
    seq, held, head = i32(np.zeros(R)), i32(np.zeros(R)), i32([0])
    free, shared = i32(rng.permutation(n_pages)), i32(np.zeros(n_pages))
    more = dict(window=window, sinks=sinks, held_len=held) if window else {}
    tokens, stamp, refusals = [[] for _ in range(R)], 0, 0

    def books():
        h = ints(held) if window else np.zeros(R, np.int64)
        return ints(seq).copy(), ints(table).copy(), ints(free).copy(), int(head), ints(shared).copy(), h.copy()

    for step in range(30):
        lens = np.asarray([len(t) for t in tokens])
        new = np.where((lens > 0) | (rng.random(R) < 0.4), rng.integers(0, 40, R), 0)
        new = np.where(lens + new > most, 0, new)
        cu = np.concatenate([[0], np.cumsum(new)])
        slots = avtp.cache_slots(i32(cu), int(cu[-1]), page_size=page, n_pages=n_pages, block_table=table, free_pages=free,
                                 free_head=head, past_len=seq, seq_len=seq, free_head_out=head)[0]
        marks = (stamp + torch.arange(int(cu[-1])) % 250).float()
        stamp = (stamp + 7) % 100
        rows = (marks[:, None, None] * torch.ones(len(marks), 1, 64)).bfloat16().cuda()
        avtp.cache_write(cache, slots, rows, rows)
        flat = rows[:, 0, 0].float().cpu().tolist()
        for r in range(R):
            tokens[r] += flat[cu[r]:cu[r + 1]]
        # forks, of prefixes in every second step
        s, t, f, h, n_shared, hl = books()
        empty, parents = [r for r in range(R) if s[r] == 0], [r for r in range(R) if s[r] > 0]
        if empty and parents:
            p = [int(rng.choice(parents)) for _ in empty]
            n = [int(rng.choice([m for m in range(s[r] + 1) if not needs_lost(m, hl[r], page, window, sinks)])) for r in p]
            n = n if step % 2 else None
            src, dst, _ = avtp.cache_fork(i32(p), i32(empty), seq, table, page_size=page, n_pages=n_pages, free_pages=free,
                                          free_head=head, shared=shared, free_head_out=head,
                                          fork_len=None if n is None else i32(n), **more)
            avtp.cache_copy(cache, src, dst)
            want = fork_plain(p, empty, s, t, f, h, page, n_shared, n, window, sinks, hl if window else None)
            got = books()
            assert np.array_equal(got[1], want[0]) and np.array_equal(got[0], want[1]) and got[3] == want[2]
            assert np.array_equal(got[4], want[3]) and (not window or np.array_equal(got[5], want[6]))
            for i, (a, b) in enumerate(zip(p, empty)):
                tokens[b] = tokens[a][:len(tokens[a]) if n is None else n[i]]
        # selections in place, and what they leave goes back
        s, t, f, h, n_shared, hl = books()
        keep = []
        for r in range(R):
            mine = list(range(s[r]))
            if s[r] and rng.random() < 0.3:
                fixed = int(rng.integers(0, s[r] + 1)) if rng.random() < 0.7 else 0
                mine = [j for j in mine if holds(j // page, s[r], hl[r], page, window, sinks) or rng.random() < 0.02]
                mine = [j for i, j in enumerate(mine) if j == i and j < fixed or rng.random() < 0.5]
            else:
                mine = mine if all(holds(j // page, s[r], hl[r], page, window, sinks) for j in mine) else None
            keep.append(mine)
        lens = np.asarray([s[r] if keep[r] is None or not may_stay(r, keep[r], s, t, n_shared, hl, page, window, sinks)
                           else len(keep[r]) for r in range(R)])
        # (a row that has let go of pages and is to stay as it is names a token of such a page)
        named = [list(range(s[r])) if keep[r] is None else keep[r] for r in range(R)]
        kept = avtp.CacheCompactCall(cache, i32(np.cumsum([0] + [len(x) for x in named])),
                                     i32(np.concatenate(named + [[0]])), seq, table, shared=shared, **more).run()
        ends = rng.random(R) < 0.1
        given = kept.len_out * i32(~ends)
        avtp.CacheFreeCall(seq, given, table, page_size=page, n_pages=n_pages, free_pages=free, free_head=head,
                           shared=shared, seq_len_out=seq, free_head_out=head,
                           **(dict(more, held_len_out=held) if window else {})).run()
        want_len = np.where(ends, 0, lens)
        wf, wh, ws = free_plain(s, want_len, t, f, h, page, n_shared, window, sinks, hl if window else None)
        got = books()
        assert np.array_equal(ints(kept.len_out), lens)
        assert np.array_equal(got[0], want_len) and np.array_equal(got[2], wf) and got[3] == wh
        assert np.array_equal(got[4], ws) and (not window or np.array_equal(got[5], want_len))
        for r in range(R):
            if keep[r] is not None and lens[r] == len(keep[r]):
                tokens[r] = [tokens[r][j] for j in keep[r]]
            else:
                refusals += 1
            tokens[r] = tokens[r][:want_len[r]]
        rows_now = k[:, :, 0, 0].float().cpu().numpy()
        for r in range(R):
            for j, x in enumerate(tokens[r]):
                if holds(j // page, want_len[r], want_len[r], page, window, sinks):
                    assert rows_now[got[1][r, j // page], j % page] == x
    assert refusals > 0 or window == 0
