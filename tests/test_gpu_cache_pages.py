"""The upkeep of the cache's pages on the GPU against plain forms one page and one token at a time."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.cache_util import pool
from tests.gpu_util import ensure_built
from tests.pages_util import compact_plain, fork_plain, free_plain, holds

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


def status(call):
    return avtp.read_device_status(call.workspace)


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def ints(t):
    return t.cpu().numpy()


# ---------------------------------------------------------------- free
class Freed:
    """Requests of given lengths on pages of their own in random order, all of them taken from the free list."""

    def __init__(self, seq, new, page, seed=0, window=0, sinks=0, held=None, stride=0, extra=3):
        rng = np.random.default_rng(seed)
        self.seq, self.new, self.page = np.asarray(seq), np.asarray(new), page
        self.window, self.sinks, self.held = window, sinks, None if held is None else np.asarray(held)
        need = -(-self.seq // page)
        self.n_pages = int(need.sum()) + extra
        ids = rng.permutation(self.n_pages)
        self.columns = max(int(need.max()), 1)
        self.table = np.full((len(seq), self.columns + stride), -3, dtype=np.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = ids[at:at + n]
            at += int(n)
        self.head = at
        self.free = np.concatenate([np.full(at, -9), ids[at:]]).astype(np.int32)
        self.shared = None

    def call(self, **kw):
        self.dev = dict(seq=i32(self.seq), new=i32(self.new), free=i32(self.free), head=i32([self.head]),
                        table=i32(self.table)[:, :self.columns])
        d = self.dev
        if self.held is not None:
            kw.update(window=self.window, sinks=self.sinks, held_len=i32(self.held))
        if self.shared is not None:
            d["shared"] = kw["shared"] = i32(self.shared)
        return avtp.CacheFreeCall(d["seq"], d["new"], d["table"], page_size=self.page, n_pages=self.n_pages,
                                  free_pages=d["free"], free_head=d["head"], **kw)

    def check(self, c):
        free, head, shared = free_plain(self.seq, self.new, self.table, self.free, self.head, self.page, self.shared,
                                        self.window, self.sinks, self.held)
        assert status(c) == avtp.OK
        assert int(c.free_head_out) == head and np.array_equal(ints(c.free_pages), free)
        assert np.array_equal(ints(c.seq_len_out), self.new)
        assert np.array_equal(ints(self.dev["table"]), self.table[:, :self.columns])
        if shared is not None:
            assert np.array_equal(ints(self.dev["shared"]), shared)
        if self.held is not None:
            assert np.array_equal(ints(c.held_out), self.new)


FREE_CASES = {
    "one_done": ([100], [0], 16),
    "nothing": ([100, 5, 0], [100, 5, 0], 16),
    "cut": ([100, 64, 65, 1, 16], [99, 63, 64, 0, 1], 16),
    "page_of_one": ([5, 3], [2, 0], 1),
    "odd_page": ([100, 3, 77], [29, 3, 0], 7),
    "empty_call": ([0], [0], 16),
    "many": (list(range(0, 3000, 7)), [n if n % 3 else n // 2 for n in range(0, 3000, 7)], 16),
    "many_rows": ([17 + i % 30 for i in range(2500)], [0 if i % 2 else 17 for i in range(2500)], 16),
    "rows_at_the_limit": ([5] * 2048, [0] * 2048, 4),
    "rows_past_the_limit": ([5] * 2049, [0] * 2049, 4),
    "long": ([200000, 3, 70000], [0, 3, 5], 16),
    "more_than_registers_hold": ([1200000, 3, 40], [0, 3, 0], 16),
}


@pytest.mark.parametrize("name", FREE_CASES)
def test_free(name):
    f = Freed(*FREE_CASES[name], stride=2 if len(name) % 2 else 0)
    f.check(f.call().run())


WINDOWS = {
    # seq, new, held, window, sinks
    "steps": ([100, 40, 41, 17, 500], [100, 40, 41, 17, 500], [0, 0, 0, 0, 300], 40, 0),
    "sinks": ([100, 300, 500, 20], [100, 300, 0, 20], [60, 0, 300, 0], 33, 5),
    "long_sinks": ([100, 300, 500, 60], [90, 300, 70, 0], [0, 0, 0, 0], 20, 120),
    "cut_and_window": ([100, 300, 500], [97, 290, 499], [80, 280, 490], 64, 16),
    "cut_into_sinks": ([100, 300], [10, 16], [0, 0], 64, 40),
    "done_behind_the_window": ([400, 50, 64], [0, 0, 0], [390, 50, 0], 16, 16),
    "window_of_one": ([100, 33, 1], [100, 33, 1], [50, 0, 0], 1, 0),
    "wider_than_all": ([100, 33, 1], [90, 0, 1], [50, 0, 0], 1 << 30, 1 << 30),
}


@pytest.mark.parametrize("page", [1, 7, 16])
@pytest.mark.parametrize("name", WINDOWS)
def test_free_what_a_window_has_left(name, page):
    seq, new, held, window, sinks = WINDOWS[name]
    f = Freed(seq, new, page, window=window, sinks=sinks, held=held, seed=len(name))
    f.check(f.call().run())


def shared_rows(f, groups):
    """Rows of each group share the first row's pages up to a column: (rows, columns). Counts follow."""
    for rows, columns in groups:
        for r in rows[1:]:
            f.table[r, :columns] = f.table[rows[0], :columns]
    holders = np.zeros(f.n_pages, dtype=np.int64)
    for r in range(len(f.seq)):
        for j in range(-(-int(f.seq[r]) // f.page)):
            if holds(j, f.seq[r], 0 if f.held is None else f.held[r], f.page, f.window, f.sinks):
                holders[f.table[r, j]] += 1
    f.shared = np.maximum(holders - 1, 0)


@pytest.mark.parametrize("done", [[0], [1], [0, 1], [0, 1, 2, 3], [3, 5], [0, 1, 2, 3, 4, 5]])
def test_free_of_shared_pages(done):
    seq = np.asarray([100, 90, 200, 100, 64, 300])
    f = Freed(seq, [0 if r in done else n for r, n in enumerate(seq)], 16, seed=4)
    shared_rows(f, [((0, 1, 3), 4), ((2, 5), 9)])
    f.check(f.call().run())


def test_free_of_many_shared_pages_does_not_depend_on_who_comes_first():
    R, n = 300, 1000
    f = Freed([n] * R, [0 if r % 3 else n for r in range(R)], 16, seed=5)
    shared_rows(f, [(tuple(range(g, g + 10)), 50) for g in range(0, R, 10)])
    f.check(f.call().run())


def test_free_of_more_shared_pages_than_registers_hold():
    R, n = 1800, 1000
    f = Freed([n] * R, [0 if r % 3 else n for r in range(R)], 16, seed=7)
    shared_rows(f, [(tuple(range(g, g + 6)), 30) for g in range(0, R, 6)])
    f.check(f.call().run())


@pytest.mark.parametrize("R", [2048, 2049, 2500])
def test_free_over_its_own_lengths_of_many_requests(R):
    """Lengths, held lengths and the list's head advanced in place, from shared memory or not."""
    rng = np.random.default_rng(R)
    seq = rng.integers(0, 90, R)
    held = np.maximum(seq - rng.integers(20, 60, R), 0)
    new = np.where(rng.random(R) < 0.3, 0, seq)
    f = Freed(seq, new, 4, window=9, sinks=5, held=held, seed=R)
    f.call()  # for its tensors
    d = f.dev
    dev_held = i32(held)
    c = avtp.CacheFreeCall(d["seq"], d["new"], d["table"], page_size=4, n_pages=f.n_pages, free_pages=d["free"],
                           free_head=d["head"], window=9, sinks=5, held_len=dev_held, seq_len_out=d["seq"],
                           held_len_out=dev_held, free_head_out=d["head"]).run()
    f.check(c)


def test_free_of_shared_pages_in_a_window():
    f = Freed([500, 500, 400, 90], [500, 490, 0, 80], 16, window=100, sinks=20, held=[300, 300, 200, 0], seed=6)
    shared_rows(f, [((0, 1), 20)])
    f.check(f.call().run())


def test_free_in_place_step_after_step_in_a_graph():
    f = Freed([600, 300], [600, 300], 16, window=50, sinks=3, held=[0, 0], extra=40)
    c = f.call()
    d = f.dev
    held = i32([0, 0])
    c = avtp.CacheFreeCall(d["seq"], d["new"], d["table"], page_size=16, n_pages=f.n_pages, free_pages=d["free"],
                           free_head=d["head"], window=50, sinks=3, held_len=held, seq_len_out=d["seq"], held_len_out=held,
                           free_head_out=d["head"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    free, head, seq, h = f.free, f.head, f.seq, np.asarray([0, 0])
    # (shorter by no more than the window has left: 590 and 580 tokens need the same first page, 300 and 292 too)
    for new in ([590, 300], [585, 300], [580, 292], [580, 0], [0, 0]):
        d["new"].copy_(i32(new))
        graph.replay()
        free, head, _ = free_plain(seq, new, f.table, free, head, 16, None, 50, 3, h)
        seq, h = np.asarray(new), np.asarray(new)
        assert status(c) == avtp.OK
        assert int(d["head"]) == head and np.array_equal(ints(d["free"]), free)
        assert np.array_equal(ints(d["seq"]), seq) and np.array_equal(ints(held), h)


REFUSED_FREES = {
    "longer": lambda f: f.new.__setitem__(1, 51),
    "negative": lambda f: f.new.__setitem__(1, -1),
    "negative_length": lambda f: f.seq.__setitem__(0, -1),
    "beyond_the_table": lambda f: f.seq.__setitem__(1, 16 * f.columns + 1),
    "page": lambda f: f.table.__setitem__((0, 3), f.n_pages),
    "page_minus": lambda f: f.table.__setitem__((0, 3), -1),
    "held": lambda f: f.held.__setitem__(0, 101),
    "held_minus": lambda f: f.held.__setitem__(0, -1),
    "cut_behind_the_window": lambda f: (f.held.__setitem__(1, 50), f.new.__setitem__(1, 20)),
    "list": lambda f: setattr(f, "head", 2),
    "head": lambda f: setattr(f, "head", -1),
    "head_behind_the_list": lambda f: setattr(f, "head", 1000),
}


@pytest.mark.parametrize("name", REFUSED_FREES)
def test_a_refused_free_writes_nothing(name):
    f = Freed([100, 50, 30], [0, 50, 30], 16, window=20, sinks=0, held=[0, 0, 0])
    REFUSED_FREES[name](f)
    refused(f)


def refused(f):
    c = f.call()
    before = {k: t.clone() for k, t in f.dev.items()}
    c.run()
    assert status(c) == avtp.ERR_DEVICE_INPUT
    for k, t in f.dev.items():
        assert torch.equal(t, before[k]), k
    assert (c.seq_len_out == -1).all() and int(c.free_head_out) == -1


def test_a_page_let_go_of_more_often_than_it_is_held_is_refused():
    f = Freed([100, 90], [0, 0], 16)
    shared_rows(f, [((0, 1), 4)])
    f.shared[f.table[0, 2]] = 0
    refused(f)
    f.shared[f.table[0, 2]] = -1
    refused(f)


def test_a_cut_inside_a_shared_page_is_refused():
    f = Freed([100, 90], [40, 90], 16)
    shared_rows(f, [((0, 1), 4)])
    refused(f)
    f.new[0] = 48  # at a page's end: the next token gets a page of its own
    f.check(f.call().run())
    f.new[0] = 70  # in a page of its own
    f.check(f.call().run())


# ---------------------------------------------------------------- fork and copy
class Forked(Freed):
    def __init__(self, seq, parent, child, page, length=None, rows=None, seed=0, window=0, sinks=0, held=None, spare=0):
        R = rows if rows is not None else max([len(seq)] + [c + 1 for c in child])
        full = list(seq) + [0] * (R - len(seq))
        super().__init__(full, full, page, seed=seed, window=window, sinks=sinks,
                         held=None if held is None else list(held) + [0] * (R - len(held)), extra=len(parent) + spare)
        self.columns = self.table.shape[1]
        self.parent, self.child, self.length = parent, child, length
        shared_rows(self, [])

    def call(self, **kw):
        self.dev = dict(seq=i32(self.seq), table=i32(self.table), shared=i32(self.shared), free=i32(self.free),
                        head=i32([self.head]), parent=i32(self.parent), child=i32(self.child))
        d = self.dev
        if self.held is not None:
            d["held"] = i32(self.held)
            kw.update(window=self.window, sinks=self.sinks, held_len=d["held"])
        if self.length is not None:
            kw["fork_len"] = i32(self.length)
        return avtp.CacheForkCall(d["parent"], d["child"], d["seq"], d["table"], page_size=self.page, n_pages=self.n_pages,
                                  free_pages=d["free"], free_head=d["head"], shared=d["shared"], **kw)

    def check(self, c):
        table, seq, head, shared, src, dst, held = fork_plain(
            self.parent, self.child, self.seq, self.table, self.free, self.head, self.page, self.shared, self.length,
            self.window, self.sinks, self.held)
        assert status(c) == avtp.OK
        d = self.dev
        assert np.array_equal(ints(d["table"]), table) and np.array_equal(ints(d["seq"]), seq)
        assert np.array_equal(ints(d["shared"]), shared) and int(c.free_head_out) == head
        assert np.array_equal(ints(c.copy_src), src) and np.array_equal(ints(c.copy_dst), dst)
        assert np.array_equal(ints(d["free"]), self.free)
        if held is not None:
            assert np.array_equal(ints(d["held"]), held)


FORKS = {
    "one": dict(seq=[100], parent=[0], child=[1], page=16),
    "several": dict(seq=[100, 64, 3], parent=[0, 0, 2, 1, 1], child=[3, 7, 4, 5, 6], page=16),
    "full_pages_alone": dict(seq=[64, 32], parent=[0, 1, 0], child=[2, 3, 4], page=16),
    "empty_parent": dict(seq=[0, 5], parent=[0, 1], child=[2, 3], page=16),
    "prefixes": dict(seq=[100, 64], parent=[0, 0, 0, 1, 1], child=[2, 3, 4, 5, 6], page=16, length=[0, 1, 64, 63, 33]),
    "page_of_one": dict(seq=[9], parent=[0, 0], child=[1, 2], page=1, length=[9, 4]),
    "odd_page": dict(seq=[100], parent=[0, 0], child=[1, 2], page=7, length=[98, 55]),
    "none": dict(seq=[10], parent=[], child=[], page=16),
    "many": dict(seq=[1000 + 13 * i for i in range(100)], parent=[i // 5 for i in range(500)],
                 child=[100 + (i * 7) % 500 for i in range(500)], page=16),
    "more_than_registers_hold": dict(seq=[1600 + i for i in range(60)], parent=[i // 15 for i in range(900)],
                                     child=[60 + (i * 7) % 900 for i in range(900)], page=16),
    "children_at_the_limit": dict(seq=[5], parent=[0] * 2048, child=list(range(1, 2049)), page=4),
    "children_past_the_limit": dict(seq=[5, 9], parent=[i % 2 for i in range(2100)], child=list(range(2, 2102)), page=4),
    "window": dict(seq=[500, 90, 33], parent=[0, 0, 1, 2], child=[3, 4, 5, 6], page=16, window=40, sinks=20,
                   held=[480, 0, 33], length=[500, 490, 90, 10]),
    "window_long_ago": dict(seq=[500, 90], parent=[0, 1], child=[2, 3], page=7, window=40, sinks=0, held=[300, 90]),
}


@pytest.mark.parametrize("name", FORKS)
def test_fork(name):
    f = Forked(**FORKS[name])
    f.check(f.call().run())


REFUSED_FORKS = {
    "parent": lambda f: f.parent.__setitem__(0, 9),
    "parent_minus": lambda f: f.parent.__setitem__(0, -1),
    "child": lambda f: f.child.__setitem__(0, 9),
    "child_minus": lambda f: f.child.__setitem__(0, -1),
    "twice": lambda f: f.child.__setitem__(1, 3),
    "itself": lambda f: f.child.__setitem__(0, 0),
    "child_of_a_child": lambda f: f.parent.__setitem__(1, 3),
    "length": lambda f: f.length.__setitem__(0, 101),
    "length_minus": lambda f: f.length.__setitem__(0, -1),
    "parent_length": lambda f: f.seq.__setitem__(0, -4),
    "beyond_the_table": lambda f: f.seq.__setitem__(0, 16 * f.columns + 1),
    "page": lambda f: f.table.__setitem__((0, 2), f.n_pages),
    "last_page": lambda f: f.table.__setitem__((0, 6), -1),
    "free_page": lambda f: f.free.__setitem__(f.head, f.n_pages),
    "list": lambda f: setattr(f, "head", len(f.free) - 1),
    "head": lambda f: setattr(f, "head", -1),
    "behind_the_window": lambda f: (f.held.__setitem__(0, 100), f.length.__setitem__(0, 20)),
}


@pytest.mark.parametrize("name", REFUSED_FORKS)
def test_a_refused_fork_writes_nothing(name):
    f = Forked([100, 50, 30], [0, 1], [3, 4], 16, length=[100, 50], rows=6, window=30, sinks=0, held=[0, 0, 0])
    REFUSED_FORKS[name](f)
    c = f.call()
    before = {k: t.clone() for k, t in f.dev.items()}
    c.run()
    assert status(c) == avtp.ERR_DEVICE_INPUT
    for k, t in f.dev.items():
        assert torch.equal(t, before[k]), k
    assert (c.copy_src == -1).all() and (c.copy_dst == -1).all() and int(c.free_head_out) == -1


@pytest.mark.parametrize("order", ["token", "head", "mixed", "padded", "shared"])
@pytest.mark.parametrize("page,Hkv,d", [(16, 4, 128), (7, 3, 64), (1, 1, 64), (100, 8, 128)])
def test_copy_of_pages(order, page, Hkv, d):
    g = torch.Generator().manual_seed(page)
    n_pages = 9
    k, v = pool(n_pages, page, Hkv, d, order)
    for t in (k, v):
        t.copy_(torch.randn(n_pages, page, Hkv, d, generator=g).bfloat16())
    want = [t.clone() for t in (k, v)]
    src, dst = [3, -1, 0, 5, -1, 3], [4, 6, -1, 7, -1, 1]
    for s, t in zip(src, dst):
        if s >= 0 and t >= 0:
            for w in want:
                w[t] = w[s]
    call = avtp.CacheCopyCall(avtp.PagedCache(k, v), i32(src), i32(dst)).run()
    assert status(call) == avtp.OK and torch.equal(k, want[0]) and torch.equal(v, want[1])
    call = avtp.CacheCopyCall(avtp.PagedCache(k, v), i32([n_pages, 0, 2, 8]), i32([1, n_pages, -2, 2])).run()
    want[0][2], want[1][2] = want[0][8], want[1][8]
    assert status(call) == avtp.ERR_DEVICE_INPUT and torch.equal(k, want[0]) and torch.equal(v, want[1])
    none = avtp.CacheCopyCall(avtp.PagedCache(k, v), i32([]), i32([])).run()
    assert status(none) == avtp.OK and torch.equal(k, want[0])


@pytest.mark.parametrize("n", [2048, 2049, 5000])
def test_copy_of_many_pages(n):
    """Pairs checked by one CTA, or by those that copy."""
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(2 * n, 1, 1, 64, generator=g).bfloat16().cuda() for _ in range(2))
    ids = torch.randperm(2 * n, generator=g)
    src, dst = ids[:n].clone(), ids[n:].clone()
    src[5] = -1
    for bad in (False, True):
        want = [t.clone() for t in (k, v)]
        if bad:
            src[n - 1], dst[3] = 2 * n, -2
        ok = ((src >= 0) & (src < 2 * n) & (dst >= 0)).nonzero()[:, 0]
        for t in want:
            t[dst[ok].cuda()] = t[src[ok].cuda()]
        call = avtp.CacheCopyCall(avtp.PagedCache(k, v), i32(src), i32(dst)).run()
        assert status(call) == (avtp.ERR_DEVICE_INPUT if bad else avtp.OK)
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])


# ---------------------------------------------------------------- compact
class Compacted:
    def __init__(self, seq, keep, page, Hkv=2, d=64, order="token", seed=0, other=True, base=False):
        """keep: positions of each request, or how many of them."""
        rng = np.random.default_rng(seed)
        self.seq, self.page, R = np.asarray(seq), page, len(seq)
        self.keep = [np.sort(rng.permutation(n)[:k]) if np.isscalar(k) else np.asarray(k, dtype=np.int64)
                     for n, k in zip(seq, keep)]
        self.base = np.cumsum([0] + list(seq))[:-1] if base else None
        n = np.asarray([len(k) for k in self.keep])
        self.cu = np.concatenate([[0], np.cumsum(n)])
        flat = [k + (self.base[r] if base else 0) for r, k in enumerate(self.keep)]
        self.idx = np.concatenate(flat + [np.full(2, 1 << 20)]).astype(np.int32)  # entries behind the last are not read
        need, to = -(-self.seq // page), -(-n // page)
        self.n_pages = int(need.sum() + (to.sum() if other else 0)) + 2
        ids = rng.permutation(self.n_pages)
        self.table = np.full((R, max(1, int(need.max()))), -3, dtype=np.int32)
        self.to = np.full((R, max(1, int(to.max())) + 1), -3, dtype=np.int32)
        at = 0
        for t, counts in ((self.table, need), (self.to, to if other else 0 * to)):
            for r, c in enumerate(counts):
                t[r, :c] = ids[at:at + c]
                at += int(c)
        self.other = other
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = pool(self.n_pages, page, Hkv, d, order)
        for t in (self.k, self.v):
            t.copy_(torch.randn(self.n_pages, page, Hkv, d, generator=g).bfloat16())
        self.before = [t.cpu().float().numpy() for t in (self.k, self.v)]

    def call(self, **kw):
        if self.other:
            kw["dst_table"] = i32(self.to)
        if self.base is not None:
            kw["base_cu"] = i32(self.base)
        return avtp.CacheCompactCall(avtp.PagedCache(self.k, self.v), i32(self.cu), i32(self.idx), i32(self.seq),
                                     i32(self.table), **kw)

    def want(self, rows=None):
        """With ``rows``: those requests alone."""
        cu, idx, base, table, to = self.cu, self.idx, self.base, self.table, self.to if self.other else self.table
        if rows is not None:
            idx = np.concatenate([idx[cu[r]:cu[r + 1]] for r in rows] + [idx[:0]])
            cu = np.concatenate([[0], np.cumsum([self.cu[r + 1] - self.cu[r] for r in rows])]).astype(int)
            base = None if base is None else base[rows]
            table, to = table[rows], to[rows]
        return [compact_plain(t, cu, idx, table, to, self.page, base) for t in self.before]

    def same(self, want):
        return all(np.array_equal(t.cpu().float().numpy(), w) for t, w in zip((self.k, self.v), want))


COMPACTS = {
    "one": ([100], [30], 16),
    "several": ([100, 64, 3, 0, 17], [30, 64, 1, 0, 0], 16),
    "all": ([50, 33], [50, 33], 16),
    "prefix": ([100], [list(range(40)) + [60, 99]], 16),
    "last": ([100, 20], [[99], [19]], 16),
    "page_of_one": ([40], [13], 1),
    "odd_page": ([100, 31], [61, 7], 7),
    "long": ([9000, 4000], [3000, 3999], 64),
    "many": ([100 + i for i in range(200)], [50 + i // 2 for i in range(200)], 16),
    "chunks": ([20000, 50, 9000], [9001, 20, 4097], 64),
    "requests_past_the_limit": ([20 + i % 9 for i in range(1100)], [7 + i % 5 for i in range(1100)], 4),
}


@pytest.mark.parametrize("other", [True, False])
@pytest.mark.parametrize("name", COMPACTS)
def test_compact(name, other):
    c = Compacted(*COMPACTS[name], other=other, base=len(name) % 2 == 0, seed=len(name))
    call = c.call().run()
    assert status(call) == avtp.OK and np.array_equal(ints(call.len_out), np.diff(c.cu))
    assert c.same(c.want())


@pytest.mark.parametrize("other", [True, False])
@pytest.mark.parametrize("order", ["token", "head", "mixed", "padded", "shared"])
@pytest.mark.parametrize("Hkv,d", [(8, 128), (1, 64), (3, 128), (20, 64)])
def test_compact_of_any_order_of_pages(order, other, Hkv, d):
    c = Compacted([300, 77], [140, 50], 16, Hkv, d, order, other=other)
    call = c.call().run()
    assert status(call) == avtp.OK and c.same(c.want())


@pytest.mark.parametrize("other", [True, False])
def test_a_captured_compaction_replays_on_new_positions(other):
    c = Compacted([300, 200], [100, 60], 16, other=other)
    kept = avtp.CacheCompactCall(avtp.PagedCache(c.k, c.v), i32(c.cu), i32(c.idx), i32(c.seq), i32(c.table),
                                 **(dict(dst_table=i32(c.to)) if other else {}))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept.run()
    new = Compacted([300, 200], [100, 60], 16, other=other, seed=0)
    for r, n in enumerate((100, 60)):  # other positions, the same numbers of them
        new.idx[new.cu[r]:new.cu[r + 1]] = np.arange(n) * 2 + r + 1
    kept._keep[1].copy_(i32(new.idx))
    graph.replay()
    torch.cuda.synchronize()
    assert status(kept) == avtp.OK
    c.idx = new.idx
    assert c.same(c.want())


@pytest.mark.parametrize("other", [True, False])
def test_compact_of_nothing(other):
    c = Compacted([30, 20], [0, 0], 16, other=other)
    call = c.call().run()
    assert status(call) == avtp.OK and c.same(c.before) and (call.len_out == 0).all()


def test_compact_to_other_pages_takes_positions_in_any_order():
    c = Compacted([100], [[5, 99, 5, 0, 64]], 16)
    call = c.call().run()
    assert status(call) == avtp.OK and c.same(c.want())


def test_compact_to_other_pages_skips_what_is_wrong():
    c = Compacted([100, 60, 50], [[1, 2, 100, 4], [0, 1], [3, 4]], 16)
    c.idx[4] = -1            # request 1's first
    c.table[2, 0] = c.n_pages
    call = c.call().run()
    assert status(call) == avtp.ERR_DEVICE_INPUT
    good = Compacted([100, 60, 50], [[1, 2, 100, 4], [0, 1], [3, 4]], 16)
    want = good.before
    for w in want:
        for r, j, p in ((0, 0, 1), (0, 1, 2), (0, 3, 4), (1, 1, 1)):
            w[good.to[r, j // 16], j % 16] = w[good.table[r, p // 16], p % 16]
    assert c.same(want)
    d = Compacted([100], [30], 16)
    d.to[0, 1] = -1
    call = d.call().run()
    want = [w.copy() for w in d.before]
    for w in want:
        for j, p in enumerate(d.keep[0][:16]):
            w[d.to[0, 0], j] = w[d.table[0, p // 16], p % 16]
    assert status(call) == avtp.ERR_DEVICE_INPUT and d.same(want)


BAD_IN_PLACE = {
    "order": lambda c: c.idx.__setitem__(3, c.idx[2]),
    "beyond": lambda c: c.idx.__setitem__(29, 100),
    "negative": lambda c: c.idx.__setitem__(0, -1),
    "source_page": lambda c: c.table.__setitem__((0, 6), c.n_pages),
    "destination_page": lambda c: c.table.__setitem__((0, 1), -1),
}


@pytest.mark.parametrize("name", BAD_IN_PLACE)
def test_compact_in_place_leaves_a_request_with_a_fault_as_it_was(name):
    keep = list(range(3, 90, 3)) + [99]
    c = Compacted([100, 60], [keep, 20], 16, other=False)
    BAD_IN_PLACE[name](c)
    call = c.call().run()
    assert status(call) == avtp.ERR_DEVICE_INPUT
    assert c.same(c.want(rows=[1]))


def test_compact_in_place_of_shared_pages():
    """Pages that others hold may stay, and are not written."""
    c = Compacted([100, 60], [list(range(32)) + [50, 60, 99], 20], 16, other=False)
    shared = np.zeros(c.n_pages, dtype=np.int32)
    shared[c.table[0, :2]] = 1  # the prefix, which stays where it is
    call = c.call(shared=i32(shared)).run()
    assert status(call) == avtp.OK and c.same(c.want())
    c = Compacted([100, 60], [list(range(32)) + [50, 60, 99], 20], 16, other=False)
    shared[c.table[0, 2]] = 1
    call = c.call(shared=i32(shared)).run()
    assert status(call) == avtp.ERR_DEVICE_INPUT and c.same(c.want(rows=[1]))


def test_compact_of_a_request_that_let_go_of_pages():
    """Tokens on pages that a window has left are not the request's: not to be kept, nor to be written."""
    more = dict(window=32, sinks=16, held_len=i32([100, 60]))
    c = Compacted([100, 60], [[2, 70, 80, 99], [1, 40]], 16)
    call = c.call(**more).run()
    assert status(call) == avtp.OK and c.same(c.want())
    c = Compacted([100, 60], [[2, 40, 80, 99], [1, 40]], 16)
    call = c.call(**more).run()
    want = [w.copy() for w in c.before]
    for w in want:
        for r, j, p in ((0, 0, 2), (0, 2, 80), (0, 3, 99), (1, 0, 1), (1, 1, 40)):
            w[c.to[r, j // 16], j % 16] = w[c.table[r, p // 16], p % 16]
    assert status(call) == avtp.ERR_DEVICE_INPUT and c.same(want)
    c = Compacted([100, 60], [list(range(1, 16)) + list(range(70, 80)), [1, 40]], 16, other=False)
    call = c.call(**more).run()  # 25 tokens: the last ones would go to the second page
    assert status(call) == avtp.ERR_DEVICE_INPUT and c.same(c.want(rows=[1]))


@pytest.mark.parametrize("other", [True, False])
@pytest.mark.parametrize("what", ["first", "decreasing", "beyond"])
def test_compact_with_bad_offsets_writes_nothing(what, other):
    c = Compacted([100, 60], [30, 20], 16, other=other)
    if what == "first":
        c.cu[0] = 1
    elif what == "decreasing":
        c.cu[1] = 51
    else:
        c.cu[2] = len(c.idx) + 1
    call = c.call().run()
    assert status(call) == avtp.ERR_DEVICE_INPUT and c.same(c.before) and (call.len_out == -1).all()


def test_calls_on_another_stream():
    """Buffers that a call makes come from the stream that it runs on."""
    s = torch.cuda.Stream()
    c = Compacted([300, 200], [100, 60], 16)
    f = Forked([100, 50], [0, 1, 1], [2, 3, 4], 16)
    f.call()
    g = Freed([100, 50], [0, 50], 16)
    g.call()
    torch.cuda.synchronize()
    kept = avtp.cache_compact(avtp.PagedCache(c.k, c.v), i32(c.cu), i32(c.idx), i32(c.seq), i32(c.table),
                              dst_table=i32(c.to), stream=s)
    d = f.dev
    src, dst, head = avtp.cache_fork(d["parent"], d["child"], d["seq"], d["table"], page_size=16, n_pages=f.n_pages,
                                     free_pages=d["free"], free_head=d["head"], shared=d["shared"], stream=s)
    avtp.cache_copy(avtp.PagedCache(c.k, c.v), i32([0]), i32([-1]), stream=s)
    e = g.dev
    seq, ghead = avtp.cache_free(e["seq"], e["new"], e["table"], page_size=16, n_pages=g.n_pages, free_pages=e["free"],
                                 free_head=e["head"], stream=s)
    s.synchronize()
    assert c.same(c.want()) and np.array_equal(ints(kept), np.diff(c.cu))
    want = fork_plain(f.parent, f.child, f.seq, f.table, f.free, f.head, 16, f.shared)
    assert np.array_equal(ints(d["table"]), want[0]) and np.array_equal(ints(src), want[4]) and int(head) == want[2]
    free, h, _ = free_plain(g.seq, g.new, g.table, g.free, g.head, 16)
    assert np.array_equal(ints(e["free"]), free) and int(ghead) == h and np.array_equal(ints(seq), g.new)


def test_the_binding_refuses():
    c = Compacted([100, 60], [30, 20], 16)
    cache, cu, idx, seq, table = avtp.PagedCache(c.k, c.v), i32(c.cu), i32(c.idx), i32(c.seq), i32(c.table)
    for kw in (dict(dst_table=i32(c.to[:1])), dict(base_cu=i32([0])), dict(shared=seq), dict(window=3), dict(len_out=cu),
               dict(held_len=cu)):
        with pytest.raises(ValueError):
            avtp.cache_compact(cache, cu, idx, seq, table, **kw)
    with pytest.raises(ValueError):
        avtp.cache_compact(cache, cu, idx.long(), seq, table)
    one, pages = i32([0]), dict(page_size=16, n_pages=c.n_pages, free_pages=idx)
    shared = i32(np.zeros(c.n_pages))
    for kw in (dict(shared=None), dict(shared=one), dict(shared=shared, window=2), dict(shared=shared, fork_len=cu)):
        with pytest.raises(ValueError):
            avtp.cache_fork(one, one, seq, table, **pages, **kw)
    for kw in (dict(free_head=None), dict(free_head=cu), dict(free_head=one, window=4), dict(free_head=one, shared=one)):
        with pytest.raises(ValueError):
            avtp.cache_free(seq, seq, table, **pages, **kw)
    with pytest.raises(ValueError):
        avtp.cache_copy(cache, seq, one)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 5)])
def test_a_run_of_slots_forks_and_frees(window, sinks):
    """Steps of a serving program, every number on the device: new tokens, forks, cuts and ends; the books agree with the
    plain forms', and every token's rows are found where the table says."""
    rng = np.random.default_rng(8 + window)
    page, R, n_pages, Hkv, d = 16, 12, 400, 1, 64
    k, v = pool(n_pages, page, Hkv, d, fill=0.0)
    cache = avtp.PagedCache(k, v)
    table = i32(np.full((R, 40), -1))
    seq, held, head = i32(np.zeros(R)), i32(np.zeros(R)), i32([0])
    free, shared = i32(rng.permutation(n_pages)), i32(np.zeros(n_pages))
    more = dict(window=window, sinks=sinks, held_len=held) if window else {}
    tokens = [[] for _ in range(R)]  # what each request's tokens hold
    stamp = 0
    for step in range(25):
        lens = np.asarray([len(t) for t in tokens])
        new = np.where((lens > 0) | (rng.random(R) < 0.3), rng.integers(0, 40, R), 0)
        new = np.where(lens + new > 600, 0, new)
        cu = np.concatenate([[0], np.cumsum(new)])
        slots = avtp.cache_slots(i32(cu), int(cu[-1]), page_size=page, n_pages=n_pages, block_table=table, free_pages=free,
                                 free_head=head, past_len=seq, seq_len=seq, free_head_out=head)[0]
        rows = (stamp + torch.arange(int(cu[-1])) % 250).float()
        stamp += 7
        rows = (rows[:, None, None] * torch.ones(len(rows), Hkv, d)).bfloat16().cuda()
        avtp.cache_write(cache, slots, rows, rows)
        flat = rows[:, 0, 0].float().cpu().tolist()
        for r in range(R):
            tokens[r] += flat[cu[r]:cu[r + 1]]
        lens = np.asarray([len(t) for t in tokens])
        empty = [r for r in range(R) if lens[r] == 0]
        parents = [r for r in range(R) if lens[r] > 0]
        if empty and parents and step % 2:
            p = [int(rng.choice(parents)) for _ in empty]
            want = fork_plain(p, empty, ints(seq), ints(table), ints(free), int(head), page, ints(shared), None, window,
                              sinks, ints(held) if window else None)
            src, dst, _ = avtp.cache_fork(i32(p), i32(empty), seq, table, page_size=page, n_pages=n_pages, free_pages=free,
                                          free_head=head, shared=shared, free_head_out=head, **more)
            avtp.cache_copy(cache, src, dst)
            assert np.array_equal(ints(table), want[0]) and np.array_equal(ints(shared), want[3]) and int(head) == want[2]
            for a, b in zip(p, empty):
                tokens[b] = list(tokens[a])
        lens = np.asarray([len(t) for t in tokens])
        after = np.where(rng.random(R) < 0.15, 0, lens)
        f, h, s = free_plain(ints(seq), after, ints(table), ints(free), int(head), page, ints(shared), window, sinks,
                             ints(held) if window else None)
        call = avtp.CacheFreeCall(seq, i32(after), table, page_size=page, n_pages=n_pages, free_pages=free, free_head=head,
                                  shared=shared, seq_len_out=seq, free_head_out=head,
                                  **(dict(more, held_len_out=held) if window else {})).run()
        assert status(call) == avtp.OK
        assert np.array_equal(ints(free), f) and int(head) == h and np.array_equal(ints(shared), s)
        assert np.array_equal(ints(seq), after)
        pages, got = ints(table), k[:, :, 0, 0].float().cpu().numpy()
        for r in range(R):
            tokens[r] = tokens[r][:after[r]]
            for p, x in enumerate(tokens[r]):
                if holds(p // page, after[r], after[r], page, window, sinks):
                    assert got[pages[r, p // page], p % page] == x


def test_a_pruned_batch_goes_on_pruned_in_place():
    """Rows written where a prune put them, a second selection moved together in place, the pages behind it freed."""
    rng = np.random.default_rng(2)
    page, Hkv, d, n_pages = 16, 2, 64, 80
    lens = [300, 170]
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(T, Hkv, d, generator=g).bfloat16().cuda() for _ in range(2))
    cache = avtp.PagedCache(*pool(n_pages, page, Hkv, d))
    table, free = i32(np.full((2, 30), -1)), i32(rng.permutation(n_pages))
    slots, seq, head = avtp.cache_slots(i32(cu), T, page_size=page, n_pages=n_pages, block_table=table, free_pages=free)
    avtp.cache_write(cache, slots, k, v)
    kept = np.sort(rng.permutation(T)[:200])  # positions of the packed batch, as kept_idx has them
    kept_cu = np.searchsorted(kept, cu)
    n = avtp.cache_compact(cache, i32(kept_cu), i32(kept), seq, table, base_cu=i32(cu))
    seq2, head2 = avtp.cache_free(seq, n, table, page_size=page, n_pages=n_pages, free_pages=free, free_head=head)
    assert np.array_equal(ints(seq2), np.diff(kept_cu))
    assert int(head2) == int(sum(-(-np.diff(kept_cu) // page)))
    for r in range(2):
        p = np.arange(kept_cu[r + 1] - kept_cu[r])
        at = torch.from_numpy(ints(table)[r, p // page]).long().cuda(), torch.from_numpy(p % page).cuda()
        rows = torch.from_numpy(kept[kept_cu[r]:kept_cu[r + 1]]).cuda()
        assert torch.equal(cache.k[at], k[rows]) and torch.equal(cache.v[at], v[rows])


def test_the_readme_example_of_positions_and_upkeep():
    """The example run as it stands, behind slots for the step's tokens: two requests cut to their kept tokens, and two
    rows more that go on from the first."""
    with open(os.path.join(os.path.dirname(__file__), "..", "README.md"), encoding="utf-8") as f:
        code = [c for c in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "cache_fork" in c]
    assert len(code) == 1
    g = torch.Generator(device="cuda").manual_seed(3)

    def rand(*shape):
        return torch.randn(*shape, device="cuda", generator=g).to(torch.bfloat16)

    n_pages, lens, keep = 24, [300, 130, 0, 0], [np.arange(0, 300, 3), np.arange(7, 130)]
    cache = avtp.PagedCache.new(n_pages, page_size=64, n_kv_heads=8, head_dim=128)
    cache.k.normal_(generator=g)
    cache.v.normal_(generator=g)
    table = torch.full((4, 8), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    cu = i32(np.concatenate([[0], np.cumsum(lens)]))
    slots, seq_len, free_head = avtp.cache_slots(cu, sum(lens), page_size=64, n_pages=n_pages, block_table=table,
                                                 free_pages=free)
    T = sum(lens)
    env = dict(avtp=avtp, torch=torch, cache=cache, slots=slots, n_pages=n_pages, table=table, free=free,
               free_head=free_head, seq_len=seq_len, q_new=rand(T, 32, 128), k_new=rand(T, 8, 128),
               v_new=rand(T, 8, 128), wq=rand(128), wk=rand(128), pos=i32(np.tile(np.arange(T), (3, 1))),
               plane_of_pair=i32(np.arange(64) % 3), keep_cu=i32([0, 100, 223, 223, 223]),
               keep_idx=i32(np.concatenate(keep)), parent=i32([0, 0]), child=i32([2, 3]),
               shared=torch.zeros(n_pages, dtype=torch.int32, device="cuda"))
    exec(compile(code[0], "README.md", "exec"), env)  # noqa: S102
    assert torch.isfinite(env["q"].float()).all()
    assert env["seq_len"].tolist() == [100, 123, 100, 100] and env["free_head"].tolist() == [2 + 2 + 2]
    # what a row holds is the kept tokens' values as they came in, and a child's are its parent's
    flat = table.long()
    for r, want in ((0, keep[0]), (1, keep[1] + 300), (2, keep[0]), (3, keep[0])):
        j = torch.arange(len(want), device="cuda")
        assert torch.equal(cache.v[flat[r][j // 64], j % 64], env["v_new"][torch.as_tensor(want).cuda()])
    assert torch.equal(flat[2, :1], flat[0, :1]) and len({int(flat[r, 1]) for r in (0, 2, 3)}) == 3
