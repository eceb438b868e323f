"""Attention over the paged cache in a sliding window with sinks, against a plain 64-bit form. What no new token of a
request sees holds NaN, and pages wholly out of sight have no entry in the table."""
import math

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.cache_util import NAN, Batch
from tests.gpu_util import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


def status(call):
    return avtp.read_device_status(call.workspace)


class Windowed(Batch):
    def __init__(self, requests, Hq, Hkv, d, page, window, sinks, hide=True, **kw):
        super().__init__(requests, Hq, Hkv, d, page, **kw)
        self.window, self.sinks = window, sinks
        for r, (s, n) in enumerate(requests):
            low = max(0, s - n - window + 1)  # of the first new token
            if not hide or n == 0 or low <= sinks:
                continue
            p = torch.arange(sinks, low)
            at = self.table[r, p // page].long().cuda(), (p % page).cuda()
            self.cache.k[at] = NAN
            self.cache.v[at] = NAN
            self.table[r, -(-sinks // page):low // page] = -9
        self.dev["table"] = self.table.cuda()

    def call(self, **kw):
        return super().call(window=self.window, sinks=self.sinks, **kw)

    def check(self, o, lse, scale=None):
        """As Batch.check, over the keys that each token sees: the roundings are the same ones."""
        scale = scale if scale is not None else self.d ** -0.5
        o, lse = o.float().cpu().double(), None if lse is None else lse.cpu().double()
        G = self.Hq // self.Hkv
        for r, (s, n) in enumerate(self.requests):
            a = int(self.cu[r])
            if n == 0:
                continue
            k, v = (t.double() for t in self.rows[r])
            place = (s - n + torch.arange(n))[:, None]
            u = torch.arange(s)[None]
            hidden = (u > place) | ((u <= place - self.window) & (u >= self.sinks))
            cnt = (~hidden).sum(1).double()[:, None]
            want, A = torch.zeros(n, self.Hq, self.d).double(), torch.zeros(n, self.Hq, self.d).double()
            ref, S = torch.full((n, self.Hq), -math.inf).double(), torch.zeros(n, self.Hq).double()
            for h in range(self.Hq if s else 0):
                q, kh, vh = self.q[a:a + n, h].double(), k[:, h // G], v[:, h // G]
                z = (q @ kh.T * scale).masked_fill_(hidden, -math.inf)
                S[:, h] = (q.abs() @ kh.abs().T * scale).masked_fill_(hidden, 0.0).amax(-1)
                ref[:, h] = torch.logsumexp(z, -1)
                p = torch.nan_to_num(torch.exp(z - ref[:, h, None]))
                want[:, h], A[:, h] = p @ vh, p @ vh.abs()
            e = (self.d + 4) * 2.0 ** -24 * S
            tol = (2.0 ** -8 * (1 + 2.0 ** -7) * (A + 2 * want.abs())
                   + A * (2 * e + 2.0 ** -21 + 2 * cnt * 2.0 ** -24)[..., None])
            got = o[a:a + n]
            assert torch.isfinite(got).all(), f"request {r}: not finite"
            off = (got - want).abs() - tol
            assert off.max() <= 0, f"request {r}: O off by {float((got - want).abs().max())}"
            if lse is not None:
                got = lse[:, a:a + n].t()
                empty = torch.isinf(ref)
                assert torch.equal(torch.isinf(got), empty) and (got[empty] < 0).all()
                size = ref.abs() + S + torch.log(cnt.clamp(min=1))
                tol = e + 2.0 ** -22 + cnt * 2.0 ** -24 + 4 * 2.0 ** -24 * size
                off = ((got - ref).abs() - tol)[~empty]
                assert off.numel() == 0 or off.max() <= 0, f"request {r}: LSE off"


def run(b, **kw):
    c = b.call(**kw).run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)
    return c


SHAPES = {"four": (32, 8, 128), "seven": (28, 4, 128), "plain": (4, 4, 64), "shared": (8, 1, 128), "small": (4, 2, 64),
          "twenty": (20, 1, 64), "most": (128, 1, 64)}
WINDOWS = [(1, 0), (1, 5), (16, 0), (100, 4), (64, 64), (129, 130), (500, 16)]


# ---------------------------------------------------------------- few rows
@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("shape,page", [("four", 64), ("seven", 16), ("plain", 48), ("shared", 128), ("small", 16),
                                        ("twenty", 32)])
def test_single_tokens(shape, page, window, sinks):
    run(Windowed([(700, 1), (1, 1), (90, 1), (2000, 1), (129, 1)], *SHAPES[shape], page, window, sinks))


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("shape,new", [("seven", 4), ("plain", 16), ("small", 13), ("four", 5)])
def test_drafted_tokens(shape, new, window, sinks):
    run(Windowed([(700, new), (new, new), (90, new), (2000, 1), (300, 0)], *SHAPES[shape], 16, window, sinks))


@pytest.mark.parametrize("past", [63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257])
@pytest.mark.parametrize("d", [64, 128])
def test_windows_that_begin_at_a_tiles_ends(d, past):
    for window, sinks in ((64, 0), (65, 1), (63, 64), (past, 0), (128, 63)):
        run(Windowed([(past + 1, 1), (past + 40, 2)], 4, 2, d, 16, window, sinks))


# ---------------------------------------------------------------- chunks
@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("shape,page", [("four", 64), ("seven", 16), ("plain", 48), ("shared", 128), ("small", 16),
                                        ("twenty", 32), ("most", 16)])
def test_chunks(shape, page, window, sinks):
    run(Windowed([(700, 300), (40, 40), (1000, 65), (129, 1), (90, 33)], *SHAPES[shape], page, window, sinks))


@pytest.mark.parametrize("past", [127, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_whose_windows_begin_at_a_blocks_ends(d, past):
    for window, sinks in ((128, 0), (129, 1), (127, 128), (past, 0), (64, 127)):
        run(Windowed([(past + 70, 70), (past + 257, 257)], 4, 2, d, 16, window, sinks))


@pytest.mark.parametrize("shape,n,window,sinks", [("four", 2600, 300, 4), ("plain", 5000, 700, 0), ("seven", 1500, 100, 200),
                                                  ("small", 4300, 2000, 130)])
def test_chunks_of_many_units(shape, n, window, sinks):
    """More units than are passed one by one, by their sum in closed form."""
    run(Windowed([(n + 500, n), (300, 40), (n, n)], *SHAPES[shape], 64, window, sinks))


@pytest.mark.parametrize("requests,Hq,Hkv,d,window,sinks", [
    ([(300 + 7 * i, 40) for i in range(32)], 32, 32, 64, 100, 4),
    ([(200 + 31 * i, 70) for i in range(19)], 48, 48, 64, 129, 0),
    ([(500, 90), (0, 60), (700, 0), (45, 50)] + [(1000 - 30 * i, 50 + 9 * i) for i in range(25)], 40, 40, 64, 64, 130),
    ([(400, 45), (300, 1), (90, 2)] * 10, 96, 96, 64, 70, 7),
    ([(300, 300), (1700, 1500)], 128, 16, 128, 100, 4),
    ([(1925, 1824)], 128, 16, 128, 127, 0)])
def test_as_many_chunks_as_fill_the_device_some_times(requests, Hq, Hkv, d, window, sinks):
    """Six units and more for each SM, nearly all of one length, none of which is in pieces."""
    run(Windowed(requests, Hq, Hkv, d, 32, window, sinks))


@pytest.mark.parametrize("shape,n", [("four", 700), ("seven", 401), ("plain", 600), ("twenty", 333), ("most", 130),
                                     ("four", 1), ("seven", 3)])
def test_a_window_of_one_token(shape, n):
    """A token that sees itself alone: its weight is 1 against its own maximum, and its value comes back as it was."""
    b = Windowed([(n + 77, n), (n, n)], *SHAPES[shape], 64, 1, 0)
    c = run(b)
    G, at = b.Hq // b.Hkv, 0
    for r, (s, m) in enumerate(b.requests):
        assert torch.equal(c.o[at:at + m].cpu(), b.rows[r][1][s - m:].repeat_interleave(G, 1).cpu())
        at += m


@pytest.mark.parametrize("order", ["token", "head", "mixed", "padded", "shared"])
@pytest.mark.parametrize("d", [64, 128])
def test_orders_of_pages(order, d):
    run(Windowed([(700, 300), (900, 1), (333, 70)], 8, 2, d, 32, 90, 20, order=order))


def test_a_mixed_batch():
    """Both kernels at work: chunks beside single tokens, idle and empty requests, rows behind the last."""
    b = Windowed([(900, 400), (2000, 1), (0, 1), (500, 0), (77, 1), (1500, 513), (3000, 2)], 28, 4, 128, 16, 200, 17, tail=5)
    o = torch.full((b.T, 28, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((28, b.T), 4.0, device="cuda")
    run(b, o=o, lse=lse)
    assert (o[-5:] == 3.0).all() and (lse[:, -5:] == 4.0).all()


@pytest.mark.parametrize("new", [1, 50])
def test_more_requests_than_a_warp_holds(new):
    rng = np.random.default_rng(new)
    run(Windowed([(int(rng.integers(new, 900)), new if i % 5 else 1) for i in range(75)], 8, 4, 64, 16, 120, 9))


@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 3), (500, 0)])
def test_tokens_that_see_nothing(window, sinks):
    """A request with fewer cached tokens than new ones: its first rows are empty."""
    run(Windowed([(3, 10), (0, 5), (100, 200), (1, 1), (260, 300)], 8, 2, 128, 16, window, sinks))


@pytest.mark.parametrize("idle", [1, 3, 40])
@pytest.mark.parametrize("live", [0, 1, 50])
def test_idle_requests_of_a_padded_batch(live, idle):
    """Requests without cached tokens: rows of zeros, beside others or alone; rows behind the last stay."""
    b = Windowed([(300 + 11 * i, 1) for i in range(live)] + [(0, 1 + i % 2) for i in range(idle)], 8, 2, 64, 16, 100, 4,
                 tail=2)
    o = torch.full((b.T, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((8, b.T), 4.0, device="cuda")
    run(b, o=o, lse=lse)
    assert (o[-2:] == 3.0).all() and (lse[:, -2:] == 4.0).all()


@pytest.mark.parametrize("R", [5, 40])
def test_a_refused_call_with_idle_requests_writes_nothing(R):
    b = Windowed([(300, 1)] * (R - 2) + [(0, 1), (0, 1)], 8, 2, 64, 16, 100, 4)
    b.dev["seq"][1] = -1
    o = torch.full((b.T, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((8, b.T), 4.0, device="cuda")
    c = b.call(o=o, lse=lse).run()
    assert status(c) == avtp.ERR_DEVICE_INPUT and (o == 3.0).all() and (lse == 4.0).all()


def test_long_requests_in_pieces():
    run(Windowed([(30000, 1)], 8, 2, 128, 64, 20000, 1000))
    run(Windowed([(9000, 200)], 4, 1, 64, 64, 5000, 500))


@pytest.mark.parametrize("requests", [[(700, 1), (90, 1)], [(700, 300), (90, 1)]])
def test_a_window_as_long_as_the_table_is_no_window(requests):
    b = Windowed(requests, 8, 2, 128, 16, 1 << 30, 7)
    c = run(b)
    plain = Batch.call(b).run()
    assert torch.equal(c.o, plain.o) and torch.equal(c.lse, plain.lse)


@pytest.mark.parametrize("requests", [[(700, 1), (90, 1)], [(700, 300), (90, 1)]])
def test_sinks_up_to_the_window_hide_nothing(requests):
    """Every key is a sink's or in a window: what avtp_cache_attention computes, within the same bounds."""
    b = Windowed(requests, 8, 2, 128, 16, 50, 1 << 30)
    c = run(b)
    Batch.check(b, c.o, c.lse)


def test_large_and_sharp_logits():
    b = Windowed([(700, 1), (900, 300)], 8, 2, 128, 16, 130, 4, k_scale=8.0)
    run(b)


@pytest.mark.parametrize("requests", [[(900, 1), (300, 2)], [(900, 400), (500, 70)]])
def test_results_do_not_change_from_run_to_run(requests):
    b = Windowed(requests, 28, 4, 128, 16, 200, 10)
    c = b.call()
    c.run()
    o, lse = c.o.clone(), c.lse.clone()
    for _ in range(5):
        c.run()
        assert torch.equal(c.o, o) and torch.equal(c.lse, lse)


def test_a_captured_call_replays_on_new_lengths():
    b = Windowed([(900, 1), (300, 1)], 8, 2, 64, 16, 100, 4, hide=False)  # the shorter request's window begins earlier
    c = b.call()
    c.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    d = Windowed([(902, 1), (280, 1)], 8, 2, 64, 16, 100, 4, seed=3)
    # its tokens where the captured call's table says
    for r, (s, _) in enumerate(d.requests):
        p = torch.arange(max(4, s - 100), s)
        at = b.table[r, p // 16].long().cuda(), (p % 16).cuda()
        first = b.table[r, 0].long().cuda()
        for t, rows in ((b.cache.k, d.rows[r][0]), (b.cache.v, d.rows[r][1])):
            t[at] = rows[p].cuda()
            t[first, :4] = rows[:4].cuda()
    b.dev["seq"].copy_(d.dev["seq"])
    b.dev["q"].copy_(d.dev["q"])
    graph.replay()
    torch.cuda.synchronize()
    assert status(c) == avtp.OK
    d.check(c.o, c.lse)


def test_a_bad_page_in_sight_is_recorded_and_one_out_of_sight_is_not_read():
    for n in (1, 100):
        b = Windowed([(700, n), (500, n)], 8, 2, 128, 16, 64, 16)
        low = 700 - n - 64 + 1
        b.dev["table"][0, low // 16] = b.cache.n_pages
        c = b.call().run()
        assert status(c) == avtp.ERR_DEVICE_INPUT
        good = Windowed([(500, n)], 8, 2, 128, 16, 64, 16)
        good.q, good.rows = b.q[n:], b.rows[1:]
        good.check(c.o[n:], c.lse[:, n:])


def test_two_calls_at_once_with_workspaces_of_their_own():
    a, b = (Windowed([(3000 + i, 1), (900, 200)], 8, 2, 128, 16, 300, 8, seed=i) for i in range(2))
    ca, cb = a.call(), b.call()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(10):
        ca.run(s)
        cb.run(t)
    torch.cuda.synchronize()
    a.check(ca.o, ca.lse)
    b.check(cb.o, cb.lse)


def test_refusals():
    b = Windowed([(90, 1)], 8, 2, 128, 16, 10, 2)
    for window, sinks in ((0, 0), (-1, 0), (5, -1)):
        with pytest.raises(avtp.AVTPError):
            Batch.call(b, window=window, sinks=sinks)
    with pytest.raises(ValueError):
        Batch.call(b, sinks=3)


# ---------------------------------------------------------------- together
def test_a_step_of_generation_in_a_window():
    """Slots, norms and rotary positions into the pages, attention in the window, the pages that it left given back: the
    rows agree with the same steps without pages, in 64 bits, over several tokens."""
    page, Hq, Hkv, d, W, S, n_pages = 16, 4, 2, 64, 40, 5, 40
    g = torch.Generator().manual_seed(5)
    inv = torch.from_numpy(avtp.rope_frequencies(d)[0]).cuda()
    qn, kn = ((1 + 0.2 * torch.randn(d, generator=g)).bfloat16().cuda() for _ in range(2))
    k, v = (torch.full((n_pages, page, Hkv, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = avtp.PagedCache(k, v)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    table = torch.full((2, 30), -1, dtype=torch.int32).cuda()
    free, head = torch.randperm(n_pages, generator=g).int().cuda(), i32([0])
    seq, held = i32([0, 0]), i32([0, 0])
    kept = [[], []]  # rotated keys and values of every token, as the cache holds them
    for step, new in enumerate([[150, 70]] + [[1, 1]] * 30):
        cu = np.concatenate([[0], np.cumsum(new)])
        T = int(cu[-1])
        q, kk, vv = (torch.randn(T, h, d, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
        pos = torch.cat([torch.arange(int(s), int(s) + n) for s, n in zip(seq.cpu(), new)]).int().cuda()
        slots, _, _ = avtp.cache_slots(i32(cu), T, page_size=page, n_pages=n_pages, block_table=table, free_pages=free,
                                       free_head=head, past_len=seq, seq_len=seq, free_head_out=head)
        rows = torch.empty_like(kk)
        q2, _ = avtp.rope(pos, inv, q=q, k=kk, v=vv, k_out=rows, q_norm=qn, k_norm=kn, cache=cache, slot_map=slots)
        o, lse = avtp.cache_attention(cache, q2, i32(cu), seq, table, max_new=max(new), window=W, sinks=S)
        for r in range(2):
            kept[r].append((rows[cu[r]:cu[r + 1]].cpu(), vv[cu[r]:cu[r + 1]].cpu()))
        b = Windowed.__new__(Windowed)
        b.requests, b.cu, b.Hq, b.Hkv, b.d, b.window, b.sinks = list(zip(seq.tolist(), new)), cu, Hq, Hkv, d, W, S
        b.q, b.rows = q2.cpu(), [tuple(torch.cat(x) for x in zip(*kept[r])) for r in range(2)]
        b.check(o, lse)
        call = avtp.CacheFreeCall(seq, seq, table, page_size=page, n_pages=n_pages, free_pages=free, free_head=head,
                                  window=W, sinks=S, held_len=held, seq_len_out=seq, held_len_out=held,
                                  free_head_out=head).run()
        assert status(call) == avtp.OK
        # the pages given back hold nothing that is seen again
        gone = free[int(head):].long()
        k[gone] = NAN
        v[gone] = NAN
    assert n_pages - int(head) <= n_pages and int(head) == sum(
        len([j for j in range(-(-s // page)) if j < -(-S // page) or j >= max(0, s - W + 1) // page]) for s in seq.tolist())
