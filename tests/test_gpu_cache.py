"""The paged cache on the GPU: slots, writes and attention against plain 64-bit forms (cache_util)."""
import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp, synth
from tests.cache_util import NAN, Batch, pool, slots_plain
from tests.gpu_util import DevWorkload, bf16_dev, ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


def status(call):
    return avtp.read_device_status(call.workspace)


# ---------------------------------------------------------------- slots
def _slots_case(past, new, page, seed=0, extra_free=2, head=0, tail=0, cols=1):
    rng = np.random.default_rng(seed)
    past, new = np.asarray(past, dtype=np.int32), np.asarray(new, dtype=np.int32)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    have, need = -(-past // page), -(-(past + new) // page)
    n_pages = int(need.sum()) + extra_free + head
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(past), int(need.max(initial=0)) + cols), -5, dtype=np.int32)
    at = 0
    for r, h in enumerate(have):
        table[r, :h] = ids[at:at + h]
        at += int(h)
    return dict(past=past, cu=cu, page=page, n_pages=n_pages, table=table, free=ids[at:].copy(), head=head,
                n_tokens=int(cu[-1]) + tail)


def _slots_call(c, **kw):
    dev = {k: torch.from_numpy(c[k].copy()).cuda() for k in ("past", "cu", "table", "free")}
    return avtp.CacheSlotsCall(dev["cu"], c["n_tokens"], page_size=c["page"], n_pages=c["n_pages"],
                               block_table=dev["table"], free_pages=dev["free"], past_len=dev["past"],
                               free_head=torch.tensor([c["head"]], dtype=torch.int32).cuda(), **kw), dev


SLOT_CASES = {
    "step": ([7, 64, 63, 0, 128, 1], [1, 1, 1, 1, 1, 1], 64),
    "nothing_new": ([7, 64, 0], [0, 0, 0], 16),
    "first_chunk": ([0, 0, 0], [33, 0, 700], 16),
    "mixed": ([5, 300, 16, 15, 17], [0, 1, 16, 17, 300], 16),
    "page_of_one": ([3, 0], [4, 2], 1),
    "odd_page": ([100, 3], [29, 41], 7),
    "one_cta_most": ([0, 11], [1900, 148], 32),
    "two_kernels": ([0, 11, 5], [1900, 148, 1], 32),
    "two_kernels_more": ([0, 11, 5], [8000, 192, 1], 32),
    "large": ([0, 11, 5, 0, 1000], [40000, 0, 3, 9000, 777], 48),
}


@pytest.mark.parametrize("name", sorted(SLOT_CASES))
def test_slots_match_the_plain_form(name):
    past, new, page = SLOT_CASES[name]
    c = _slots_case(past, new, page, head=3, tail=5)
    call, dev = _slots_call(c)
    call.run()
    assert status(call) == avtp.OK
    table, slots, seq, head = slots_plain(c["cu"], c["past"], c["table"], c["free"], c["head"], page, c["n_tokens"])
    assert np.array_equal(call.block_table.cpu().numpy(), table)
    assert np.array_equal(call.slot_map.cpu().numpy(), slots)
    assert np.array_equal(call.seq_len.cpu().numpy(), seq)
    assert int(call.free_head_out.item()) == head
    assert np.array_equal(dev["past"].cpu().numpy(), c["past"])


@pytest.mark.parametrize("R", [1, 31, 1024, 1025, 2048, 2049, 3000])
def test_slots_of_many_requests(R):
    rng = np.random.default_rng(R)
    c = _slots_case(rng.integers(0, 90, R), rng.integers(0, 12, R), 16, seed=R)
    call, _ = _slots_call(c)
    call.run()
    assert status(call) == avtp.OK
    table, slots, seq, head = slots_plain(c["cu"], c["past"], c["table"], c["free"], 0, 16, c["n_tokens"])
    assert np.array_equal(call.block_table.cpu().numpy(), table)
    assert np.array_equal(call.slot_map.cpu().numpy(), slots)
    assert np.array_equal(call.seq_len.cpu().numpy(), seq)
    assert int(call.free_head_out.item()) == head


def test_slots_advance_in_place_in_a_captured_graph():
    c = _slots_case([14, 0, 31], [1, 1, 1], 16, extra_free=40, cols=4)
    dev = {k: torch.from_numpy(c[k].copy()).cuda() for k in ("past", "cu", "table", "free")}
    head = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = avtp.CacheSlotsCall(dev["cu"], 3, page_size=16, n_pages=c["n_pages"], block_table=dev["table"],
                               free_pages=dev["free"], past_len=dev["past"], seq_len=dev["past"], free_head=head,
                               free_head_out=head)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    past, table, h = c["past"], c["table"], 0
    for _ in range(40):
        graph.replay()
        table, slots, past, h = slots_plain(c["cu"], past, table, c["free"], h, 16, 3)
        assert np.array_equal(call.slot_map.cpu().numpy(), slots)
        assert np.array_equal(dev["past"].cpu().numpy(), past)
        assert np.array_equal(dev["table"].cpu().numpy(), table)
        assert int(head.item()) == h


@pytest.mark.parametrize("tokens", [40, 20000])
@pytest.mark.parametrize("what", ["offsets_fall", "offsets_long", "first", "negative_past", "table_full", "pool_empty",
                                  "free_page", "free_page_negative", "partial_page", "head"])
def test_slots_refuse_and_write_nothing(what, tokens):
    c = _slots_case([5, 17, 0], [3, tokens, 4], 16, tail=2)
    if what == "offsets_fall":
        c["cu"][2] = c["cu"][1] - 1
    elif what == "offsets_long":
        c["cu"][3] += 3
    elif what == "first":
        c["cu"][0] = 1
    elif what == "negative_past":
        c["past"][1] = -1
    elif what == "table_full":
        c["past"][1] = c["table"].shape[1] * 16
    elif what == "pool_empty":
        c["free"] = c["free"][:-3]
    elif what == "free_page":
        c["free"][1] = c["n_pages"]
    elif what == "free_page_negative":
        c["free"][0] = -1
    elif what == "partial_page":
        c["table"][0, 0] = c["n_pages"] + 9
    elif what == "head":
        c["head"] = -1
    seq = torch.full((3,), -9, dtype=torch.int32, device="cuda")
    slot_map = torch.full((c["n_tokens"],), -9, dtype=torch.int32, device="cuda")
    out = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    call, dev = _slots_call(c, seq_len=seq, slot_map=slot_map, free_head_out=out)
    call.run()
    assert status(call) == avtp.ERR_DEVICE_INPUT
    assert (seq == -9).all() and (slot_map == -9).all() and int(out) == -9
    assert np.array_equal(dev["table"].cpu().numpy(), c["table"])


# ---------------------------------------------------------------- write
@pytest.mark.parametrize("order", ["token", "head", "shared", "padded", "mixed"])
@pytest.mark.parametrize("Hkv,d", [(1, 64), (1, 128), (3, 64), (2, 128), (5, 128), (8, 128), (16, 64)])
def test_write_puts_rows_in_their_slots(Hkv, d, order):
    g = torch.Generator(device="cuda").manual_seed(Hkv * d)
    n_pages, page, n, n_rows = 23, 13, 211, 400
    k_pool, v_pool = pool(n_pages, page, Hkv, d, order, fill=3.0)
    want_k, want_v = k_pool.clone(), v_pool.clone()
    base = torch.randn(2, n_rows, Hkv * d + 8, device="cuda", generator=g).to(torch.bfloat16)
    k, v = base[0, :, :Hkv * d].unflatten(1, (Hkv, d)), base[1, :, :Hkv * d].unflatten(1, (Hkv, d))
    slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:n].to(torch.int32)
    slots[::7] = -1
    kept = torch.randint(0, n_rows, (n,), device="cuda", generator=g).to(torch.int32)  # some rows twice
    live = slots >= 0
    at, row = slots[live].long(), kept[live].long()
    for kept_idx in (kept, None):
        src = row if kept_idx is not None else torch.nonzero(live).flatten()
        want_k[at // page, at % page] = k[src]
        want_v[at // page, at % page] = v[src]
        call = avtp.CacheWriteCall(avtp.PagedCache(k_pool, v_pool), slots, k, v, kept_idx=kept_idx).run()
        assert status(call) == avtp.OK
        assert torch.equal(k_pool, want_k) and torch.equal(v_pool, want_v)


def test_write_skips_and_records_bad_slots_and_rows():
    k_pool, v_pool = pool(4, 16, 2, 64, fill=0.0)
    k = torch.ones(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache = avtp.PagedCache(k_pool, v_pool)
    for slots, kept in (([0, 64, 5], [0, 1, 2]), ([0, -2, 5], [0, 1, 2]), ([0, 3, 5], [0, 8, 2]),
                        ([0, 3, 5], [0, -1, 2])):
        k_pool.zero_()
        call = avtp.CacheWriteCall(cache, torch.tensor(slots, dtype=torch.int32, device="cuda"), k, k,
                                   kept_idx=torch.tensor(kept, dtype=torch.int32, device="cuda")).run()
        assert status(call) == avtp.ERR_DEVICE_INPUT
        assert float(k_pool.float().sum()) == 2 * 128  # the good rows alone
    call = avtp.CacheWriteCall(cache, torch.zeros(0, dtype=torch.int32, device="cuda"), k, k).run()
    assert status(call) == avtp.OK


# ---------------------------------------------------------------- attention
HEADS = [(4, 2, 64), (28, 4, 128), (32, 8, 128), (8, 1, 128), (16, 16, 64), (5, 1, 64), (128, 1, 64), (66, 2, 128)]

STEP = [(1, 1), (64, 1), (0, 1), (63, 1), (65, 1), (700, 1), (129, 0), (16, 1), (17, 1), (0, 0), (2000, 1)]
DRAFT = [(5, 5), (64, 3), (3, 7), (130, 8), (1000, 2), (9, 0), (0, 4), (257, 6)]
CHUNK = [(40, 40), (300, 129), (70, 1), (128, 128), (513, 200), (30, 64), (0, 3), (256, 0), (900, 17)]


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("page", [16, 48, 64, 256])
def test_single_tokens(Hq, Hkv, d, page):
    b = Batch(STEP, Hq, Hkv, d, page, seed=page)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("page", [32, 80])
def test_a_few_tokens_a_request(Hq, Hkv, d, page):
    b = Batch(DRAFT, Hq, Hkv, d, page, seed=page)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("page", [16, 128])
def test_chunks_beside_single_tokens(Hq, Hkv, d, page):
    b = Batch(CHUNK, Hq, Hkv, d, page, seed=page + 1)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("order", ["head", "shared", "padded", "mixed"])
@pytest.mark.parametrize("requests", [STEP, CHUNK], ids=["step", "chunk"])
def test_page_orders(order, requests):
    b = Batch(requests, 14, 2, 128, 32, order=order, seed=3)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("Hq,Hkv,d,requests", [
    (8, 1, 128, [(20000, 1)]),                       # one row block over every CTA
    (32, 8, 128, [(3425, 1)]),
    (4, 2, 64, [(9000, 1), (1, 1), (12000, 2)]),
    (8, 2, 128, [(5000, 900)]),
    (8, 4, 64, [(3000, 3000)]),
    (7, 1, 128, [(1500, 800), (4000, 1), (2500, 33), (10, 10)]),
], ids=["mqa", "one", "small", "chunk", "prefill", "mixed"])
def test_long_requests(Hq, Hkv, d, requests):
    b = Batch(requests, Hq, Hkv, d, 64, seed=11)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("Hq,Hkv,d", [(7, 1, 64), (2, 2, 64), (28, 4, 128), (5, 1, 128)])
@pytest.mark.parametrize("seq,new", [(1500, 1), (2111, 1), (3425, 4), (5000, 2), (20000, 1)])
def test_one_request_in_few_and_many_pieces(Hq, Hkv, d, seq, new):
    b = Batch([(seq, new)], Hq, Hkv, d, 48, seed=seq)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("R", [159, 160, 161, 700])
def test_many_requests(R):
    rng = np.random.default_rng(R)
    b = Batch([(int(rng.integers(0, 200)), int(rng.integers(0, 3))) for _ in range(R)], 4, 2, 64, 16, seed=R)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


def _kinds(R, seed, chunk, few):
    """R requests: one in five a chunk of up to ``chunk`` tokens, the others up to ``few``."""
    rng = np.random.default_rng(seed)
    new = [int(rng.integers(1, chunk) if r % 5 == 2 else rng.integers(0, few + 1)) for r in range(R)]
    return [(int(rng.integers(0, 400)) + (n if r % 11 else 0), n) for r, n in enumerate(new)]


@pytest.mark.parametrize("Hq,Hkv,d,chunk,few", [(8, 2, 64, 90, 3), (28, 4, 128, 50, 1), (6, 6, 64, 300, 20)])
@pytest.mark.parametrize("R", [33, 64, 200])
def test_many_requests_of_either_kind(R, Hq, Hkv, d, chunk, few):
    b = Batch(_kinds(R, R + d, chunk, few), Hq, Hkv, d, 16, seed=R)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


def test_many_requests_of_two_row_warps():
    b = Batch(_kinds(70, 3, 8, 8), 8, 2, 128, 32, seed=12)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("Hq,Hkv,d,requests", [
    (16, 1, 128, [(900, 700)]),                                       # 16 tokens a block of rows, 44 of them
    (128, 1, 64, [(40, 130), (500, 120), (1, 1), (67, 67)]),          # two; some see nothing
    (32, 2, 64, [(300, 700), (513, 513), (20, 530), (0, 529), (600, 1)]),
    (34, 1, 128, [(400, 260)] * 35),                                  # three, 87 of them, many requests
], ids=["one", "all_heads", "blind", "many"])
def test_chunks_of_many_blocks_of_rows(Hq, Hkv, d, requests):
    b = Batch(requests, Hq, Hkv, d, 32, seed=17)
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("requests", [STEP, CHUNK, _kinds(36, 4, 60, 2)], ids=["step", "chunk", "many"])
def test_a_table_of_more_keys_than_steps(requests):
    """Rows of the table for 2^31 tokens: bounds with which a line of single tiles would pass 2^31."""
    b = Batch(requests, 16, 8, 64, 1024, seed=13, spare_pages=1)
    wide = torch.full((len(requests), 1 << 21), -7, dtype=torch.int32, device="cuda")
    wide[:, :b.table.shape[1]] = b.dev["table"]
    b.dev["table"] = wide
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


@pytest.mark.parametrize("scale,k_scale", [(1.0, 4.0), (1e-3, 1.0), (None, 0.0)])
def test_sharp_and_flat_softmax(scale, k_scale):
    for requests in (STEP, CHUNK):
        b = Batch(requests, 8, 2, 64, 32, seed=5, k_scale=k_scale)
        c = b.call(softmax_scale=scale).run()
        assert status(c) == avtp.OK
        b.check(c.o, c.lse, scale)


@pytest.mark.parametrize("requests", [STEP, DRAFT, CHUNK], ids=["step", "draft", "chunk"])
def test_strides_guards_and_rows_behind_the_last(requests):
    """q, O and the LSE in wider tensors, all around them and behind the last request's rows left as
    they were; the workspace exactly as large as it has to be."""
    b = Batch(requests, 8, 2, 128, 32, seed=7, tail=5)
    T, live = b.T, int(b.cu[-1])
    wide = torch.full((T + 2, 8 * 128 + 40), NAN, dtype=torch.bfloat16, device="cuda")
    q = wide[1:-1, 16:16 + 1024].unflatten(1, (8, 128))
    q[:live] = b.dev["q"][:live]
    b.dev["q"] = q
    o_base = torch.full((T + 2, 8 * 128 + 24), -3.0, dtype=torch.bfloat16, device="cuda")
    lse_base = torch.full((10, T + 9), -3.0, device="cuda")
    o, lse = o_base[1:-1, 8:8 + 1024].unflatten(1, (8, 128)), lse_base[1:-1, 4:4 + T]
    size = b.call().workspace.numel()
    ws_base = torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    c = b.call(o=o, lse=lse, workspace=ws_base[4096:4096 + size]).run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)
    assert (ws_base[:4096] == 0xA5).all() and (ws_base[4096 + size:] == 0xA5).all()
    o[:live] = -3.0
    lse[:, :live] = -3.0
    assert (o_base == -3.0).all() and (lse_base == -3.0).all()


def test_without_lse_and_same_bits_every_time():
    for requests in (STEP, CHUNK, [(7000, 1), (3000, 300)]):
        b = Batch(requests, 16, 4, 128, 64, seed=9)
        with_lse = b.call().run()
        without = b.call(lse=False).run()
        assert without.lse is None
        for _ in range(3):
            again = b.call(workspace=without.workspace).run()
            assert torch.equal(again.o, with_lse.o) and torch.equal(again.lse, with_lse.lse)
        assert torch.equal(without.o, with_lse.o)


def test_two_graphs_on_one_workspace_and_another_stream():
    b1, b2 = Batch(STEP, 8, 2, 128, 32, seed=1), Batch(CHUNK, 8, 2, 128, 32, seed=2)
    big = b2.call()
    ws = torch.full((max(big.workspace.numel(), b1.call().workspace.numel()),), 0xFF, dtype=torch.uint8, device="cuda")
    calls = [b1.call(workspace=ws), b2.call(workspace=ws)]
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):
            for g, c in zip(graphs, calls):
                c.o.fill_(7.0)
                g.replay()
        outs = [c.o.clone() for c in calls]
    side.synchronize()
    for b, c, o in zip((b1, b2), calls, outs):
        b.check(o, c.lse)
    # an explicit stream, with its own workspace, beside the current one
    fresh = b2.call()
    fresh.run(stream=side)
    b1.call(workspace=ws).run()
    torch.cuda.synchronize()
    b2.check(fresh.o, fresh.lse)


def test_changed_lengths_between_replays():
    b = Batch([(500, 1), (70, 1), (1000, 1)], 8, 2, 128, 32, seed=4)
    c = b.call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for lengths in ((500, 70, 1000), (1, 64, 65), (0, 0, 0), (499, 3, 640)):
        b.dev["seq"].copy_(torch.tensor(lengths, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        shorter = Batch.__new__(Batch)
        shorter.__dict__.update(b.__dict__)
        shorter.requests = [(n, 1) for n in lengths]
        shorter.rows = [(k[:n], v[:n]) for (k, v), n in zip(b.rows, lengths)]
        shorter.check(c.o, c.lse)


@pytest.mark.parametrize("what", ["offsets_fall", "offsets_long", "negative", "table_short", "max_new", "first"])
@pytest.mark.parametrize("requests", [[(70, 1), (40, 1), (300, 1)], [(70, 60), (40, 1), (300, 200)]],
                         ids=["step", "chunk"])
def test_attention_refuses_bad_lengths_and_writes_nothing(what, requests):
    b = Batch(requests, 8, 2, 128, 32, seed=6)
    kw = {}
    if what == "offsets_fall":
        b.dev["cu"][2] = int(b.cu[1]) - 1
    elif what == "offsets_long":
        b.dev["cu"][3] += 4
    elif what == "first":
        b.dev["cu"][0] = 1
    elif what == "negative":
        b.dev["seq"][1] = -1
    elif what == "table_short":
        b.dev["seq"][1] = b.table.shape[1] * 32 + 1
    elif what == "max_new":
        b.dev["cu"][1:] += b.max_new
        b.dev["q"] = torch.zeros(b.T + b.max_new, 8, 128, dtype=torch.bfloat16, device="cuda")
        kw["max_new"] = b.max_new
    o = torch.full_like(b.dev["q"], -3.0)
    c = b.call(o=o, **kw).run()
    assert status(c) == avtp.ERR_DEVICE_INPUT
    assert (o == -3.0).all()


@pytest.mark.parametrize("chunk", [2, 60], ids=["step", "chunk"])
@pytest.mark.parametrize("what", ["offsets_fall", "negative", "table_short", "max_new"])
def test_attention_refuses_bad_lengths_among_many_requests(what, chunk):
    b = Batch(_kinds(40, 5, chunk, 1), 8, 2, 128, 32, seed=14)
    kw = {}
    if what == "offsets_fall":
        b.dev["cu"][20] = int(b.cu[19]) - 1
    elif what == "negative":
        b.dev["seq"][37] = -1
    elif what == "table_short":
        b.dev["seq"][39] = b.table.shape[1] * 32 + 1
    elif what == "max_new":
        kw["max_new"] = b.max_new - 1
    o = torch.full_like(b.dev["q"], -3.0)
    c = b.call(o=o, **kw).run()
    assert status(c) == avtp.ERR_DEVICE_INPUT
    assert (o == -3.0).all()


@pytest.mark.parametrize("new", [1, 60])
def test_attention_refuses_positions_of_more_than_32_bits(new):
    """2^31 - 1 keys of a table that has the pages for them: the block behind the last key would not
    have a 32-bit position."""
    b = Batch([(90, new), (70, 1)], 2, 1, 64, 1 << 20, seed=15, spare_pages=0)
    wide = torch.zeros(2, 1 << 11, dtype=torch.int32, device="cuda")
    b.dev["table"] = wide
    for most in ((1 << 31) - 1, (1 << 31) - 255):
        b.dev["seq"][0] = most
        o = torch.full_like(b.dev["q"], -3.0)
        c = b.call(o=o).run()
        assert status(c) == avtp.ERR_DEVICE_INPUT
        assert (o == -3.0).all()


@pytest.mark.parametrize("new", [1, 300])
def test_a_table_bound_of_2_to_51_keys(new):
    """The bound alone, of which a request uses one page: steps stay as short as 2^31 keys need."""
    b = Batch([(5000, new)], 4, 1, 128, 1 << 20, seed=19, spare_pages=0)
    c = b.call()
    c._a.max_pages = (1 << 31) - 1
    c._a.table_stride = (1 << 31) - 1
    c.run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)


def test_buffers_of_a_call_on_another_stream_are_that_streams():
    """Work still queued on the current stream writes memory that it has given back; a call on a side
    stream must not be handed that memory for its outputs or workspace."""
    b = Batch(CHUNK, 8, 2, 128, 32, seed=18)
    d = b.dev
    side = torch.cuda.Stream()
    size = b.call().workspace.numel()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        dead = [torch.empty_like(d["q"]), torch.empty(8, b.T, device="cuda"),
                torch.empty(size, dtype=torch.uint8, device="cuda")]
        torch.cuda._sleep(20_000_000)
        for t in dead:
            t.fill_(7)
        del dead, t
        o, lse = avtp.cache_attention(b.cache, d["q"], d["cu"], d["seq"], d["table"], max_new=b.max_new, stream=stream)
        torch.cuda.synchronize()
        b.check(o, lse)


def test_two_calls_at_once_on_two_streams():
    """Each with a workspace of its own, over the same cache."""
    b = Batch([(700, 300), (70, 1), (0, 2), (900, 129), (2500, 1)], 16, 4, 128, 64, seed=16)
    calls = [b.call() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(30):
        for c, s in zip(calls, streams):
            c.run(stream=s)
    torch.cuda.synchronize()
    for c in calls:
        assert status(c) == avtp.OK
        b.check(c.o, c.lse)
    assert torch.equal(calls[0].o, calls[1].o) and torch.equal(calls[0].lse, calls[1].lse)


@pytest.mark.parametrize("requests", [[(70, 1), (100, 1), (300, 1)], [(200, 100), (100, 40), (300, 129)]],
                         ids=["step", "chunk"])
@pytest.mark.parametrize("page", [-1, 1 << 30, "past_end"])
def test_a_bad_page_is_recorded_and_spoils_its_request_alone(requests, page):
    b = Batch(requests, 8, 2, 128, 32, seed=8)
    b.dev["table"][1, 1] = b.cache.n_pages if page == "past_end" else page
    c = b.call().run()
    assert status(c) == avtp.ERR_DEVICE_INPUT
    a, e = int(b.cu[1]), int(b.cu[2])
    # the other requests' rows are right
    b.requests = [b.requests[0], (b.requests[1][0], 0), b.requests[2]]
    b.check(c.o, c.lse)
    assert e > a


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("page,order", [(16, "token"), (64, "head")])
def test_prune_then_slots_write_and_attention(page, order):
    """A pruned prefill's K and V rows go to pages by the prune's own device outputs, then follow-up
    chunks and single tokens attend to them, each step's rows written before."""
    segs = [[("t", 5), ("i", 300), ("t", 3), ("i", 129), ("t", 9)], [("i", 64), ("t", 7)], [("t", 12), ("i", 500), ("t", 2)]]
    wl = synth.make_custom(segs, keep_ratio=0.3, n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=256)
    dw = DevWorkload(wl)
    Hq, Hkv, d, R, T = 8, 2, 128, 3, wl.layout.n_tokens
    g = torch.Generator(device="cuda").manual_seed(1)

    def rand(*shape):
        return torch.randn(*shape, device="cuda", generator=g).to(torch.bfloat16)

    k, v = rand(T, Hkv, d), rand(T, Hkv, d)
    out = avtp.prune(dw.L, "hidden_variation", keep_ratio=dw.keep_ratio, keep_ratio_host=wl.keep_ratio,
                     rows={"k": k, "v": v}, h_cur=dw.t["h_cur"], h_prior=dw.t["h_prior"])
    n_pages = 90
    cache = avtp.PagedCache(*pool(n_pages, page, Hkv, d, order))
    free = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((R, 50), -1, dtype=torch.int32, device="cuda")
    head = torch.zeros(1, dtype=torch.int32, device="cuda")
    past = torch.zeros(R, dtype=torch.int32, device="cuda")

    def slots(cu, n):
        c = avtp.CacheSlotsCall(cu, n, page_size=page, n_pages=n_pages, block_table=table, free_pages=free,
                                free_head=head, free_head_out=head, past_len=past, seq_len=past).run()
        assert status(c) == avtp.OK
        return c.slot_map

    slot_map = slots(out.out_cu_seqlens, out.n_kept)
    avtp.cache_write(cache, slot_map, k, v, kept_idx=out.kept_idx)
    cu = out.out_cu_seqlens.cpu().numpy()
    rows = [[out.outputs["k"][cu[r]:cu[r + 1]], out.outputs["v"][cu[r]:cu[r + 1]]] for r in range(R)]
    for new in ([40, 1, 0], [1, 1, 1], [1, 1, 1], [3, 70, 2]):
        cu_new = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        cu_dev, n = torch.from_numpy(cu_new).cuda(), int(cu_new[-1])
        q, kn, vn = rand(n, Hq, d), rand(n, Hkv, d), rand(n, Hkv, d)
        avtp.cache_write(cache, slots(cu_dev, n), kn, vn)
        o, lse = avtp.cache_attention(cache, q, cu_dev, past, table, max_new=max(new))
        for r in range(R):
            rows[r] = [torch.cat([old, x[cu_new[r]:cu_new[r + 1]]]) for old, x in zip(rows[r], (kn, vn))]
        b = Batch.__new__(Batch)
        b.__dict__.update(requests=[(len(rows[r][0]), new[r]) for r in range(R)], Hq=Hq, Hkv=Hkv, d=d, cu=cu_new,
                          q=q.cpu(), rows=[tuple(t.cpu() for t in rows[r]) for r in range(R)])
        assert past.tolist() == [s for s, _ in b.requests]
        b.check(o, lse)


def test_a_whole_prompt_through_the_cache_matches_the_forward():
    """The first chunk of every request, nothing cached before: the layer's attention forward."""
    segs = [[("t", 200), ("i", 150)], [("t", 33)], [("i", 300), ("t", 12)]]
    wl = synth.make_custom(segs, keep_ratio=0.5, n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=256)
    dw = DevWorkload(wl)
    T = wl.layout.n_tokens
    v = torch.randn(T, 2, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(torch.bfloat16)
    q, k = dw.t["q"], dw.t["k"]
    o, lse, _, _ = avtp.attn_forward(dw.L, q=q, k=k, v=v, scores=False)
    cache = avtp.PagedCache(*pool(60, 16, 2, 128))
    table = torch.zeros(3, 30, dtype=torch.int32, device="cuda")
    free = torch.arange(60, dtype=torch.int32, device="cuda").flip(0).contiguous()
    slot_map, seq, _ = avtp.cache_slots(dw.L.cu_seqlens, T, page_size=16, n_pages=60, block_table=table,
                                        free_pages=free)
    avtp.cache_write(cache, slot_map, k, v)
    o2, lse2 = avtp.cache_attention(cache, q, dw.L.cu_seqlens, seq, table, max_new=350)
    b = Batch.__new__(Batch)
    cu = wl.layout.cu_seqlens
    b.__dict__.update(requests=[(int(n), int(n)) for n in np.diff(cu)], Hq=8, Hkv=2, d=128, cu=cu, q=q.cpu(),
                      rows=[(k[a:e].cpu(), v[a:e].cpu()) for a, e in zip(cu[:-1], cu[1:])])
    b.check(o2, lse2)
    b.check(o.to(torch.bfloat16), lse)
