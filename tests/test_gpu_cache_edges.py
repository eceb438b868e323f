"""The paged cache on the GPU: what lies outside the requests' tokens, bounds far above them, and the
forms of slots and writes that large calls take."""
import math
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp, synth
from tests.cache_util import Batch, pool, slots_plain
from tests.gpu_util import DevWorkload, ensure_built

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


def status(call):
    return avtp.read_device_status(call.workspace)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 8, 128), (16, 16, 64), (20, 4, 128)])
def test_slots_behind_a_requests_last_token_change_no_bit(Hq, Hkv, d):
    """The keys' rows that follow a request's last token in its page, as zeros, NaN and infinities. A key
    near the end stands out by 2^8 to 2^13 weights: far enough that a row's reference may move for it, not so
    far that its own sum makes it."""
    b = Batch([(164 + r % 9, 1) for r in range(60)], Hq, Hkv, d, 64, seed=d)
    G = Hq // Hkv
    for r, (s, _) in enumerate(b.requests):
        q = b.q[r].float().view(Hkv, G, d)[:, 0]
        key = (9.0 * d ** 0.5 * q / (q * q).sum(-1, keepdim=True)).to(torch.bfloat16)
        b.rows[r][0][s - 2] = key
        b.cache.k[int(b.table[r, (s - 2) // 64]), (s - 2) % 64] = key.cuda()
    spare = torch.isnan(b.cache.k)
    got = []
    for fill in (0.0, float("nan"), float("inf"), -3e38):
        b.cache.k[spare] = fill
        c = b.call().run()
        assert status(c) == avtp.OK
        b.check(c.o, c.lse)
        got.append((c.o, c.lse))
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])


@pytest.mark.parametrize("Hq,Hkv,d,requests", [
    (2, 2, 64, [(33, 33)]),  # fewer rows than a tile's tokens
    (8, 2, 128, [(300, 129), (40, 40), (513, 200)]),
    (34, 1, 128, [(70, 70), (9, 5)]),
], ids=["short", "chunks", "odd_group"])
def test_chunks_take_no_bit_from_slots_or_queries_behind_the_last(Hq, Hkv, d, requests):
    """A chunk's last tile of queries reaches behind the last request, its last block of keys behind the last
    token: zeros, NaN and infinities there."""
    b = Batch(requests, Hq, Hkv, d, 64, seed=Hq, tail=70)
    live = int(b.cu[-1])
    spare_k, spare_v = torch.isnan(b.cache.k), torch.isnan(b.cache.v)
    got = []
    for fill in (0.0, float("nan"), float("inf"), -3e38):
        b.cache.k[spare_k] = fill
        b.cache.v[spare_v] = fill
        b.dev["q"][live:] = fill
        o = torch.full_like(b.dev["q"], 5.0)
        c = b.call(o=o).run()
        assert status(c) == avtp.OK
        b.check(c.o, c.lse)
        assert (o[live:] == 5.0).all()
        got.append((o[:live].clone(), c.lse[:, :live].clone()))
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])


def _step_shift(blocks, keys, tile, Hkv):
    """The library's rule: steps of a line of `blocks` row blocks a KV head stay below 2^31."""
    shift = 0
    while blocks * ((keys // tile >> shift) + 4) * Hkv >= 1 << 31:
        shift += 1
    return shift


MANY = [(int(n), 1) for n in np.random.default_rng(8).integers(0, 3000, 34)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hkv,requests", [
    (8, [(4100, 1), (0, 1), (3000, 1)] + [(700, 1)] * 14),
    (8, [(2500, 1), (2300, 560), (900, 40)] + [(1500, 1)] * 14),  # 560 tokens of 16 heads: 35 blocks of rows
    (4, MANY + [(1, 1), (3500, 1)]),
    (4, MANY + [(2200, 544), (1200, 30)]),
], ids=["step", "chunk", "many", "many_chunks"])
def test_steps_of_several_tiles(Hkv, requests, d):
    """A table for 2^31 keys, with which a line of single tiles would pass 2^31 steps in either kernel: steps of
    two or more, several of them a row block and more than there are CTAs, so that runs end inside blocks."""
    G, page, columns = 16, 1024, 1 << 21
    R, T = len(requests), sum(n for _, n in requests)
    keys = min(columns * page, (1 << 31) - 256)
    few = _step_shift(R, keys, 64 if d == 128 else 128, Hkv)
    assert few > 0
    ctas = torch.cuda.get_device_properties(0).multi_processor_count
    if max(n for _, n in requests) > 1:
        chunk = _step_shift(R + T // (2 * (128 // G)), keys, 128, Hkv)
        assert chunk > 0 and max(n for _, n in requests) > 32 * 2 * (128 // G)
        assert max(s for s, n in requests if n > 1) > 4 * (128 << chunk)
    else:
        tile = (64 if d == 128 else 128) << few
        assert sum(-(-s // tile) for s, _ in requests) * Hkv > ctas and max(s for s, _ in requests) > 4 * tile
    b = Batch(requests, G * Hkv, Hkv, d, page, seed=21, spare_pages=1)
    wide = torch.full((R, columns), -7, dtype=torch.int32, device="cuda")
    wide[:, :b.table.shape[1]] = b.dev["table"]
    b.dev["table"] = wide
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)
    again = b.call().run()
    assert torch.equal(c.o, again.o) and torch.equal(c.lse, again.lse)


def _relative_error_squared(b, o, rounded):
    """(measured, modelled) squared 2-norm of O's error against 64 bits. The model: a value rounded to bf16 is
    off by a step of 2^-7 m / sqrt(12), m its mantissa's 2^e; over mantissas spread as 1/m, squared and relative
    to the value, 2^-14 / 12 * int_1^2 m^-3 dm / ln 2 = 2^-14 / 12 * 0.541. O's own rounding brings that of
    |O|^2; the weights', independent of one another, that of sum_u p_u^2 |v_u - O|^2 where O is divided by the sum
    of the rounded weights (`rounded`), of sum_u p_u^2 |v_u|^2 where it is divided by that of the exact ones."""
    unit = 2.0 ** -14 / 12 * (3 / 8 / math.log(2))
    off = want_off = 0.0
    G = b.Hq // b.Hkv
    o = o.double().cpu()
    for r, (s, n) in enumerate(b.requests):
        a = int(b.cu[r])
        k, v = (t.double() for t in b.rows[r])
        z = torch.einsum("nhgd,shd->nhgs", b.q[a:a + n].double().view(n, b.Hkv, G, b.d), k) * b.d ** -0.5
        hidden = torch.arange(s)[None] >= (s - n + 1 + torch.arange(n))[:, None]
        p = torch.softmax(z.masked_fill(hidden[:, None, None], -math.inf), -1)
        want = torch.einsum("nhgs,shd->nhgd", p, v)
        off += float((o[a:a + n].view_as(want) - want).square().sum())
        vv = torch.einsum("nhgs,sh->nhg", p * p, v.square().sum(-1))
        if rounded:
            pv = torch.einsum("nhgs,shd->nhgd", p * p, v)
            vv += (p * p).sum(-1) * want.square().sum(-1) - 2 * (pv * want).sum(-1)
        want_off += unit * float(want.square().sum() + vv.sum())
    return off, want_off


@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (16, 16, 64)])
@pytest.mark.parametrize("kind", ["step", "chunk"])
def test_the_error_of_many_rows_is_that_of_its_roundings(kind, Hq, Hkv, d):
    """Beside the bounds per element, which hold the worst of every rounding at once: no more than 1.15 times
    the 2-norm that the roundings of P and O bring."""
    requests = [(900, 1), (2000, 1), (3425, 1), (333, 1)] * 3 if kind == "step" else [(513, 200), (900, 300)]
    b = Batch(requests, Hq, Hkv, d, 64, seed=23)
    c = b.call().run()
    assert status(c) == avtp.OK
    off, model = _relative_error_squared(b, c.o, rounded=kind == "step")
    assert off <= 1.15 ** 2 * model, (off / model) ** 0.5


# ---------------------------------------------------------------- slots
@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in_place"])
@pytest.mark.parametrize("R", [1024, 1025, 2048, 2049, 3000, 5000])
def test_slots_of_many_idle_requests_in_one_cta(R, in_place):
    """A step of 2048 new tokens at most: one CTA over several rounds of requests, and with more of them than its
    shared memory keeps."""
    rng = np.random.default_rng(R)
    new = (rng.random(R) < 0.4).astype(np.int32)
    past = rng.integers(0, 70, R).astype(np.int32)
    past[rng.random(R) < 0.2] = 64  # at the end of a page
    assert 0 < new.sum() <= 2048 - 9
    page, spare = 16, 3
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    have, need = -(-past // page), -(-(past + new) // page)
    n_pages = int(need.sum()) + spare + 2
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((R, int(need.max()) + 1), -5, dtype=np.int32)
    first = np.concatenate([[0], np.cumsum(have)])
    for r in range(R):
        table[r, :have[r]] = ids[first[r]:first[r + 1]]
    free = ids[first[-1]:]
    n = int(cu[-1]) + 9
    dev = {k: torch.from_numpy(x.copy()).cuda() for k, x in dict(cu=cu, past=past, table=table, free=free).items()}
    head = torch.tensor([2], dtype=torch.int32, device="cuda")
    kw = dict(seq_len=dev["past"], free_head_out=head) if in_place else {}
    c = avtp.CacheSlotsCall(dev["cu"], n, page_size=page, n_pages=n_pages, block_table=dev["table"],
                            free_pages=dev["free"], free_head=head, past_len=dev["past"], **kw).run()
    assert status(c) == avtp.OK
    want = slots_plain(cu, past, table, free, 2, page, n)
    assert np.array_equal(c.block_table.cpu().numpy(), want[0])
    assert np.array_equal(c.slot_map.cpu().numpy(), want[1])
    assert np.array_equal(c.seq_len.cpu().numpy(), want[2])
    assert int(c.free_head_out.item()) == want[3]


@pytest.mark.parametrize("new", [40, 3000])
def test_a_write_behind_refused_slots_leaves_the_cache_alone(new):
    """A free list that runs out, found on the device: the slot map that the call made names no slot, whatever its
    memory held before."""
    cache = avtp.PagedCache.new(300, 16, 2, 64)
    for t in (cache.k, cache.v):
        t.fill_(3.0)
    k = torch.ones(new, 2, 64, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    table = torch.full((1, 300), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(2, dtype=torch.int32, device="cuda")
    old = [torch.arange(new, dtype=torch.int32, device="cuda") for _ in range(4)]  # slots of another step
    del old
    slots, _, _ = avtp.cache_slots(cu, new, page_size=16, n_pages=300, block_table=table, free_pages=free)
    avtp.cache_write(cache, slots, k, k)
    assert (cache.k == 3.0).all() and (cache.v == 3.0).all() and (table == -1).all()


# ---------------------------------------------------------------- write
@pytest.mark.parametrize("n", [257, 600, 40000])  # more CTAs than a cluster's, up to several rows a group of lanes
@pytest.mark.parametrize("what", ["slot_end", "slot_negative", "row_end", "row_negative"])
def test_a_large_write_skips_and_records_bad_slots_and_rows(what, n):
    Hkv, d, page = 2, 64, 16
    n_pages = -(-n // page) + 2
    cache = avtp.PagedCache.new(n_pages, page, Hkv, d)
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn(n, Hkv, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:n].to(torch.int32)
    kept = torch.randperm(n, device="cuda", generator=g).to(torch.int32)
    ws = avtp.new_workspace(256)
    for bad in (0, n // 2, n - 1):
        s, i = slots.clone(), kept.clone()
        if what.startswith("slot"):
            s[bad] = n_pages * page if what == "slot_end" else -2
        else:
            i[bad] = n if what == "row_end" else -1
        for t in (cache.k, cache.v):
            t.fill_(3.0)
        c = avtp.CacheWriteCall(cache, s, k, v, kept_idx=i, workspace=ws).run()  # holds the error before
        assert status(c) == avtp.ERR_DEVICE_INPUT
        good = torch.arange(n, device="cuda") != bad
        for pool_, rows in ((cache.k, k), (cache.v, v)):
            want = torch.full_like(pool_, 3.0).view(-1, Hkv, d)
            want[s[good].long()] = rows[i[good].long()]
            assert torch.equal(pool_.view(-1, Hkv, d), want)
    c = avtp.CacheWriteCall(cache, slots, k, v, kept_idx=kept, workspace=ws).run()
    assert status(c) == avtp.OK


@pytest.mark.parametrize("order", ["token", "head"])
def test_a_write_of_tens_of_thousands_of_rows(order):
    """Several rows a group of lanes in every CTA."""
    Hkv, d, page, n, n_rows = 8, 128, 48, 40000, 30000
    n_pages = n // page + 7
    k_pool, v_pool = pool(n_pages, page, Hkv, d, order, fill=3.0)
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(n_rows, Hkv, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:n].to(torch.int32)
    slots[torch.rand(n, device="cuda", generator=g) < 0.1] = -1
    kept = torch.randint(0, n_rows, (n,), device="cuda", generator=g).to(torch.int32)
    want_k, want_v = k_pool.clone(), v_pool.clone()
    live = slots >= 0
    at, row = slots[live].long(), kept[live].long()
    want_k[at // page, at % page] = k[row]
    want_v[at // page, at % page] = v[row]
    c = avtp.CacheWriteCall(avtp.PagedCache(k_pool, v_pool), slots, k, v, kept_idx=kept).run()
    assert status(c) == avtp.OK
    assert torch.equal(k_pool, want_k) and torch.equal(v_pool, want_v)


# ---------------------------------------------------------------- plain launches
def plain_launch_calls():
    """A step's slots, writes and attention of both kernels, one behind the other with nothing waited for between."""
    b = Batch([(700, 130), (3000, 1), (70, 1), (0, 1), (2200, 300)] + [(90, 1)] * 40, 16, 4, 128, 32, seed=31)
    g = torch.Generator(device="cuda").manual_seed(2)
    n, page = 5000, 32
    k, v = (torch.randn(n, 4, 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    cache = avtp.PagedCache(*pool(200, page, 4, 128, fill=0.0))
    table = torch.full((3, 120), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(200, device="cuda", generator=g).to(torch.int32)
    cu = torch.tensor([0, 1500, 1501, 5000], dtype=torch.int32, device="cuda")
    out = []
    for _ in range(3):
        s = avtp.CacheSlotsCall(cu, n, page_size=page, n_pages=200, block_table=table, free_pages=free).run()
        w = [avtp.CacheWriteCall(cache, s.slot_map[:m], k[:m], v[:m]).run() for m in (n, 40)]
        c = b.call().run()
        q = k.repeat_interleave(2, 1)
        a = avtp.CacheAttentionCall(cache, q, cu, s.seq_len, table, max_new=3499).run()
        out.append([s.slot_map, s.seq_len, s.free_head_out, table.clone(), cache.k.clone(), cache.v.clone(), c.o, c.lse,
                    a.o, a.lse])
        for call in (s, *w, c, a):
            assert status(call) == avtp.OK
    return b, out


def test_launches_without_overlap_give_the_same_bits(tmp_path):
    """AVTP_PDL=0, read once a process: every kernel behind the whole of the one before."""
    b, here = plain_launch_calls()
    b.check(here[0][6], here[0][7])
    path = str(tmp_path / "out.pt")
    code = ("import sys, torch\nfrom tests.test_gpu_cache_edges import plain_launch_calls\n"
            "torch.save([[t.cpu() for t in x] for x in plain_launch_calls()[1]], sys.argv[1])\n")
    subprocess.run([sys.executable, "-c", code, path], check=True, cwd=ROOT, timeout=300,
                   env={**os.environ, "AVTP_PDL": "0"})
    there = torch.load(path)
    assert len(there) == len(here) == 3
    for step in (*here, *there):
        for x, y in zip(here[0], step, strict=True):
            assert torch.equal(x.cpu(), y.cpu())


# ---------------------------------------------------------------- the documented calls
def test_the_readme_example_attends_to_the_kept_tokens_and_the_new_ones():
    """The example run as it stands: the new tokens' rows against 64 bits over the kept rows and their own."""
    with open(os.path.join(ROOT, "README.md"), encoding="utf-8") as f:
        code = [c for c in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "cache_attention" in c]
    assert len(code) == 1
    segs = [[("t", 5), ("i", 300), ("t", 9)], [("i", 64), ("t", 7)], [("t", 12), ("i", 500), ("t", 2)]]
    wl = synth.make_custom(segs, keep_ratio=0.3, n_q_heads=32, n_kv_heads=8, head_dim=128, hidden=256, pos_planes=3)
    dw = DevWorkload(wl)
    g = torch.Generator(device="cuda").manual_seed(5)

    def rand(*shape):
        return torch.randn(*shape, device="cuda", generator=g).to(torch.bfloat16)

    R, T, n_pages = 3, wl.layout.n_tokens, 40
    env = dict(q=dw.t["q"], k=dw.t["k"], v=rand(T, 8, 128), h_cur=dw.t["h_cur"], h_prior=dw.t["h_prior"],
               pos=dw.t["pos"], keep_ratio=dw.keep_ratio, keep_ratio_np=wl.keep_ratio, cu_seqlens=wl.layout.cu_seqlens,
               img_cu=wl.layout.img_cu, img_start=wl.layout.img_start, img_len=wl.layout.img_len, n_pages=n_pages,
               table=torch.full((R, 12), -1, dtype=torch.int32, device="cuda"),
               free=torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32),
               q_new=rand(R, 32, 128), k_new=rand(R, 8, 128), v_new=rand(R, 8, 128),
               cu_new=torch.arange(R + 1, dtype=torch.int32, device="cuda"))
    exec(compile(code[0], "README.md", "exec"), env)  # noqa: S102
    kept, cu = env["out"].kept_idx.long(), env["out"].out_cu_seqlens.cpu().numpy()
    rows = [tuple(torch.cat([env[x][kept[cu[r]:cu[r + 1]]], env[x + "_new"][r:r + 1]]).cpu() for x in ("k", "v"))
            for r in range(R)]
    b = Batch.__new__(Batch)
    b.__dict__.update(requests=[(len(kr), 1) for kr, _ in rows], Hq=32, Hkv=8, d=128, cu=np.arange(R + 1),
                      q=env["q_new"].cpu(), rows=rows)
    assert env["seq_len"].tolist() == [s for s, _ in b.requests]
    b.check(env["o"], env["lse"])
