"""The paged cache on the GPU: what lies outside the requests' tokens, bounds far above them, and the
forms of slots and writes that large calls take."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp, synth
from tests.cache_util import Batch
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
