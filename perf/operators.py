"""The paged-cache operators whose time is followed: slots, writes and attention over the cache.

A program that serves pruned requests keeps each layer's keys and values in a cache of pages:

* ``slots``: block tables, slot maps and lengths of a step's new tokens, from the lengths alone;
* ``write``: the step's K and V rows, for a pruned prefill only the kept ones, to their slots;
* ``attention``: the step's queries over the cache, a chunk of new tokens or a single one a request.

``own`` false computes them by elementary torch operations in 32 bits; ``own`` true calls the
library. A case is a batch (requests of ``past`` cached and ``new`` tokens, drawn from the case's
own numbers) and the heads of the model's layer. Values come from the seed.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import numpy as np
import torch

own = False
DEV = "cuda"

# query heads, KV heads, head_dim of the models' layers, and generic ones: no groups, one KV head
TINY = dict(q_heads=4, kv_heads=2, head_dim=64)
LLAVA = dict(q_heads=28, kv_heads=4, head_dim=128)
QWEN = dict(q_heads=32, kv_heads=8, head_dim=128)
PLAIN = dict(q_heads=16, kv_heads=16, head_dim=64)
SHARED = dict(q_heads=8, kv_heads=1, head_dim=128)


def batch(layout, requests, past, new, page, chunks=0, idle=0):
    """``past`` and ``new``: the least and the most of a request. With ``chunks``, only that many
    requests have ``new`` tokens, the others one; ``idle``: the last that many hold nothing, as
    the padding of a captured batch does."""
    return dict(layout=layout, requests=requests, past_min=past[0], past_max=past[1], new_min=new[0],
                new_max=new[1], page=page, chunks=chunks, idle=idle)


def listed() -> List[Dict]:
    def case(name, op, shape, **b):
        return dict(name=name, op=op, **shape, **b)

    return [
        # the smallest call: the next token of eight requests; a few lengths, latency is all of it
        case("slots_step", "slots", QWEN, **batch(1, 8, (300, 5000), (1, 1), 64)),
        # a prefill of many ragged requests in small pages
        case("slots_prefill", "slots", QWEN, **batch(2, 256, (0, 0), (16, 1024), 16)),
        # the next token of 64 requests: two rows of a layer each
        case("write_step", "write", LLAVA, **batch(3, 64, (200, 8000), (1, 1), 16)),
        # the kept rows of four pruned requests of 64 large images, out of all their rows
        case("write_pruned", "write", QWEN, **batch(4, 4, (0, 0), (8500, 8700), 64)),
        # one chat request generating, its sixteen images pruned to a third
        case("attend_one", "attention", QWEN, **batch(5, 1, (3424, 3424), (1, 1), 64)),
        # a serving batch generating, ragged, seven heads a group, padded to a captured batch size
        case("attend_serving", "attention", LLAVA, **batch(6, 64, (200, 8000), (1, 1), 16, idle=3)),
        # unpruned video: eight requests of up to 65 thousand cached tokens
        case("attend_long", "attention", QWEN, **batch(7, 8, (30000, 65000), (1, 1), 128)),
        # several drafted tokens a request checked at once
        case("attend_draft", "attention", QWEN, **batch(8, 16, (700, 4000), (5, 5), 32)),
        # the smallest chunk, of small heads
        case("attend_chunk_tiny", "attention", TINY, **batch(9, 2, (30, 190), (33, 70), 16)),
        # a follow-up question with an image behind one request's cached prompt
        case("attend_chunk", "attention", QWEN, **batch(10, 1, (9300, 9300), (512, 512), 64)),
        # chunked prefill beside generation: two requests of the batch prefill, the others generate
        case("attend_mixed", "attention", LLAVA, **batch(11, 24, (500, 3800), (400, 513), 32, chunks=2)),
        # the largest: most of a long prompt in one chunk
        case("attend_prefill", "attention", QWEN, **batch(12, 1, (2176, 2176), (8192, 8192), 64)),
    ]


def draw(rng: random.Random) -> Dict:
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["slots", "write", "attention", "attention", "attention", "attention"])
    shape = rng.choice([TINY, LLAVA, QWEN, PLAIN, SHARED])
    page = rng.choice([16, 32, 48, 64, 128])
    layout = rng.randrange(1 << 30)

    def ragged(top):  # least and most
        return (rng.randint(max(0, top // 8), top), top)

    if op == "slots":
        requests = log_uniform(1, 512)
        return dict(op=op, **shape, **batch(layout, requests, ragged(log_uniform(1, 8000)),
                                            (1, log_uniform(1, max(1, 131072 // requests))), page))
    if op == "write":
        requests = log_uniform(1, 64)
        return dict(op=op, **shape, **batch(layout, requests, ragged(log_uniform(1, 2000)),
                                            (1, log_uniform(1, max(1, 32768 // requests))), page))
    how = rng.choice(["step", "step", "draft", "chunk", "chunk", "mixed"])
    if how in ("step", "draft"):
        requests = log_uniform(1, 128)
        past = ragged(log_uniform(16, min(65000, 500000 // requests)))
        n = 1 if how == "step" else rng.randint(2, 16)
        return dict(op=op, **shape, **batch(layout, requests, past, (n, n), page, idle=rng.choice([0, 0, 1])))
    requests = rng.randint(1, 8) if how == "chunk" else rng.randint(2, 24)
    new = log_uniform(17, 6000 // requests)
    past = log_uniform(1, min(20000, 40000000 // (requests * new)))  # fewer logits than the largest case
    return dict(op=op, **shape, **batch(layout, requests, ragged(past), (max(17, new // 2), new), page,
                                        chunks=0 if how == "chunk" else rng.randint(1, 2)))


# ---------------------------------------------------------------- the batch
def lengths(case: Dict):
    """Cached and new tokens of every request (int64 arrays)."""
    rng = random.Random(case["layout"])
    R = case["requests"]
    past = np.asarray([rng.randint(case["past_min"], case["past_max"]) for _ in range(R)], dtype=np.int64)
    new = np.asarray([rng.randint(case["new_min"], case["new_max"]) for _ in range(R)], dtype=np.int64)
    if case["chunks"]:
        new[case["chunks"]:] = 1
    return past, new


def visible(case: Dict):
    """Cached tokens with the new ones (attention: nothing of an idle request), and new tokens."""
    past, new = lengths(case)
    total = past + new
    if case["idle"] and case["idle"] < len(total):
        total[-case["idle"]:] = 0
    return total, new


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def pages_of(total, case, gen):
    """(block table [R, W], pages in the pool, pages not in the table): the pages of a pool that
    requests have taken and returned for a while, in no order."""
    P, R = case["page"], case["requests"]
    need = -(-total // P)
    W = int(need.max()) + 1
    n_pages = int(need.sum()) + 8
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    first = torch.from_numpy(np.cumsum(need) - need).to(DEV)
    j = torch.arange(W, device=DEV)
    at = (first[:, None] + j).clamp(max=n_pages - 1)
    table = torch.where(j < torch.from_numpy(need).to(DEV)[:, None], order[at], torch.full_like(order[at], -1))
    return table.contiguous(), n_pages, order[int(need.sum()):].contiguous()


def inputs(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device=DEV).manual_seed(seed)
    past, new = lengths(case)
    P, Hq, Hkv, d = case["page"], case["q_heads"], case["kv_heads"], case["head_dim"]
    cu = np.concatenate([[0], np.cumsum(new)])
    T = int(cu[-1])
    x = dict(cu=i32(cu), n_tokens=T)
    if case["op"] == "slots":
        # the past tokens' pages are in the table, the new ones come from the free list; a seed of
        # its own moves a few lengths, which are this operator's values
        past = past + np.random.RandomState(seed % (1 << 32)).randint(0, 3, len(past))
        need = -(-(past + new) // P)
        have = -(-past // P)
        n_pages = int(need.sum()) + 8
        W = int(need.max()) + 2
        order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
        first = torch.from_numpy(np.cumsum(have) - have).to(DEV)
        j = torch.arange(W, device=DEV)
        at = (first[:, None] + j).clamp(max=n_pages - 1)
        table = torch.where(j < torch.from_numpy(have).to(DEV)[:, None], order[at], torch.full_like(order[at], -1))
        taken = int(have.sum())
        x.update(past=i32(past), table=table.contiguous(), n_pages=n_pages, free=order[taken:].contiguous(),
                 head=i32([3]))
        return x
    total, new = visible(case)
    if case["op"] == "write":
        table, n_pages, _ = pages_of(past + new, case, gen)
        # kept rows out of about three times as many, ascending
        rows = 3 * T
        kept = torch.randperm(rows, generator=gen, device=DEV)[:T].sort().values.to(torch.int32)
        t = torch.arange(T, device=DEV)
        req = torch.repeat_interleave(torch.arange(len(new), device=DEV), torch.from_numpy(new).to(DEV))
        pos = torch.from_numpy(past).to(DEV)[req] + t - x["cu"].long()[req]
        x["slots"] = (table.long()[req, pos // P] * P + pos % P).to(torch.int32)
        x["kept"] = kept
        for n in ("k", "v"):
            x[n] = torch.randn(rows, Hkv, d, device=DEV, dtype=torch.bfloat16, generator=gen)
            x["pool_" + n] = torch.zeros(n_pages, P, Hkv, d, device=DEV, dtype=torch.bfloat16)
        return x
    table, n_pages, _ = pages_of(total, case, gen)
    x.update(table=table, n_pages=n_pages, seq=i32(total), max_new=int(new.max()))
    # keys and queries of unit variance, a few of the queries sharper than the others
    x["q"] = (torch.randn(T, Hq, d, device=DEV, generator=gen)
              * torch.exp(0.5 * torch.randn(T, Hq, 1, device=DEV, generator=gen))).to(torch.bfloat16)
    for n in ("k", "v"):
        x["pool_" + n] = torch.randn(n_pages, P, Hkv, d, device=DEV, dtype=torch.bfloat16, generator=gen)
    return x


def prepare(case: Dict, seed: int):
    x = inputs(case, seed)
    state = dict(case=case, x=x)
    if own:  # the prepared call, its outputs and its workspace, which a serving program keeps
        from paper_2608_26806_gb300 import avtp

        if case["op"] == "slots":
            state["call"] = avtp.CacheSlotsCall(x["cu"], x["n_tokens"], page_size=case["page"], n_pages=x["n_pages"],
                                                block_table=x["table"], free_pages=x["free"], free_head=x["head"],
                                                past_len=x["past"])
        else:
            cache = avtp.PagedCache(x["pool_k"], x["pool_v"])
            if case["op"] == "write":
                state["call"] = avtp.CacheWriteCall(cache, x["slots"], x["k"], x["v"], kept_idx=x["kept"])
            else:
                state["call"] = avtp.CacheAttentionCall(cache, x["q"], x["cu"], x["seq"], x["table"],
                                                        max_new=x["max_new"])
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    case, x = state["case"], state["x"]
    if own:
        c = state["call"].run()
        if case["op"] == "slots":
            return dict(table=c.block_table, slots=c.slot_map, seq=c.seq_len, head=c.free_head_out)
        if case["op"] == "write":
            return dict(k=c.cache.k, v=c.cache.v)
        return dict(o=c.o, lse=c.lse)
    return dict(slots=plain_slots, write=plain_write, attention=plain_attention)[case["op"]](case, x)


def plain_slots(case, x):
    P, cu, past = case["page"], x["cu"].long(), x["past"].long()
    total = past + cu[1:] - cu[:-1]
    have, need = (past + P - 1) // P, (total + P - 1) // P
    ends = torch.cumsum(need - have, 0)
    first = x["head"].long() + ends - (need - have)
    j = torch.arange(x["table"].shape[1], device=DEV)
    fresh = (j >= have[:, None]) & (j < need[:, None])
    at = (first[:, None] + j - have[:, None]).clamp(0, x["free"].shape[0] - 1)
    table = torch.where(fresh, x["free"][at], x["table"])
    t = torch.arange(x["n_tokens"], device=DEV)
    req = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=len(total) - 1)
    pos = past[req] + t - cu[req]
    slots = torch.where(t < cu[-1], table[req, pos // P].long() * P + pos % P, torch.full_like(pos, -1))
    return dict(table=table, slots=slots.to(torch.int32), seq=total.to(torch.int32),
                head=(x["head"].long() + ends[-1]).to(torch.int32))


def plain_write(case, x):
    at, kept = x["slots"].long(), x["kept"].long()
    shape = (-1, case["kv_heads"], case["head_dim"])
    x["pool_k"].view(shape)[at] = x["k"][kept]
    x["pool_v"].view(shape)[at] = x["v"][kept]
    return dict(k=x["pool_k"], v=x["pool_v"])


def plain_attention(case, x):
    """Requests padded to the longest: their queries to max_new tokens, their keys to the table's width."""
    Hq, Hkv, d, P = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    cu, seq, R, N = x["cu"].long(), x["seq"].long(), case["requests"], x["max_new"]
    new = cu[1:] - cu[:-1]
    i = torch.arange(N, device=DEV)
    rows = (cu[:-1, None] + i).clamp(max=x["n_tokens"] - 1)
    q = x["q"].float()[rows].view(R, N, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(R, Hkv, -1, d)
    pages = x["table"].long().clamp(min=0)
    k = x["pool_k"][pages].view(R, -1, Hkv, d).permute(0, 2, 3, 1).float()
    z = torch.matmul(q * d ** -0.5, k).view(R, Hkv, Hq // Hkv, N, -1)
    del k
    limit = (seq - new)[:, None] + i + 1  # keys that each new token sees
    j = torch.arange(z.shape[-1], device=DEV)
    hidden = (j >= limit[:, :, None]) | (j >= seq[:, None, None])
    z.masked_fill_(hidden[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = z.sub_(m).exp_()
    s = p.sum(-1, keepdim=True)
    v = x["pool_v"][pages].view(R, -1, Hkv, d).permute(0, 2, 1, 3).float()
    v = torch.where((j < seq[:, None])[:, None, :, None], v, torch.zeros((), device=DEV))
    o = torch.matmul(p.view(R, Hkv, -1, p.shape[-1]), v).view(R, Hkv, Hq // Hkv, N, d)
    o = o / torch.where(s > 0, s, torch.ones_like(s))
    lse = (m + s.log())[..., 0]
    t = torch.arange(x["n_tokens"], device=DEV)
    req = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    at = t - cu[req]
    o = o.permute(0, 3, 1, 2, 4).reshape(R, N, Hq, d)[req, at]
    lse = lse.permute(0, 3, 1, 2).reshape(R, N, Hq)[req, at]
    return dict(o=o.to(torch.bfloat16), lse=lse.t().contiguous())


# ---------------------------------------------------------------- what a pass cannot do without
def work(case: Dict) -> Dict[str, float]:
    past, new = lengths(case)
    P, Hq, Hkv, d = case["page"], case["q_heads"], case["kv_heads"], case["head_dim"]
    R, T = case["requests"], float(new.sum())
    if case["op"] == "slots":
        take = float((-(-(past + new) // P) - -(-past // P)).sum())
        return dict(bytes=4.0 * (2 * R + 2) + 8.0 * take + 4.0 * R + 4.0 * T + 4, flops=4.0 * T)
    if case["op"] == "write":
        return dict(bytes=8.0 * T * Hkv * d + 8.0 * T, flops=0.0)
    total, new = visible(case)
    nbytes = 4.0 * d * Hkv * float(total.sum()) + T * Hq * (4.0 * d + 4.0) + 4.0 * float((-(-total // P)).sum())
    pairs = 0.0
    for t, n in zip(total, new):  # the i-th of n new tokens sees t - n + i + 1 keys
        seen = np.clip(t - n + 1 + np.arange(n), 0, None)
        pairs += float(seen.sum())
    return dict(bytes=nbytes, flops=4.0 * d * Hq * pairs)


# ---------------------------------------------------------------- the same in 64 bits
def exact(case: Dict, seed: int):
    x = inputs(case, seed)
    if case["op"] == "slots":
        return None  # whole numbers
    Hq, Hkv, d, P = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    if case["op"] == "write":
        got = {}
        for n in ("k", "v"):
            pool = x["pool_" + n].double()
            pool[x["slots"].long() // P, x["slots"].long() % P] = x[n].double().index_select(0, x["kept"].long())
            got[n] = pool
        return got
    total, new = visible(case)
    o = torch.zeros(x["n_tokens"], Hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((Hq, x["n_tokens"]), -math.inf, dtype=torch.float64, device=DEV)
    a = 0
    for r, (t, n) in enumerate(zip(total.tolist(), new.tolist())):
        if t:
            at = x["table"][r, :-(-t // P)].long()
            k = x["pool_k"][at].reshape(-1, Hkv, d)[:t].double()
            v = x["pool_v"][at].reshape(-1, Hkv, d)[:t].double()
            for h in range(Hq):
                kh, vh = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
                for c in range(0, n, 2048):
                    e = min(n, c + 2048)
                    z = x["q"][a + c:a + e, h].double() @ kh.T / math.sqrt(d)
                    later = torch.arange(t, device=DEV)[None] > (t - n + torch.arange(c, e, device=DEV))[:, None]
                    z = z.masked_fill(later, -math.inf)
                    norm = torch.logsumexp(z, 1)
                    lse[h, a + c:a + e] = norm
                    o[a + c:a + e, h] = torch.exp(z - norm.clamp(min=-1e300)[:, None]) @ vh
        a += n
    return dict(o=o, lse=lse)
