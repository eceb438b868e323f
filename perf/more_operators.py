"""More operators of the paged cache whose time is followed: what happens to a step's queries and keys
before its attention, attention in a sliding window, and the pages' upkeep.

* ``rope``: the norms of queries and keys for each head and their rotary positions in one pass, the keys
  and values to their slots of the cache, or the keys to rows;
* ``window``: the step's queries over the cache, each over its last keys and the first few tokens (sinks);
* ``compact``: the kept tokens' rows of cached requests to pages of their own;
* ``fork``: requests that go on from the same cached prompt share its pages, and copy the last one;
* ``free``: the pages of finished, cut and windowed requests back to the free list.

``own`` false computes them by elementary torch operations; ``own`` true calls the library. A case is a
batch drawn from the case's own numbers and the heads of a layer. Values come from the seed.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import numpy as np
import torch

own = False
DEV = "cuda"

# query heads, KV heads, head_dim: layers of the repository's workloads, and generic ones
TINY = dict(q_heads=4, kv_heads=2, head_dim=64)
SEVEN = dict(q_heads=28, kv_heads=4, head_dim=128)
FOUR = dict(q_heads=32, kv_heads=8, head_dim=128)
PLAIN = dict(q_heads=16, kv_heads=16, head_dim=64)
SHARED = dict(q_heads=8, kv_heads=1, head_dim=128)


def rope(layout, tokens, *, style="half", rot, planes=1, norm=True, cache=True, first=0, factor=1.0, base=10000.0,
         page=64):
    """``rot`` dimensions of a head are rotated; positions begin at ``first`` and are divided by ``factor``."""
    return dict(op="rope", layout=layout, tokens=tokens, style=style, rot=rot, planes=planes, norm=norm, cache=cache,
                first=first, factor=factor, base=base, page=page)


def batch(op, layout, requests, past, new, page, **more):
    """``past`` and ``new``: the least and the most of a request (of a request's cached and new tokens, or of
    what the operator names)."""
    return dict(op=op, layout=layout, requests=requests, past_min=past[0], past_max=past[1], new_min=new[0],
                new_max=new[1], page=page, **more)


def listed() -> List[Dict]:
    def case(name, shape, b):
        return dict(name=name, **shape, **b)

    return [
        # the next token of 64 requests behind pruned prompts: normed, rotated and written to its page
        case("rope_step", FOUR, rope(1, 64, rot=128, planes=3, first=3000, base=5e6)),
        # a prompt of sixteen images, positions in three planes (time, height, width)
        case("rope_prefill", FOUR, rope(2, 9856, rot=128, planes=3, base=5e6)),
        # half of each small head, interleaved pairs, positions far out and scaled, keys to rows
        case("rope_part", PLAIN, rope(3, 4097, style="interleaved", rot=32, norm=False, cache=False, first=1000000,
                                      factor=8.0)),
        # a serving batch generating in a window, ragged, padded to a captured batch size
        case("window_step", SEVEN, batch("window", 4, 64, (200, 8000), (1, 1), 16, window=1024, sinks=4, idle=3)),
        # unpruned video: eight requests of up to 65 thousand cached tokens, of which a step sees few
        case("window_long", FOUR, batch("window", 5, 8, (30000, 65000), (1, 1), 128, window=4096, sinks=64, idle=0)),
        # the largest: most of a long prompt in one chunk
        case("window_prefill", FOUR, batch("window", 6, 1, (2176, 2176), (8192, 8192), 64, window=2048, sinks=16, idle=0)),
        # the images of four cached prompts pruned to a third once the question is known
        case("compact_prompts", FOUR, batch("compact", 7, 4, (8500, 8700), (2800, 3000), 64)),
        # many short requests in small pages, half of each kept
        case("compact_short", PLAIN, batch("compact", 8, 16, (100, 900), (40, 100), 16)),
        # eight questions about one pruned prompt
        case("fork_one", FOUR, batch("fork", 9, 1, (9300, 9300), (8, 8), 64)),
        # several answers sampled for each request of a batch
        case("fork_batch", SEVEN, batch("fork", 10, 64, (200, 4000), (1, 4), 16)),
        # a serving batch's end of step: one request in four is done, others take drafted tokens back
        case("free_step", FOUR, batch("free", 11, 256, (200, 8000), (1, 5), 16, window=0, sinks=0, held=False)),
        # pages that the window has left, some of them shared by forked requests
        case("free_window", SEVEN, batch("free", 12, 64, (2000, 30000), (0, 3), 16, window=1024, sinks=4, held=True)),
    ]


def draw(rng: random.Random) -> Dict:
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def ragged(top):  # least and most
        return (rng.randint(max(1, top // 8), top), top)

    op = rng.choice(["rope", "rope", "window", "window", "window", "compact", "fork", "free"])
    shape = rng.choice([TINY, SEVEN, FOUR, PLAIN, SHARED])
    page = rng.choice([16, 32, 48, 64, 128])
    layout = rng.randrange(1 << 30)
    if op == "rope":
        tokens, d = log_uniform(1, 16384), shape["head_dim"]
        return dict(**shape, **rope(layout, tokens, style=rng.choice(["half", "interleaved"]),
                                    rot=rng.choice([d, d, d // 2, d // 4, 24]), planes=rng.choice([1, 3]),
                                    norm=rng.random() < 0.6, cache=rng.random() < 0.6, first=log_uniform(1, 4000000),
                                    factor=rng.choice([1.0, 4.0, 32.0]), base=rng.choice([1e4, 5e5, 5e6]), page=page))
    if op == "window":
        window, sinks = log_uniform(1, 8192), rng.choice([0, 1, 4, rng.randint(5, 300)])
        how = rng.choice(["step", "draft", "chunk", "chunk"])
        if how != "chunk":
            requests, n = log_uniform(1, 128), 1 if how == "step" else rng.randint(2, 16)
            past = ragged(log_uniform(16, min(65000, 500000 // requests)))
            return dict(**shape, **batch(op, layout, requests, past, (n, n), page, window=window, sinks=sinks,
                                         idle=rng.choice([0, 0, 1])))
        requests = rng.randint(1, 8)
        new = log_uniform(17, 6000 // requests)
        past = log_uniform(1, min(20000, 40000000 // (requests * new)))
        return dict(**shape, **batch(op, layout, requests, ragged(past), (max(17, new // 2), new), page, window=window,
                                     sinks=sinks, idle=0))
    if op == "compact":
        requests = log_uniform(1, 64)
        past = log_uniform(20, max(40, 65536 // requests))
        keep = rng.randint(1, past)
        return dict(**shape, **batch(op, layout, requests, ragged(past), (max(1, keep // 2), keep), page))
    if op == "fork":
        requests = log_uniform(1, 64)
        return dict(**shape, **batch(op, layout, requests, ragged(log_uniform(20, max(40, 131072 // requests))),
                                     (0, rng.randint(1, 8)), page))
    requests, held = log_uniform(1, 512), rng.random() < 0.5
    past = ragged(log_uniform(20, max(40, 1000000 // requests)))
    return dict(**shape, **batch(op, layout, requests, past, (0, rng.randint(1, 8)), page,
                                 window=log_uniform(16, 4096) if held else 0, sinks=rng.choice([0, 4, 100]) if held else 0,
                                 held=held))


# ---------------------------------------------------------------- the batch
def lengths(case: Dict):
    """Cached tokens of every request, and its other number (int64 arrays)."""
    rng = random.Random(case["layout"])
    R = case["requests"]
    past = np.asarray([rng.randint(case["past_min"], case["past_max"]) for _ in range(R)], dtype=np.int64)
    new = np.asarray([rng.randint(case["new_min"], case["new_max"]) for _ in range(R)], dtype=np.int64)
    return past, new


def visible(case: Dict):
    """``window``: cached tokens with the new ones (nothing of an idle request), and new tokens."""
    past, new = lengths(case)
    total = past + new
    if case["idle"] and case["idle"] < len(total):
        total[-case["idle"]:] = 0
    return total, new


def children(case: Dict):
    """``fork``: the parent of every child. Parents are rows 0 .. R-1 of the table, children the rows behind."""
    _, n = lengths(case)
    return np.repeat(np.arange(case["requests"]), n) if n.sum() else np.asarray([0])


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def ceil_div(x, p):
    return -(-x // p)


def tables(needs, most, gen, spare):
    """Block tables for requests of ``needs`` pages each (-1 behind them; a column more than the ``most`` that
    they may have), pages in no order: (table, pages in the pool, pages that no request holds)."""
    width, n_pages = int(most.max()) + 1, int(most.sum()) + spare
    needs = torch.from_numpy(np.asarray(needs, dtype=np.int64)).to(DEV)
    total = int(needs.sum())
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    j = torch.arange(width, device=DEV)
    at = ((torch.cumsum(needs, 0) - needs)[:, None] + j).clamp(max=n_pages - 1)
    table = torch.where(j < needs[:, None], order[at], torch.full_like(order[at], -1))
    return table.contiguous(), n_pages, order[total:].contiguous()


def pools(case, x, n_pages, gen):
    for n in ("k", "v"):
        x["pool_" + n] = torch.randn(n_pages, case["page"], case["kv_heads"], case["head_dim"], device=DEV,
                                     dtype=torch.bfloat16, generator=gen)



def inputs(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return dict(rope=rope_inputs, window=window_inputs, compact=compact_inputs, fork=fork_inputs,
                free=free_inputs)[case["op"]](case, seed, gen)


def rope_inputs(case, seed, gen):
    T, Hq, Hkv, d, P, rot = (case[n] for n in ("tokens", "q_heads", "kv_heads", "head_dim", "page", "rot"))
    x = {}
    for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv)):
        x[n] = torch.randn(T, h, d, device=DEV, generator=gen).mul_(2.0).to(torch.bfloat16)
    if case["norm"]:
        for n in ("q_norm", "k_norm"):
            x[n] = (1 + 0.2 * torch.randn(d, device=DEV, generator=gen)).to(torch.bfloat16)
    # text runs on in every plane; images (here stretches of 600 tokens) take rows and columns in two of them
    t = torch.arange(T, device=DEV)
    pos = case["first"] + t
    rows = [pos] if case["planes"] == 1 else [pos, pos - t % 600 + t % 600 // 24, pos - t % 600 + t % 24]
    x["pos"] = torch.stack(rows).to(torch.int32)
    inv = case["base"] ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot) / case["factor"]
    x["inv_freq"] = inv.to(torch.float32).to(DEV)
    x["mscale"] = 0.1 * math.log(case["factor"]) + 1.0
    x["plane"] = i32(np.arange(rot // 2) * case["planes"] // (rot // 2))
    if case["cache"]:
        n_pages = ceil_div(T, P) + 8
        order = torch.randperm(n_pages, generator=gen, device=DEV)
        x["slots"] = (order[t // P] * P + t % P).to(torch.int32)
        for n in ("k", "v"):
            x["pool_" + n] = torch.zeros(n_pages, P, Hkv, d, device=DEV, dtype=torch.bfloat16)
    return x


def window_inputs(case, seed, gen):
    total, new = visible(case)
    T, d = int(new.sum()), case["head_dim"]
    needs = ceil_div(total, case["page"])
    table, n_pages, _ = tables(needs, needs, gen, 8)
    x = dict(cu=i32(np.concatenate([[0], np.cumsum(new)])), n_tokens=T, table=table, seq=i32(total),
             max_new=int(new.max()))
    # keys and queries of unit variance, a few of the queries sharper than the others
    x["q"] = (torch.randn(T, case["q_heads"], d, device=DEV, generator=gen)
              * torch.exp(0.5 * torch.randn(T, case["q_heads"], 1, device=DEV, generator=gen))).to(torch.bfloat16)
    pools(case, x, n_pages, gen)
    return x


def compact_inputs(case, seed, gen):
    past, keep = lengths(case)
    keep = np.minimum(keep, past)
    R, P = case["requests"], case["page"]
    needs, to = ceil_div(past, P), ceil_div(keep, P)
    needs = np.concatenate([needs, to])
    both, n_pages, _ = tables(needs, needs, gen, 4)
    # the kept positions of each request, ascending, as a selection gives them
    u = torch.rand(R, int(past.max()), generator=gen, device=DEV)
    lens, n = (torch.from_numpy(v).to(DEV)[:, None] for v in (past, keep))
    u = torch.where(torch.arange(u.shape[1], device=DEV) < lens, u, torch.full_like(u, 2.0))
    at = u.argsort(1)
    at = torch.where(torch.arange(u.shape[1], device=DEV) < n, at, torch.full_like(at, 1 << 30)).sort(1).values
    x = dict(seq=i32(past), table=both[:R].contiguous(), to=both[R:].contiguous(),
             keep_cu=i32(np.concatenate([[0], np.cumsum(keep)])), keep=at[at < 1 << 30].to(torch.int32))
    pools(case, x, n_pages, gen)
    return x


def fork_inputs(case, seed, gen):
    past, _ = lengths(case)
    # a seed of its own moves the lengths a little, which are this operator's values
    R, P, parent = case["requests"], case["page"], children(case)
    C = len(parent)
    most = ceil_div(past + 2, P)
    past = past + np.random.RandomState(seed % (1 << 32)).randint(0, 3, len(past))
    needs = np.concatenate([ceil_div(past, P), np.zeros(C, dtype=np.int64)])
    table, n_pages, free = tables(needs, most, gen, C + 8)
    x = dict(table=table, seq=i32(np.concatenate([past, np.zeros(C)])), parent=i32(parent), child=i32(R + np.arange(C)),
             n_pages=n_pages, free=free, head=i32([3]), shared=torch.zeros(n_pages, dtype=torch.int32, device=DEV))
    x["shared_before"] = x["shared"].clone()
    pools(case, x, n_pages, gen)
    return x


def free_inputs(case, seed, gen):
    past, cut = lengths(case)
    R, P = case["requests"], case["page"]
    most = ceil_div(past + 2, P)
    past = past + np.random.RandomState(seed % (1 << 32)).randint(0, 3, len(past))
    done = np.arange(R) % 4 == 1
    new = np.where(done, 0, np.maximum(past - cut, 1))
    needs = ceil_div(past, P)
    table, n_pages, rest = tables(needs, most, gen, 8)
    taken = int(needs.sum())
    x = dict(table=table, n_pages=n_pages, seq=i32(past), new=i32(new), head=i32([taken]),
             free=torch.cat([torch.full((taken,), -1, dtype=torch.int32, device=DEV), rest]))
    if case["held"]:
        # pages left behind at an earlier step are no longer the request's
        x["held"] = i32(np.maximum(np.minimum(past, new + (new == 0) * past) - 700, 0))
        # every second request shares the pages of its first half with the one before, up to the cut
        full = np.minimum(past // 2, np.roll(past, 1) // 2) // P
        with_last = torch.from_numpy(np.where(np.arange(R) % 2 == 1, full, 0)).to(DEV)
        take = torch.arange(table.shape[1], device=DEV) < with_last[:, None]
        x["table"] = torch.where(take, table.roll(1, 0), table).contiguous()
        # such a pair left the same pages behind
        both = x["held"].clone()
        both[0::2][:R // 2] = torch.minimum(x["held"][0::2][:R // 2], x["held"][1::2])
        both[1::2] = both[0::2][:R // 2]
        x["held"] = both
        first = left_of(both.long(), case)
        j = torch.arange(table.shape[1], device=DEV)
        sinks = ceil_div(case["sinks"], P)
        owned = (j < torch.from_numpy(needs).to(DEV)[:, None]) & ((j < sinks) | (j >= first[:, None]))
        at = torch.where(owned, x["table"], torch.full_like(table, n_pages)).long().view(-1)
        holders = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV).index_add_(
            0, at, torch.ones(at.numel(), dtype=torch.int32, device=DEV))[:n_pages]
        x["shared_before"] = (holders - 1).clamp(min=0)
        x["shared"] = x["shared_before"].clone()
    return x


def left_of(length, case):
    return ((length - case["window"] + 1).clamp(min=0) // case["page"] if case["window"] else torch.zeros_like(length))


def prepare(case: Dict, seed: int):
    x = inputs(case, seed)
    state = dict(case=case, x=x)
    if own:  # the prepared calls, their outputs and workspaces, which a serving program keeps
        from paper_2608_26806_gb300 import avtp

        cache = avtp.PagedCache(x["pool_k"], x["pool_v"]) if "pool_k" in x else None
        op = case["op"]
        if op == "rope":
            state["call"] = avtp.RopeCall(
                x["pos"], x["inv_freq"], q=x["q"], k=x["k"], v=x["v"] if cache else None, style=case["style"],
                pair_plane=x["plane"], attn_factor=x["mscale"], q_norm=x.get("q_norm"), k_norm=x.get("k_norm"), eps=1e-6,
                cache=cache, slot_map=x.get("slots"))
        elif op == "window":
            state["call"] = avtp.CacheAttentionCall(cache, x["q"], x["cu"], x["seq"], x["table"], max_new=x["max_new"],
                                                    window=case["window"], sinks=case["sinks"])
        elif op == "compact":
            state["call"] = avtp.CacheCompactCall(cache, x["keep_cu"], x["keep"], x["seq"], x["table"], dst_table=x["to"])
        elif op == "fork":
            state["call"] = avtp.CacheForkCall(x["parent"], x["child"], x["seq"], x["table"], page_size=case["page"],
                                               n_pages=x["n_pages"], free_pages=x["free"], free_head=x["head"],
                                               shared=x["shared"])
            state["copy"] = avtp.CacheCopyCall(cache, state["call"].copy_src, state["call"].copy_dst)
        else:
            more = dict(window=case["window"], sinks=case["sinks"], held_len=x["held"],
                        shared=x["shared"]) if case["held"] else {}
            state["call"] = avtp.CacheFreeCall(x["seq"], x["new"], x["table"], page_size=case["page"],
                                               n_pages=x["n_pages"], free_pages=x["free"], free_head=x["head"], **more)
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    case, x = state["case"], state["x"]
    op = case["op"]
    if "shared" in x:  # as it is before every such step
        x["shared"].copy_(x["shared_before"])
    if own:
        c = state["call"].run()
        if op == "rope":
            return dict(q=c.q_out, k=x["pool_k"], v=x["pool_v"]) if case["cache"] else dict(q=c.q_out, k=c.k_out)
        if op == "window":
            return dict(o=c.o, lse=c.lse)
        if op == "compact":
            return dict(k=x["pool_k"], v=x["pool_v"])
        if op == "fork":
            state["copy"].run()
            return dict(table=x["table"], seq=x["seq"], shared=x["shared"], head=c.free_head_out, src=c.copy_src,
                        dst=c.copy_dst, k=x["pool_k"], v=x["pool_v"])
        got = dict(free=x["free"], head=c.free_head_out, seq=c.seq_len_out)
        return dict(got, held=c.held_out, shared=x["shared"]) if case["held"] else got
    return dict(rope=plain_rope, window=plain_window, compact=plain_compact, fork=plain_fork,
                free=plain_free)[op](case, x)


def plain_rope(case, x):
    rot, half = case["rot"], case["rot"] // 2
    # positions of each pair's plane; angles in 64 bits, since far ones have none left for their fraction
    angle = x["pos"].double()[x["plane"].long()].t() * x["inv_freq"].double()
    cos, sin = ((f(angle) * x["mscale"]).float()[:, None] for f in (torch.cos, torch.sin))

    def rotated(t, weight):
        t = t.float()
        if weight is not None:
            t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * weight.float()
        r = t[..., :rot]
        a, b = (r[..., :half], r[..., half:]) if case["style"] == "half" else (r[..., 0::2], r[..., 1::2])
        c, s = a * cos - b * sin, b * cos + a * sin
        r = torch.cat([c, s], -1) if case["style"] == "half" else torch.stack([c, s], -1).flatten(-2)
        return torch.cat([r, t[..., rot:]], -1).to(torch.bfloat16)

    q, k = rotated(x["q"], x.get("q_norm")), rotated(x["k"], x.get("k_norm"))
    if not case["cache"]:
        return dict(q=q, k=k)
    at, shape = x["slots"].long(), (-1, case["kv_heads"], case["head_dim"])
    x["pool_k"].view(shape)[at] = k
    x["pool_v"].view(shape)[at] = x["v"]
    return dict(q=q, k=x["pool_k"], v=x["pool_v"])


def plain_window(case, x):
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
    at = ((seq - new)[:, None] + i)[:, :, None]  # a query's own place among the cached tokens
    j = torch.arange(z.shape[-1], device=DEV)
    hidden = (j > at) | (j >= seq[:, None, None]) | ((j <= at - case["window"]) & (j >= case["sinks"]))
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


def plain_compact(case, x):
    P, cu, idx = case["page"], x["keep_cu"].long(), x["keep"].long()
    t = torch.arange(idx.shape[0], device=DEV)
    req = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    j = t - cu[req]
    src, dst = x["table"].long()[req, idx // P], x["to"].long()[req, j // P]
    for n in ("k", "v"):
        x["pool_" + n][dst, j % P] = x["pool_" + n][src, idx % P]
    return dict(k=x["pool_k"], v=x["pool_v"])


def plain_fork(case, x):
    P, parent, child = case["page"], x["parent"].long(), x["child"].long()
    length = x["seq"].long()[parent]
    full, tail = length // P, length % P > 0
    j = torch.arange(x["table"].shape[1], device=DEV)
    of_parent = x["table"][parent]
    ends = torch.cumsum(tail, 0)
    fresh = x["free"][x["head"].long() + ends - tail.long()]
    rows = torch.where(j < full[:, None], of_parent, x["table"][child])
    rows = torch.where((j == full[:, None]) & tail[:, None], fresh[:, None], rows)
    x["table"][child] = rows
    x["seq"][child] = length.to(torch.int32)
    at = torch.where(j < full[:, None], of_parent, torch.full_like(of_parent, x["n_pages"])).long().view(-1)
    shared = torch.cat([x["shared"], x["shared"][:1]]).index_add_(
        0, at, torch.ones(at.numel(), dtype=torch.int32, device=DEV))[:-1]
    none = torch.full_like(fresh, -1)
    last = of_parent.gather(1, full[:, None].clamp(max=of_parent.shape[1] - 1))[:, 0]
    src, dst = torch.where(tail, last, none), torch.where(tail, fresh, none)
    # copies of nothing go from and to the page behind the last child's
    spare = x["free"][x["head"].long() + len(parent)]
    a, b = torch.where(tail, last, spare).long(), torch.where(tail, fresh, spare).long()
    for n in ("k", "v"):
        x["pool_" + n][b] = x["pool_" + n][a]
    x["shared"].copy_(shared)
    return dict(table=x["table"], seq=x["seq"], shared=x["shared"], head=(x["head"] + ends[-1]).to(torch.int32), src=src,
                dst=dst, k=x["pool_k"], v=x["pool_v"])


def plain_free(case, x):
    P, seq, new, n_pages = case["page"], x["seq"].long(), x["new"].long(), x["n_pages"]
    sinks = ceil_div(case["sinks"], P)
    j = torch.arange(x["table"].shape[1], device=DEV)
    before, after = (left_of(n, case)[:, None] for n in ((x["held"].long() if case["held"] else seq * 0), new))
    had = (j < ((seq + P - 1) // P)[:, None]) & ((j < sinks) | (j >= before))
    keeps = (j < ((new + P - 1) // P)[:, None]) & ((j < sinks) | (j >= after))
    gone = (had & ~keeps).view(-1)
    page = torch.where(gone, x["table"].view(-1), torch.full_like(x["table"].view(-1), n_pages)).long()
    if case["held"]:
        # the last holder to let go of a page, in the order of the table, gives it back
        ones = gone.to(torch.int32)
        rest = torch.cat([x["shared"], x["shared"][:1]]).index_add_(0, page, -ones)
        e = torch.arange(page.numel(), device=DEV)
        last = torch.full((n_pages + 1,), -1, device=DEV).scatter_reduce_(0, page, e, "amax")
        gives = gone & (rest[page] == -1) & (last[page] == e)
        x["shared"].copy_(rest[:-1].clamp(min=0))
    else:
        gives = gone
    rank = torch.cumsum(gives, 0)
    head = x["head"].long() - rank[-1]
    at = torch.where(gives, head + rank - 1, torch.full_like(rank, x["free"].shape[0]))
    free = torch.cat([x["free"], x["free"][:1]]).scatter_(0, at, page.to(torch.int32))[:-1]
    got = dict(free=free, head=head.to(torch.int32), seq=x["new"].clone())
    return dict(got, held=x["new"].clone(), shared=x["shared"]) if case["held"] else got


# ---------------------------------------------------------------- what a pass cannot do without
def work(case: Dict) -> Dict[str, float]:
    P, Hq, Hkv, d, op = case["page"], case["q_heads"], case["kv_heads"], case["head_dim"], case["op"]
    if op == "rope":
        T = case["tokens"]
        rows = Hq + Hkv + (Hkv if case["cache"] else 0)
        return dict(bytes=4.0 * T * rows * d + 4.0 * T * (case["planes"] + case["cache"]),
                    flops=T * (Hq + Hkv) * (3.0 * case["rot"] + (4.0 * d if case["norm"] else 0)))
    if op == "window":
        total, new = visible(case)
        W, S = case["window"], case["sinks"]
        keys = pairs = 0.0
        for t, n in zip(total.tolist(), new.tolist()):
            at = t - n + np.arange(n)
            at = at[at >= 0]
            if len(at):
                near = np.maximum(at - W + 1, 0)  # the first key of each query's window
                pairs += float((at + 1 - near + np.minimum(near, S)).sum())
                keys += t - near[0] + min(near[0], S)
        T = float(new.sum())
        return dict(bytes=4.0 * d * Hkv * keys + T * Hq * (4.0 * d + 4.0) + 4.0 * keys / P, flops=4.0 * d * Hq * pairs)
    past, n = lengths(case)
    if op == "compact":
        kept = float(np.minimum(past, n).sum())
        return dict(bytes=8.0 * kept * Hkv * d + 4.0 * kept, flops=0.0)
    if op == "fork":
        parent = children(case)
        pages = float((past[parent] // P).sum())
        tails = float((past[parent] % P > 0).sum())
        return dict(bytes=8.0 * tails * P * Hkv * d + 16.0 * pages, flops=pages)
    R = case["requests"]
    done = np.arange(R) % 4 == 1
    gone = float(ceil_div(past, P)[done].sum())
    return dict(bytes=(16.0 if case["held"] else 8.0) * gone + 16.0 * R, flops=gone)


# ---------------------------------------------------------------- the same in 64 bits
def exact(case: Dict, seed: int):
    op = case["op"]
    if op == "free":
        return None  # whole numbers
    x = inputs(case, seed)
    if op == "rope":
        return exact_rope(case, x)
    if op == "window":
        return exact_window(case, x)
    P, got = case["page"], {}
    for n in ("k", "v"):
        pool, was = x["pool_" + n].double(), x["pool_" + n]
        if op == "compact":
            cu, idx = x["keep_cu"].tolist(), x["keep"].long()
            for r in range(case["requests"]):
                a, b = cu[r], cu[r + 1]
                j = torch.arange(b - a, device=DEV)
                rows = was[x["table"][r].long()[idx[a:b] // P], idx[a:b] % P]
                pool[x["to"][r].long()[j // P], j % P] = rows.double()
        else:
            seq, free, head = x["seq"].tolist(), x["free"].tolist(), int(x["head"])
            for p in x["parent"].tolist():
                if seq[p] % P:
                    pool[free[head]] = was[int(x["table"][p, seq[p] // P])].double()
                    head += 1
        got[n] = pool
    return got if op == "compact" else dict(table=None, seq=None, shared=None, head=None, src=None, dst=None, **got)


def exact_rope(case, x):
    """Each pair as a complex number, turned by its angle."""
    T, rot = case["tokens"], case["rot"]
    angle = torch.empty(T, rot // 2, dtype=torch.float64, device=DEV)
    for i, p in enumerate(x["plane"].tolist()):
        angle[:, i] = x["pos"][p].double() * float(x["inv_freq"][i])
    turn = torch.polar(torch.full_like(angle, x["mscale"]), angle)[:, None]
    pairs = torch.arange(rot, device=DEV)
    pairs = pairs.view(2, -1).t() if case["style"] == "half" else pairs.view(-1, 2)
    out = {}
    for n in ("q", "k"):
        t = x[n].double()
        if case["norm"]:
            t = t / torch.sqrt(t.square().sum(-1, keepdim=True) / case["head_dim"] + 1e-6) * x[n + "_norm"].double()
        z = torch.view_as_complex(t[..., pairs].contiguous()) * turn
        t = t.clone()
        t[..., pairs[:, 0]], t[..., pairs[:, 1]] = z.real, z.imag
        out[n] = t
    if case["cache"]:
        at, P = x["slots"].long(), case["page"]
        for n, rows in (("k", out["k"]), ("v", x["v"].double())):
            pool = x["pool_" + n].double()
            pool[at // P, at % P] = rows
            out[n] = pool
    return out


def exact_window(case, x):
    Hq, Hkv, d, P, W, S = (case[n] for n in ("q_heads", "kv_heads", "head_dim", "page", "window", "sinks"))
    total, new = visible(case)
    o = torch.zeros(x["n_tokens"], Hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((Hq, x["n_tokens"]), -math.inf, dtype=torch.float64, device=DEV)
    a = 0
    for r, (t, n) in enumerate(zip(total.tolist(), new.tolist())):
        if t:
            at = x["table"][r, :ceil_div(t, P)].long()
            k = x["pool_k"][at].reshape(-1, Hkv, d)[:t].double()
            v = x["pool_v"][at].reshape(-1, Hkv, d)[:t].double()
            for h in range(Hq):
                kh, vh = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
                for c in range(0, n, 2048):
                    e = min(n, c + 2048)
                    z = x["q"][a + c:a + e, h].double() @ kh.T / math.sqrt(d)
                    back = (t - n + torch.arange(c, e, device=DEV))[:, None] - torch.arange(t, device=DEV)[None]
                    z[back < 0] = -math.inf
                    z[:, S:][back[:, S:] >= W] = -math.inf
                    norm = torch.logsumexp(z, 1)
                    lse[h, a + c:a + e] = norm
                    o[a + c:a + e, h] = torch.exp(z - norm.clamp(min=-1e300)[:, None]) @ vh
        a += n
    return dict(o=o, lse=lse)
