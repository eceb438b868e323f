"""The paged cache's operators in plain 64-bit form, and batches to run them on."""
import math

import numpy as np
import torch

from paper_2608_26806_gb300 import avtp

NAN = float("nan")


def pool(n_pages, page, Hkv, d, order="token", gen=None, fill=NAN, dev="cuda"):
    """K and V pools holding ``fill`` everywhere, as views [n_pages, page, Hkv, d] of pages in the
    given order: "token" or "head" major, "shared" (K and V of a page side by side), "padded" (token
    strides longer than the heads) or "mixed" (K token-major, V head-major)."""
    def one(how):
        if how == "head":
            return torch.full((n_pages, Hkv, page, d), fill, dtype=torch.bfloat16, device=dev).transpose(1, 2)
        if how == "padded":
            return torch.full((n_pages, page + 1, Hkv * d + 24), fill, dtype=torch.bfloat16,
                              device=dev)[:, :page, :Hkv * d].unflatten(2, (Hkv, d))
        return torch.full((n_pages, page, Hkv, d), fill, dtype=torch.bfloat16, device=dev)

    if order == "shared":
        both = torch.full((n_pages, 2, page, Hkv, d), fill, dtype=torch.bfloat16, device=dev)
        return both[:, 0], both[:, 1]
    if order == "mixed":
        return one("token"), one("head")
    return one(order), one(order)


class Batch:
    """Requests of (cached, new) tokens, cached ones counting the new, on pages in random order."""

    def __init__(self, requests, Hq, Hkv, d, page, order="token", seed=0, tail=0, spare_pages=3, k_scale=1.0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.requests, self.Hq, self.Hkv, self.d, self.page = requests, Hq, Hkv, d, page
        seq = [s for s, _ in requests]
        new = [n for _, n in requests]
        R = len(requests)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T = int(self.cu[-1]) + tail
        need = [-(-s // page) for s in seq]
        n_pages = sum(need) + spare_pages
        ids = torch.randperm(n_pages, generator=g)
        self.table = torch.full((R, max(need + [1]) + 1), -7, dtype=torch.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = ids[at:at + n].to(torch.int32)
            at += n
        k, v = pool(n_pages, page, Hkv, d, order)
        self.rows = []  # (k, v) of every request's cached tokens, on the CPU
        for r, s in enumerate(seq):
            kr = (k_scale * torch.randn(s, Hkv, d, generator=g)).to(torch.bfloat16)
            vr = torch.randn(s, Hkv, d, generator=g).to(torch.bfloat16)
            self.rows.append((kr, vr))
            if s:
                p = torch.arange(s)
                page_id, off = self.table[r, p // page].long().cuda(), (p % page).cuda()
                k[page_id, off] = kr.cuda()
                v[page_id, off] = vr.cuda()
        self.cache = avtp.PagedCache(k, v)
        self.q = torch.randn(self.T, Hq, d, generator=g).to(torch.bfloat16)
        self.max_new = max(new + [1])
        self.dev = dict(q=self.q.cuda(), cu=torch.from_numpy(self.cu).cuda(),
                        seq=torch.tensor(seq, dtype=torch.int32).cuda(), table=self.table.cuda())

    def call(self, **kw):
        kw.setdefault("max_new", self.max_new)
        d = self.dev
        return avtp.CacheAttentionCall(self.cache, d["q"], d["cu"], d["seq"], d["table"], **kw)

    def check(self, o, lse, scale=None):
        """O and LSE of every row against 64 bits.

        Bounds, per element, with A = sum_u p_u |v_u| (p the 64-bit probabilities), n the keys of the
        row and S the largest sum |q_i k_i| scale of it. P is rounded to bf16, each weight off by
        d_u, |d_u| <= 2^-8. Divided by the sum of the exact weights, O is off by sum p_u d_u v_u, at
        most 2^-8 A; divided by the sum of the rounded ones, by sum p_u d_u (v_u - O) to first order,
        at most 2^-8 (A + |O|). O's own rounding adds 2^-8 |O|. Second order: a factor 1 + 2^-7. A
        logit is d fp32 products and sums, off by at most e = (d + 4) 2^-24 S, times 2 in a ratio of
        exponentials; the exponential itself 2^-22, twice; sums of n terms n 2^-24, twice. ln(sum) is
        off by e, the sum's relative error, and three roundings of numbers no larger than |lse| + S +
        ln n.
        """
        scale = scale if scale is not None else self.d ** -0.5
        o, lse = o.float().cpu().double(), None if lse is None else lse.cpu().double()
        G = self.Hq // self.Hkv
        for r, (s, n) in enumerate(self.requests):
            a = int(self.cu[r])
            if n == 0:
                continue
            k, v = (t.double() for t in self.rows[r])
            q = self.q[a:a + n].double().view(n, self.Hkv, G, self.d)
            z = torch.einsum("nhgd,shd->nhgs", q, k) * scale
            S = (torch.einsum("nhgd,shd->nhgs", q.abs(), k.abs()) * scale)
            seen = (s - n + 1 + torch.arange(n)).clamp(min=0)
            hidden = torch.arange(s)[None] >= seen[:, None]
            z.masked_fill_(hidden[:, None, None], -math.inf)
            S.masked_fill_(hidden[:, None, None], 0.0)
            S = S.amax(-1) if s else torch.zeros(n, self.Hkv, G, dtype=torch.float64)
            norm = torch.logsumexp(z, -1) if s else torch.full((n, self.Hkv, G), -math.inf, dtype=torch.float64)
            p = torch.exp(z - norm[..., None])
            p = torch.where(torch.isnan(p), torch.zeros_like(p), p)
            want = torch.einsum("nhgs,shd->nhgd", p, v).reshape(n, self.Hq, self.d)
            A = torch.einsum("nhgs,shd->nhgd", p, v.abs()).reshape(n, self.Hq, self.d)
            e = (self.d + 4) * 2.0 ** -24 * S.reshape(n, self.Hq)
            cnt = seen.double()[:, None]
            tol = (2.0 ** -8 * (1 + 2.0 ** -7) * (A + 2 * want.abs())
                   + A * (2 * e + 2.0 ** -21 + 2 * cnt * 2.0 ** -24)[..., None])
            got = o[a:a + n]
            assert torch.isfinite(got).all(), f"request {r}: not finite"
            off = (got - want).abs() - tol
            assert off.max() <= 0, f"request {r}: O off by {float((got - want).abs().max())}"
            if lse is not None:
                ref, got = norm.reshape(n, self.Hq), lse[:, a:a + n].t()
                empty = torch.isinf(ref)
                assert torch.equal(torch.isinf(got), empty) and (got[empty] < 0).all()
                size = ref.abs() + S.reshape(n, self.Hq) + torch.log(cnt.clamp(min=1))
                tol = e + 2.0 ** -22 + cnt * 2.0 ** -24 + 4 * 2.0 ** -24 * size
                off = ((got - ref).abs() - tol)[~empty]
                assert off.numel() == 0 or off.max() <= 0, f"request {r}: LSE off"


def slots_plain(cu, past, table, free, head, page, n_tokens):
    """avtp_cache_slots one token at a time: (table, slots, seq_len, head)."""
    table, head = table.copy(), int(head)
    slots = np.full(n_tokens, -1, dtype=np.int32)
    seq = np.zeros(len(past), dtype=np.int32)
    for r in range(len(past)):
        pos = int(past[r])
        pages = -(-pos // page)
        for t in range(int(cu[r]), int(cu[r + 1])):
            if pos // page >= pages:
                table[r, pages] = free[head]
                pages, head = pages + 1, head + 1
            slots[t] = table[r, pos // page] * page + pos % page
            pos += 1
        seq[r] = pos
    return table, slots, seq, head
