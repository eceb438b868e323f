// Who holds which pages of the paged cache: avtp_cache_fork and avtp_cache_free, on the device, from lengths that
// only the device knows. With P = page_size, S = n_sinks and W = window (0: none):
//   left(n)  = max(0, n - W + 1) / P           the first page that the window of token n needs; 0 without one
//   held(n, h) = { j < ceil(n / P) : j < ceil(S / P) or j >= left(h) }
//   free:  the pages of held(seq, held_len) that are not in held(new, new)
//   fork:  the full pages of held(len, held_len) of the parent, and its last one copied where it is not full
// A call's entries (a request's or child's pages of that kind, in order) are numbered through: a prefix sum over the
// requests, then a binary search an entry.
//
// What bounds it: latency, a chain of dependent loads a round. A call is one cluster of up to kMostCtas CTAs, each of
// which forms the sums for itself, so that barriers part the rounds and nothing else does; a thread's first kKept
// pages stay in its registers from round to round. Everything is checked before the first write. Calls one behind the
// other: 256 requests of 200-8000 tokens on pages of 16, of which 64 are done (14900 pages), 7.0 us; the pages that
// 64 windowed requests have left, with counts (16000 pages, four rounds that touch them in no order), 13.2; eight
// children of a prompt of 146 pages 7.7; 171 children of 64 (21000 entries) 10.9. (Before the look for repeated pages
// these were 5.7, 13.1, 7.7 and 10.8; then, with eight CTAs, 6.8, 19.9, 8.5 and 13.1; with entries looked up again in
// every round, and the others' findings read from their shared memory, 11.7, 36.7, 11.2 and 18.8.)
//
// A page of several holders that rows of a call let go of: every entry counts itself (rel) and the last one in order
// (last: a maximum) stands for the page, so that neither the counts nor the list's order depend on who came first.
// Both arrays are cleared where the call's entries point, not as a whole. A page of one holder has one entry, which
// finds itself in last.
//
// Without counts every page has one entry. That is seen in a bit a page of the pool, spread over the shared memory of
// the cluster and cleared ahead of the wait for the kernel before: an entry sets its page's and looks at what was
// there, ahead of the barrier behind the checks. A word has as few pages as there is room for, since they wait for each
// other (always 32: 17380 pages 8.7 us instead of 7.6). A pool of too many pages (kSeenWords) has last instead, a barrier
// and a trip to L2 more. 32, 367, 4370 and 17380 pages in a graph: 4.5, 5.2, 5.8 and 7.6 us; with last 5.3, 6.2, 6.7 and
// 8.7; without a look 4.3, 4.9, 5.5 and 6.7, and a page that two rows let go of twice in the list.
#include <cooperative_groups.h>

#include "avtp_cache.cuh"

namespace avtp {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 1024;
constexpr int kMostCtas = 16;  // of a cluster where the device has room for that many, else 8
constexpr int64_t kEntriesOfCta = 1024;  // of the table, where fewer CTAs than kMostCtas do
constexpr int kKept = 4;
constexpr int kStaged = 2048;  // requests whose numbers are kept in shared memory
constexpr int64_t kSeenWords = 12288;  // of a CTA, bits of the pool's pages, at most

// What a request or child brings: up to three ranges of table columns.
struct Span {
  int32_t lo[3], n[3];
  __device__ __forceinline__ int64_t total() const { return int64_t(n[0]) + n[1] + n[2]; }
  __device__ __forceinline__ int32_t column(int32_t k) const {
    if (k < n[0]) return lo[0] + k;
    k -= n[0];
    return k < n[1] ? lo[1] + k : lo[2] + k - n[1];
  }
};

struct Pages : CachePages {
  // Pages that a request lets go of: sinks behind its new end, what the window has left, what lies behind the end.
  __device__ __forceinline__ Span gone(int32_t seq, int32_t now, int32_t held) const {
    const int32_t have = up(seq), keep = up(now);
    const int32_t from = min(max(sinks, left(held)), have);                       // held: [0, sinks) and [from, have)
    const int32_t to = now == 0 ? have : min(max(from, max(sinks, left(now))), have);  // kept behind the sinks: [to, keep)
    Span s;
    s.lo[0] = min(sinks, keep);
    s.n[0] = min(sinks, have) - s.lo[0];
    s.lo[1] = from;
    s.n[1] = to - from;
    s.lo[2] = max(keep, to);
    s.n[2] = have - s.lo[2];
    return s;
  }
  // Full pages of the first len tokens that a request holds.
  __device__ __forceinline__ Span full(int32_t len, int32_t held) const {
    const int32_t all = len / P, from = min(max(sinks, left(held)), all);
    Span s;
    s.lo[0] = 0;
    s.n[0] = min(sinks, all);
    s.lo[1] = from;
    s.n[1] = all - from;
    s.lo[2] = 0;
    s.n[2] = 0;
    return s;
  }
};

// What a CTA's checks found, and its pages for the list, for the others of the cluster: every CTA puts its note into
// all the others' shared memory ahead of the barrier. (Reading theirs behind it took 4 us of 18 for sixteen.)
struct Note {
  int err, detail;
  int64_t gives;
  __device__ __forceinline__ void fail(int d) {
    if (atomicExch(&err, 1) == 0) detail = d;
  }
};
// All threads of the cluster, once a call; true if none has failed. Behind it everything written before it is seen.
__device__ bool agree(cg::cluster_group& cluster, Note& mine, Note (&notes)[kMostCtas], int* detail, int64_t* gives,
                      int64_t* before) {
  const int ctas = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
  const int lane = threadIdx.x & 31;
  __syncthreads();
  if (threadIdx.x < ctas) *cluster.map_shared_rank(&notes[rank], threadIdx.x) = mine;
  cluster.sync();
  Note n{0, -1, 0};
  if (lane < ctas) n = notes[lane];
  const unsigned bad = __ballot_sync(0xffffffffu, n.err != 0);
  *detail = bad ? __shfl_sync(0xffffffffu, n.detail, __ffs(bad) - 1) : -1;
  // a call's pages are a 32-bit number
  *gives = __reduce_add_sync(0xffffffffu, static_cast<int>(n.gives));
  *before = __reduce_add_sync(0xffffffffu, lane < rank ? static_cast<int>(n.gives) : 0);
  return bad == 0;
}

// Sets bits of a word in the shared memory of the cluster's CTA `rank`; what was there.
__device__ __forceinline__ uint32_t set_bit(uint32_t* word, uint32_t rank, uint32_t bit) {
  uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(word)), was;
  asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(rank));
  asm volatile("atom.relaxed.cluster.shared::cluster.or.b32 %0, [%1], %2;" : "=r"(was) : "r"(at), "r"(bit) : "memory");
  return was;
}

// Inclusive sums of N numbers a thread over the CTA; totals in all. Two barriers.
template <int N>
__device__ void block_scan(int64_t (&x)[N], int64_t (&s_warp)[N][kThreads / 32], int64_t (&all)[N]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto warp_scan = [&](int64_t v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    return v;
  };
  static_assert(kThreads == 1024, "a warp's lane a warp");
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = warp_scan(x[i]);
  __syncthreads();
  if (lane == 31) {
#pragma unroll
    for (int i = 0; i < N; ++i) s_warp[i][warp] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t sums = warp_scan(s_warp[i][lane]);
    all[i] = __shfl_sync(0xffffffffu, sums, 31);
    const int64_t before = __shfl_sync(0xffffffffu, sums, warp == 0 ? 0 : warp - 1);
    if (warp > 0) x[i] += before;
  }
}

__device__ __forceinline__ int32_t clamped(int64_t x) { return static_cast<int32_t>(x < 0x7fffffff ? x : 0x7fffffff); }

// Calls f(entry, its page, which of the thread's) for entries begin, begin + step, ... < end, with the first kKept
// pages from registers.
template <class P, class F>
__device__ __forceinline__ void each_entry(int64_t begin, int64_t end, int64_t step, const int32_t (&kept)[kKept], P page_of,
                                           F f) {
#pragma unroll
  for (int i = 0; i < kKept; ++i)
    if (begin + i * step < end) f(begin + i * step, kept[i], i);
  for (int64_t e = begin + kKept * step; e < end; e += step) f(e, page_of(e), kKept);
}

// ---------------------------------------------------------------- free
struct FreeDev {
  avtp_cache_free_args_t a;
  Pages pages;
  DevStatus* st;
  int32_t* first;  // [R + 1] where R > kStaged: entries before a request's
  int32_t* rel;    // [n_pages], with counts: entries of a page
  int32_t* last;   // [n_pages]: the last of them
  int seen;        // words of a CTA's share of the pages' bits; 0: last instead
  int seen_sh;     // log2 of the pages of a word
};

__global__ void __launch_bounds__(kThreads) k_cache_free(FreeDev d) {
  __shared__ Note s_v, s_notes[kMostCtas];
  __shared__ int64_t s_warp[1][kThreads / 32];
  __shared__ int32_t s_first[kStaged + 1], s_seq[kStaged], s_now[kStaged], s_held[kStaged];
  extern __shared__ uint32_t s_seen[];  // a bit a page, the words dealt to the CTAs in turn
  for (int i = threadIdx.x; i < d.seen; i += kThreads) s_seen[i] = 0u;
  pdl_wait();
  pdl_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  cluster.barrier_arrive();  // every CTA has started before any other writes into its shared memory
  const avtp_cache_free_args_t& a = d.a;
  const int tid = threadIdx.x, rank = static_cast<int>(cluster.block_rank()), ctas = static_cast<int>(cluster.num_blocks());
  const int R = a.n_requests;
  const Pages& pages = d.pages;
  const bool staged = R <= kStaged;
  const int64_t head = *a.free_head;
  if (tid == 0) s_v = Note{head < 0 || head > a.n_free ? 1 : 0, -1, 0};
  __syncthreads();

  // lengths, and the entries before each request's; none of a request whose lengths are refused
  int64_t total = 0;
  for (int base = 0; base < R; base += kThreads) {
    const int r = base + tid;
    int64_t n = 0;
    int32_t seq = 0, now = 0, held = 0;
    if (r < R) {
      seq = a.seq_len[r];
      now = a.new_len[r];
      held = a.window > 0 ? a.held_len[r] : 0;
      bool bad = seq < 0 || now < 0 || now > seq || held < 0 || held > seq ||
                 seq > static_cast<int64_t>(a.max_pages) * a.page_size;
      if (!bad && pages.lacks(now, held)) bad = true;
      // a new end inside a page that others hold
      if (!bad && a.shared != nullptr && now > 0 && now < seq && now % a.page_size != 0) {
        const int32_t page = a.block_table[r * a.table_stride + now / a.page_size];
        bad = page < 0 || page >= a.n_pages || a.shared[page] > 0;
      }
      if (bad) s_v.fail(r);
      else n = pages.gone(seq, now, held).total();
    }
    int64_t sum[1] = {n}, all[1];
    block_scan(sum, s_warp, all);
    if (r < R) {
      const int32_t before = clamped(total + sum[0] - n);
      if (staged) {
        s_first[r] = before;
        s_seq[r] = seq;
        s_now[r] = now;
        s_held[r] = held;
      } else if (rank == 0) {
        d.first[r] = before;
      }
    }
    total += all[0];
  }
  if (tid == 0) {
    if (staged) s_first[R] = clamped(total);
    else if (rank == 0) d.first[R] = clamped(total);
    if (total > 0x7fffffff) s_v.fail(R);
  }
  if (total > 0x7fffffff) total = 0;
  cluster.barrier_wait();
  if (staged) __syncthreads();
  else cluster.sync();

  // the CTA's entries, in order (an equal share: in whole turns of its threads 4370 pages took 7.0 us instead of 6.4)
  const int64_t each = ((total + ctas - 1) / ctas + 31) / 32 * 32;
  const int64_t e0 = each * rank, e1 = min(total, e0 + each), mine0 = e0 + tid;
  const int32_t* first = staged ? s_first : d.first;
  auto page_of = [&](int64_t e) -> int32_t {
    const int r = upper_index(first, R, e);
    const Span s = staged ? pages.gone(s_seq[r], s_now[r], s_held[r])
                          : pages.gone(a.seq_len[r], a.new_len[r], a.window > 0 ? a.held_len[r] : 0);
    return a.block_table[r * a.table_stride + s.column(static_cast<int32_t>(e - first[r]))];
  };
  int32_t kept[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i) kept[i] = mine0 + i * kThreads < e1 ? page_of(mine0 + i * kThreads) : 0;
  auto entries = [&](auto f) { each_entry(mine0, e1, kThreads, kept, page_of, f); };
  auto in_pool = [&](int32_t page) { return page >= 0 && page < a.n_pages; };
  int32_t others[kKept + 1] = {};  // the pages' holders beyond the first
  auto others_of = [&](int32_t page, int i) { return i < kKept ? others[i] : (a.shared != nullptr ? a.shared[page] : 0); };
#pragma unroll
  for (int i = 0; i < kKept; ++i)
    others[i] = a.shared != nullptr && mine0 + i * kThreads < e1 && in_pool(kept[i]) ? a.shared[kept[i]] : 0;
  int64_t repeated = -1;  // an entry whose page another has
  entries([&](int64_t e, int32_t page, int i) {
    if (!in_pool(page)) {
      s_v.fail(upper_index(first, R, e));
    } else if (d.seen > 0) {
      const uint32_t word = static_cast<uint32_t>(page) >> d.seen_sh, bit = 1u << (page - (word << d.seen_sh));
      if (set_bit(s_seen + word / ctas, word % ctas, bit) & bit) repeated = e;
    } else {
      const int32_t n = others_of(page, i);
      if (n < 0) s_v.fail(upper_index(first, R, e));
      if (n > 0) d.rel[page] = 0;
      d.last[page] = n > 0 ? -1 : static_cast<int32_t>(e);
    }
  });
  if (repeated >= 0) s_v.fail(upper_index(first, R, repeated));
  // What an entry leaves of its page's others, if it stands for the page: -1, it goes to the list. kNone: it does not.
  constexpr int32_t kNone = -2, kWrong = -3;
  auto rest_of = [&](int64_t e, int32_t page, int32_t n) {
    const bool stands = __ldcg(d.last + page) == e;
    if (n <= 0) return stands ? -1 : kWrong;
    const int32_t let_go = __ldcg(d.rel + page);
    return let_go > n + 1 ? kWrong : (stands ? n - let_go : kNone);
  };
  int32_t rest[kKept + 1] = {};
  int64_t mine[1] = {0};
  if (d.seen == 0) {
    cluster.sync();
    if (a.shared != nullptr) {
      entries([&](int64_t e, int32_t page, int i) {
        if (!in_pool(page) || others_of(page, i) <= 0) return;
        atomicAdd(d.rel + page, 1);
        atomicMax(d.last + page, static_cast<int32_t>(e));
      });
      cluster.sync();
    }
    entries([&](int64_t e, int32_t page, int i) {
      if (!in_pool(page)) return;
      const int32_t n = others_of(page, i), left = rest_of(e, page, n);
      // more entries than holders; of one holder, one that finds another
      if (left == kWrong) s_v.fail(upper_index(first, R, e));
      mine[0] += left == -1 ? 1 : 0;
      if (i < kKept) rest[i] = left;
    });
  }
  if (a.shared != nullptr) {
    int64_t all[1];
    block_scan(mine, s_warp, all);
    if (tid == 0) s_v.gives = all[0];
  }
  int detail;
  int64_t gives, at;  // pages that go to the list, and those of the CTAs before
  bool ok = agree(cluster, s_v, s_notes, &detail, &gives, &at);
  if (a.shared == nullptr) gives = total;
  if (ok && gives > head) {
    ok = false;
    detail = R;
  }
  at += head - gives;
  if (ok && a.shared == nullptr) {
    entries([&](int64_t e, int32_t page, int) { a.free_pages[at + e] = page; });
  } else if (ok) {
    for (int64_t b = e0, i = 0; b < e1; b += kThreads, ++i) {
      const int64_t e = b + tid;
      int32_t page = 0, left = kNone, n = 0;
      if (e < e1) {
        if (i < kKept) {
#pragma unroll
          for (int k = 0; k < kKept; ++k)
            if (i == k) page = kept[k], left = rest[k], n = others[k];
        } else {
          page = page_of(e);
          n = a.shared[page];
          left = rest_of(e, page, n);
        }
      }
      const bool give = left == -1;
      if (n > 0 && left >= -1) a.shared[page] = max(left, 0);
      int64_t sum[1] = {give ? 1 : 0}, all[1];
      block_scan(sum, s_warp, all);
      if (give) a.free_pages[at + sum[0] - 1] = page;
      at += all[0];
    }
  }
  // Behind agree() every CTA has its lengths; where they are not in shared memory it looks at them again above.
  if (!staged) cluster.sync();
  if (ok) {
    for (int r = rank * kThreads + tid; r < R; r += ctas * kThreads) {
      const int32_t now = staged ? s_now[r] : a.new_len[r];
      a.seq_len_out[r] = now;
      if (a.window > 0) a.held_len_out[r] = now;
    }
  }
  if (rank == 0 && tid == 0) {
    *d.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, detail, 0u};
    if (ok) *a.free_head_out = static_cast<int32_t>(head - gives);
  }
}

// ---------------------------------------------------------------- fork
struct ForkDev {
  avtp_cache_fork_args_t a;
  Pages pages;
  DevStatus* st;
  int32_t* first;  // [C + 1] where C > kStaged: entries before a child's
  int32_t* fresh;  // [C] there: copied pages before a child's
  int32_t* mark;   // [R]: which child a row is, of parents -1
};

__global__ void __launch_bounds__(kThreads) k_cache_fork(ForkDev d) {
  __shared__ Note s_v, s_notes[kMostCtas];
  __shared__ int64_t s_warp[2][kThreads / 32];
  // a child's numbers: entries before its, its copied page (-1: none), parent, length, the parent's held_len
  __shared__ int32_t s_first[kStaged + 1], s_fresh[kStaged], s_parent[kStaged], s_len[kStaged], s_held[kStaged];
  pdl_wait();
  pdl_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  cluster.barrier_arrive();  // every CTA has started before any other writes into its shared memory
  const avtp_cache_fork_args_t& a = d.a;
  const int tid = threadIdx.x, rank = static_cast<int>(cluster.block_rank()), ctas = static_cast<int>(cluster.num_blocks());
  const int C = a.n_children, P = a.page_size;
  const Pages& pages = d.pages;
  const bool staged = C <= kStaged;
  const int64_t head = a.free_head != nullptr ? *a.free_head : 0;
  if (tid == 0) s_v = Note{head < 0 || head > a.n_free ? 1 : 0, -1, 0};
  __syncthreads();
  auto in_pool = [&](int32_t page) { return page >= 0 && page < a.n_pages; };

  // lengths, the entries before each child's and the copied pages; none of a child that is refused
  int64_t total = 0, copies = 0;
  for (int base = 0; base < C; base += kThreads) {
    const int i = base + tid;
    int64_t n = 0;
    int tail = 0;
    int32_t p = -1, len = 0, held = 0;
    if (i < C) {
      const int32_t c = a.child[i];
      p = a.parent[i];
      bool bad = p < 0 || p >= a.n_requests || c < 0 || c >= a.n_requests;
      if (!bad) {
        const int32_t seq = a.seq_len[p];
        len = a.fork_len != nullptr ? a.fork_len[i] : seq;
        held = a.window > 0 ? a.held_len[p] : 0;
        bad = seq < 0 || len < 0 || len > seq || held < 0 || held > seq ||
              seq > static_cast<int64_t>(a.max_pages) * P || pages.lacks(len, held);
        if (rank == 0) d.mark[p] = -1;
      }
      if (bad) {
        s_v.fail(i);
        p = -1;
      } else {
        n = pages.full(len, held).total();
        tail = len % P != 0 ? 1 : 0;
      }
    }
    int64_t sum[2] = {n, tail}, all[2];
    block_scan(sum, s_warp, all);
    if (i < C) {
      const int32_t before = clamped(total + sum[0] - n), page = static_cast<int32_t>(copies + sum[1] - 1);
      if (staged) {
        s_first[i] = before;
        s_fresh[i] = tail ? page : -1;
        s_parent[i] = p;
        s_len[i] = len;
        s_held[i] = held;
      } else if (rank == 0) {
        d.first[i] = before;
        d.fresh[i] = tail ? page : -1;
      }
    }
    total += all[0];
    copies += all[1];
  }
  if (tid == 0) {
    if (staged) s_first[C] = clamped(total);
    else if (rank == 0) d.first[C] = clamped(total);
    if (total > 0x7fffffff || head + copies > a.n_free) s_v.fail(C);
  }
  const bool countable = total <= 0x7fffffff && head >= 0 && head + copies <= a.n_free;
  if (!countable) total = 0;
  cluster.barrier_wait();
  if (staged) __syncthreads();
  else cluster.sync();

  const int32_t* first = staged ? s_first : d.first;
  struct Child {
    int32_t parent, len, held, fresh;  // parent -1: refused
  };
  auto child_of = [&](int i) {
    if (staged) return Child{s_parent[i], s_len[i], s_held[i], s_fresh[i]};
    const int32_t p = a.parent[i];
    if (p < 0 || p >= a.n_requests) return Child{-1, 0, 0, -1};
    return Child{p, a.fork_len != nullptr ? a.fork_len[i] : a.seq_len[p], a.window > 0 ? a.held_len[p] : 0, d.fresh[i]};
  };
  // a child's copied page: the parent's last, and the list's
  auto tail_of = [&](const Child& k, int32_t* from, int32_t* to) {
    *from = *to = -1;
    if (k.parent < 0 || k.fresh < 0) return false;
    *from = a.block_table[k.parent * a.table_stride + k.len / P];
    *to = a.free_pages[head + k.fresh];
    return true;
  };
  const int64_t step = static_cast<int64_t>(ctas) * kThreads, at = rank * kThreads + tid;
  auto page_of = [&](int64_t e) {
    const int i = upper_index(first, C, e);
    const Child k = child_of(i);
    return a.block_table[k.parent * a.table_stride + pages.full(k.len, k.held).column(static_cast<int32_t>(e - first[i]))];
  };
  int32_t kept[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i) kept[i] = at + i * step < total ? page_of(at + i * step) : 0;
  auto entries = [&](auto f) { each_entry(at, total, step, kept, page_of, f); };
  int32_t from0 = -1, to0 = -1;  // of the thread's first child
  if (countable) {
    for (int64_t i = at; i < C; i += step) {
      int32_t from, to;
      if (tail_of(child_of(static_cast<int>(i)), &from, &to) && (!in_pool(from) || !in_pool(to))) s_v.fail(static_cast<int>(i));
      if (i == at) from0 = from, to0 = to;
    }
  }
  // every child once, and none of them a parent: the first CTA's to see
  if (rank == 0) {
    __syncthreads();
    auto rows_fine = [&](int i) {
      const int32_t p = a.parent[i], c = a.child[i];
      return p >= 0 && p < a.n_requests && c >= 0 && c < a.n_requests;
    };
    for (int i = tid; i < C; i += kThreads)
      if (rows_fine(i)) d.mark[a.child[i]] = i;
    __syncthreads();
    for (int i = tid; i < C; i += kThreads)
      if (rows_fine(i) && (d.mark[a.child[i]] != i || d.mark[a.parent[i]] != -1)) s_v.fail(i);
  }
  entries([&](int64_t e, int32_t page, int) {
    if (!in_pool(page)) s_v.fail(upper_index(first, C, e));
  });
  int detail;
  int64_t none, before;
  const bool ok = agree(cluster, s_v, s_notes, &detail, &none, &before);
  // parents' rows and lengths are read, children's written: no row is both
  if (ok) {
    entries([&](int64_t e, int32_t page, int) {
      const int i = upper_index(first, C, e);
      const Child k = child_of(i);
      const int32_t column = pages.full(k.len, k.held).column(static_cast<int32_t>(e - first[i]));
      a.block_table[a.child[i] * a.table_stride + column] = page;
      atomicAdd(a.shared + page, 1);
    });
    for (int64_t i = at; i < C; i += step) {
      const Child k = child_of(static_cast<int>(i));
      const int32_t c = a.child[i];
      int32_t from = from0, to = to0;
      if (i != at) tail_of(k, &from, &to);
      if (to >= 0) a.block_table[c * a.table_stride + k.len / P] = to;
      a.copy_src[i] = from;
      a.copy_dst[i] = to;
      a.seq_len[c] = k.len;
      if (a.window > 0) a.held_len[c] = min(k.held, k.len);  // of a prefix shorter than that: the same pages
    }
  }
  if (rank == 0 && tid == 0) {
    *d.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, detail, 0u};
    if (ok && a.free_head_out != nullptr) *a.free_head_out = static_cast<int32_t>(head + copies);
  }
}

// A cluster of as many CTAs as the table's entries give work. `shape` sets what follows from their number, and returns
// the bytes of dynamic shared memory, kMostBytes at most.
template <size_t kMostBytes, class Dev, class F>
cudaError_t launch(void (*kernel)(Dev), PerDevice& most, Dev d, int64_t entries, F shape, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  auto of = [&](int ctas) {
    cfg.gridDim = dim3(ctas);
    attr[0].val.clusterDim.x = ctas;
  };
  int room = 0;
  const cudaError_t e = once_per_device(most, [&](int, int* value) {
    *value = 8;
    cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (set == cudaSuccess && kMostBytes > 0)
      set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMostBytes));
    if (set != cudaSuccess) return set;
    int clusters = 0;
    of(kMostCtas);
    cfg.dynamicSmemBytes = kMostBytes;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0) *value = kMostCtas;
    else cudaGetLastError();
    return cudaSuccess;
  }, &room);
  if (e != cudaSuccess) return e;
  int ctas = 1;
  while (ctas < room && entries > ctas * kEntriesOfCta) ctas *= 2;
  of(ctas);
  cfg.dynamicSmemBytes = shape(ctas, d);
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, d);
}

}  // namespace

cudaError_t launch_cache_free(const avtp_cache_free_args_t& a, void* ws, const FreeWs& p, cudaStream_t s) {
  const FreeDev d{a, {CachePages::of(a.page_size, a.window, a.n_sinks)}, ws_at<DevStatus>(ws, p.status),
                  ws_at<int32_t>(ws, p.first), ws_at<int32_t>(ws, p.rel), ws_at<int32_t>(ws, p.last), 0, 0};
  static PerDevice most;
  auto shape = [](int ctas, FreeDev& f) -> size_t {
    const int64_t pages = (f.a.n_pages + ctas - 1) / ctas;
    while (f.seen_sh < 5 && pages > kSeenWords << f.seen_sh) ++f.seen_sh;
    const int64_t words = (((f.a.n_pages - 1) >> f.seen_sh) + ctas) / ctas;
    f.seen = f.a.shared == nullptr && words <= kSeenWords ? static_cast<int>(words) : 0;
    return f.seen * 4;
  };
  return launch<kSeenWords * 4>(k_cache_free, most, d, static_cast<int64_t>(a.n_requests) * a.max_pages, shape, s);
}

cudaError_t launch_cache_fork(const avtp_cache_fork_args_t& a, void* ws, const ForkWs& p, cudaStream_t s) {
  const ForkDev d{a, {CachePages::of(a.page_size, a.window, a.n_sinks)}, ws_at<DevStatus>(ws, p.status),
                  ws_at<int32_t>(ws, p.first), ws_at<int32_t>(ws, p.fresh), ws_at<int32_t>(ws, p.mark)};
  static PerDevice most;
  auto none = [](int, ForkDev&) -> size_t { return 0; };
  return launch<0>(k_cache_fork, most, d, static_cast<int64_t>(a.n_children) * a.max_pages, none, s);
}

}  // namespace avtp
