// Who holds which pages of the paged cache: avtp_cache_fork and avtp_cache_free, on the device, from lengths that
// only the device knows. With P = page_size, S = n_sinks and W = window (0: none):
//   left(n)  = max(0, n - W + 1) / P           the first page that the window of token n needs; 0 without one
//   held(n, h) = { j < ceil(n / P) : j < ceil(S / P) or j >= left(h) }
//   free:  the pages of held(seq, held_len) that are not in held(new, new)
//   fork:  the full pages of held(len, held_len) of the parent, and its last one copied where it is not full
// A call's entries (a request's or child's pages of that kind, in order) are numbered through: a prefix sum over the
// requests, then a binary search an entry.
//
// What bounds it: latency, three to five rounds of dependent loads, so that a call is one cluster of kCtas CTAs, whose
// barriers (1 us less than a grid's each) part the rounds. Everything is checked before the first write.
//
// A page that several rows of a call let go of: every entry counts itself (rel) and the last one in order (last: a maximum)
// stands for the page, so that neither the counts nor the list's order depend on who came first. Both arrays are
// cleared where the call's entries point, not as a whole.
#include <cooperative_groups.h>

#include "avtp_cache.cuh"

namespace avtp {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 1024;
constexpr int kCtas = 8;
constexpr int kStaged = 2048;  // requests whose numbers are kept in shared memory

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

// What a round of checks found, in a CTA's shared memory, read by all behind a barrier. A flag a round: one that
// the next round could set while a slower CTA still reads it would part the CTAs, and the next barrier not end.
constexpr int kRounds = 3;
struct Verdict {
  int err[kRounds], detail[kRounds];
  __device__ __forceinline__ void fail(int round, int d) {
    if (atomicExch(&err[round], 1) == 0) detail[round] = d;
  }
};
// All threads of the cluster; true if none has failed in this round. Behind it everything written before it is seen.
__device__ bool agree(cg::cluster_group& cluster, Verdict& mine, int round, int* detail) {
  cluster.sync();
  bool ok = true;
  for (int c = 0; c < kCtas; ++c) {
    const Verdict* v = cluster.map_shared_rank(&mine, c);
    if (v->err[round]) {
      if (ok) *detail = v->detail[round];
      ok = false;
    }
  }
  return ok;
}

// Inclusive sum over the CTA; total in *all. Two barriers.
__device__ int64_t block_scan(int64_t x, int64_t* s_warp, int64_t* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  int64_t before = 0, sum = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += s_warp[w];
    sum += s_warp[w];
  }
  *all = sum;
  return before + x;
}

// ---------------------------------------------------------------- free
struct FreeDev {
  avtp_cache_free_args_t a;
  Pages pages;
  DevStatus* st;
  int32_t* first;  // [R + 1] where R > kStaged: entries before a request's
  int32_t* rel;    // [n_pages]: entries of a page
  int32_t* last;   // [n_pages]: the last of them
};

__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads) k_cache_free(FreeDev d) {
  __shared__ Verdict s_v;
  __shared__ int64_t s_warp[kThreads / 32], s_gives;
  __shared__ int32_t s_first[kStaged + 1];
  pdl_wait();
  pdl_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  const avtp_cache_free_args_t& a = d.a;
  const int tid = threadIdx.x, rank = static_cast<int>(cluster.block_rank());
  const int R = a.n_requests;
  const Pages& pages = d.pages;
  const bool staged = R <= kStaged;
  int32_t* first = staged ? s_first : d.first;
  const int64_t head = *a.free_head;
  if (tid == 0) s_v = Verdict{{head < 0 || head > a.n_free ? 1 : 0, 0, 0}, {-1, -1, -1}};
  __syncthreads();

  // lengths, and the entries before each request's (where they go to memory the first CTA writes them)
  int64_t total = 0;
  for (int base = 0; base < R; base += kThreads) {
    const int r = base + tid;
    int64_t n = 0;
    if (r < R) {
      const int32_t seq = a.seq_len[r], now = a.new_len[r], held = a.window > 0 ? a.held_len[r] : 0;
      bool bad = seq < 0 || now < 0 || now > seq || held < 0 || held > seq ||
                 seq > static_cast<int64_t>(a.max_pages) * a.page_size;
      if (!bad && now > 0 && pages.left(now) < pages.left(held)) bad = true;  // it would need pages let go of
      // a new end inside a page that others hold
      if (!bad && a.shared != nullptr && now > 0 && now < seq && now % a.page_size != 0) {
        const int32_t page = a.block_table[r * a.table_stride + now / a.page_size];
        bad = page < 0 || page >= a.n_pages || a.shared[page] > 0;
      }
      if (bad) s_v.fail(0, r);
      else n = pages.gone(seq, now, held).total();
    }
    int64_t all;
    const int64_t incl = block_scan(n, s_warp, &all);
    const int64_t before = total + incl - n;
    if (r < R && (staged || rank == 0)) first[r] = static_cast<int32_t>(before < 0x7fffffff ? before : 0x7fffffff);
    total += all;
  }
  if (tid == 0 && (staged || rank == 0)) first[R] = static_cast<int32_t>(total < 0x7fffffff ? total : 0x7fffffff);
  if (total > 0x7fffffff && tid == 0) s_v.fail(0, R);
  int detail = -1;
  bool ok = agree(cluster, s_v, 0, &detail);

  // the CTA's entries, in order
  const int64_t each = ((total + kCtas - 1) / kCtas + kThreads - 1) / kThreads * kThreads;
  const int64_t e0 = each * rank, e1 = min(total, e0 + each);
  auto page_of = [&](int64_t e) -> int32_t {
    const int r = upper_index(first, R, e);
    const Span s = pages.gone(a.seq_len[r], a.new_len[r], a.window > 0 ? a.held_len[r] : 0);
    return a.block_table[r * a.table_stride + s.column(static_cast<int32_t>(e - first[r]))];
  };
  if (ok) {
    for (int64_t e = e0 + tid; e < e1; e += kThreads) {
      const int32_t page = page_of(e);
      if (page < 0 || page >= a.n_pages) {
        s_v.fail(1, upper_index(first, R, e));
      } else if (a.shared != nullptr) {
        d.rel[page] = 0;
        d.last[page] = -1;
      }
    }
    ok = agree(cluster, s_v, 1, &detail);
  }
  int64_t gives = total;  // pages that go to the list
  if (ok && a.shared != nullptr) {
    for (int64_t e = e0 + tid; e < e1; e += kThreads) {
      const int32_t page = page_of(e);
      atomicAdd(d.rel + page, 1);
      atomicMax(d.last + page, static_cast<int32_t>(e));
    }
    cluster.sync();
    int64_t mine = 0;
    for (int64_t e = e0 + tid; e < e1; e += kThreads) {
      const int32_t page = page_of(e), holders = a.shared[page], let_go = __ldcg(d.rel + page);
      if (holders < 0 || let_go > holders + 1) s_v.fail(2, upper_index(first, R, e));
      mine += let_go == holders + 1 && __ldcg(d.last + page) == e ? 1 : 0;
    }
    int64_t all;
    block_scan(mine, s_warp, &all);
    if (tid == 0) s_gives = all;
    ok = agree(cluster, s_v, 2, &detail);
    gives = 0;
    for (int c = 0; c < kCtas; ++c) gives += *cluster.map_shared_rank(&s_gives, c);
  }
  if (ok && gives > head) {
    ok = false;
    detail = R;
  }
  if (ok) {
    int64_t at = head - gives;
    if (a.shared == nullptr) {
      for (int64_t e = e0 + tid; e < e1; e += kThreads) a.free_pages[at + e] = page_of(e);
    } else {
      for (int c = 0; c < rank; ++c) at += *cluster.map_shared_rank(&s_gives, c);
      // counts of pages are read by entries of other CTAs above, behind the barrier of agree()
      for (int64_t b = e0; b < e1; b += kThreads) {
        const int64_t e = b + tid;
        int32_t page = 0, rest = 0;
        bool stands = false;
        if (e < e1) {
          page = page_of(e);
          stands = __ldcg(d.last + page) == e;
          if (stands) rest = a.shared[page] - __ldcg(d.rel + page);
        }
        const bool give = stands && rest < 0;
        int64_t all;
        const int64_t incl = block_scan(give ? 1 : 0, s_warp, &all);
        if (give) a.free_pages[at + incl - 1] = page;
        if (stands) a.shared[page] = max(rest, 0);
        at += all;
      }
    }
  }
  cluster.sync();  // lengths may be written over from here on, and no CTA reads another's shared memory
  if (ok) {
    for (int r = rank * kThreads + tid; r < R; r += kCtas * kThreads) {
      const int32_t now = a.new_len[r];
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
  int32_t* mark;   // [R]: how often a row is a child
};

__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads) k_cache_fork(ForkDev d) {
  __shared__ Verdict s_v;
  __shared__ int64_t s_warp[kThreads / 32];
  __shared__ int32_t s_first[kStaged + 1], s_fresh[kStaged];
  pdl_wait();
  pdl_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  const avtp_cache_fork_args_t& a = d.a;
  const int tid = threadIdx.x, rank = static_cast<int>(cluster.block_rank());
  const int C = a.n_children, P = a.page_size;
  const Pages& pages = d.pages;
  const bool staged = C <= kStaged;
  int32_t* first = staged ? s_first : d.first;
  int32_t* fresh = staged ? s_fresh : d.fresh;
  const int64_t head = a.free_head != nullptr ? *a.free_head : 0;
  if (tid == 0) s_v = Verdict{{head < 0 || head > a.n_free ? 1 : 0, 0, 0}, {-1, -1, -1}};
  __syncthreads();
  auto length = [&](int i, int p) { return a.fork_len != nullptr ? a.fork_len[i] : a.seq_len[p]; };

  int64_t total = 0, copies = 0;
  for (int base = 0; base < C; base += kThreads) {
    const int i = base + tid;
    int64_t n = 0, tail = 0;
    if (i < C) {
      const int32_t p = a.parent[i], c = a.child[i];
      bool bad = p < 0 || p >= a.n_requests || c < 0 || c >= a.n_requests;
      if (!bad) {
        const int32_t seq = a.seq_len[p], len = length(i, p), held = a.window > 0 ? a.held_len[p] : 0;
        bad = seq < 0 || len < 0 || len > seq || held < 0 || held > seq ||
              seq > static_cast<int64_t>(a.max_pages) * P || (len > 0 && pages.left(len) < pages.left(held));
        if (!bad) {
          n = pages.full(len, held).total();
          tail = len % P != 0 ? 1 : 0;
          if (rank == 0) d.mark[p] = d.mark[c] = 0;
        }
      }
      if (bad) s_v.fail(0, i);
    }
    int64_t all, all_tails;
    const int64_t incl = block_scan(n, s_warp, &all), incl_tails = block_scan(tail, s_warp, &all_tails);
    if (i < C && (staged || rank == 0)) {
      const int64_t before = total + incl - n;
      first[i] = static_cast<int32_t>(before < 0x7fffffff ? before : 0x7fffffff);
      fresh[i] = static_cast<int32_t>(copies + incl_tails - tail);
    }
    total += all;
    copies += all_tails;
  }
  if (tid == 0) {
    if (staged || rank == 0) first[C] = static_cast<int32_t>(total < 0x7fffffff ? total : 0x7fffffff);
    if (total > 0x7fffffff || head + copies > a.n_free) s_v.fail(0, C);
  }
  int detail = -1;
  bool ok = agree(cluster, s_v, 0, &detail);

  const int64_t step = static_cast<int64_t>(kCtas) * kThreads, at = rank * kThreads + tid;
  auto entry = [&](int64_t e, int* i, int* column) {
    *i = upper_index(first, C, e);
    const int32_t p = a.parent[*i];
    const Span s = pages.full(length(*i, p), a.window > 0 ? a.held_len[p] : 0);
    *column = s.column(static_cast<int32_t>(e - first[*i]));
    return a.block_table[p * a.table_stride + *column];
  };
  if (ok) {
    for (int64_t i = at; i < C; i += step) {
      if (atomicAdd(d.mark + a.child[i], 1) != 0) s_v.fail(1, static_cast<int>(i));
      const int32_t p = a.parent[i], len = length(static_cast<int>(i), p);
      if (len % P != 0) {
        const int32_t from = a.block_table[p * a.table_stride + len / P], to = a.free_pages[head + fresh[i]];
        if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) s_v.fail(1, static_cast<int>(i));
      }
    }
    for (int64_t e = at; e < total; e += step) {
      int i, column;
      const int32_t page = entry(e, &i, &column);
      if (page < 0 || page >= a.n_pages) s_v.fail(1, i);
    }
    ok = agree(cluster, s_v, 1, &detail);
  }
  if (ok) {
    for (int64_t i = at; i < C; i += step)
      if (__ldcg(d.mark + a.parent[i]) != 0) s_v.fail(2, static_cast<int>(i));
    ok = agree(cluster, s_v, 2, &detail);
  }
  // parents' rows and lengths are read, children's written: no row is both
  if (ok) {
    for (int64_t e = at; e < total; e += step) {
      int i, column;
      const int32_t page = entry(e, &i, &column);
      a.block_table[a.child[i] * a.table_stride + column] = page;
      atomicAdd(a.shared + page, 1);
    }
    for (int64_t i = at; i < C; i += step) {
      const int32_t p = a.parent[i], c = a.child[i], len = length(static_cast<int>(i), p);
      int32_t from = -1, to = -1;
      if (len % P != 0) {
        from = a.block_table[p * a.table_stride + len / P];
        to = a.free_pages[head + fresh[i]];
        a.block_table[c * a.table_stride + len / P] = to;
      }
      a.copy_src[i] = from;
      a.copy_dst[i] = to;
      a.seq_len[c] = len;
      if (a.window > 0) a.held_len[c] = len > 0 ? a.held_len[p] : 0;
    }
  }
  cluster.sync();  // no CTA reads another's shared memory from here on, nor the list's head
  if (rank == 0 && tid == 0) {
    *d.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, detail, 0u};
    if (ok && a.free_head_out != nullptr) *a.free_head_out = static_cast<int32_t>(head + copies);
  }
}

}  // namespace

cudaError_t launch_cache_free(const avtp_cache_free_args_t& a, void* ws, const FreeWs& p, cudaStream_t s) {
  FreeDev d{a, {CachePages::of(a.page_size, a.window, a.n_sinks)}, ws_at<DevStatus>(ws, p.status), ws_at<int32_t>(ws, p.first), ws_at<int32_t>(ws, p.rel),
            ws_at<int32_t>(ws, p.last)};
  return launch_kernel(k_cache_free, dim3(kCtas), dim3(kThreads), 0, s, /*pdl=*/true, d);
}

cudaError_t launch_cache_fork(const avtp_cache_fork_args_t& a, void* ws, const ForkWs& p, cudaStream_t s) {
  ForkDev d{a, {CachePages::of(a.page_size, a.window, a.n_sinks)}, ws_at<DevStatus>(ws, p.status), ws_at<int32_t>(ws, p.first), ws_at<int32_t>(ws, p.fresh),
            ws_at<int32_t>(ws, p.mark)};
  return launch_kernel(k_cache_fork, dim3(kCtas), dim3(kThreads), 0, s, /*pdl=*/true, d);
}

}  // namespace avtp
