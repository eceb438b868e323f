// Rows of the paged cache from place to place: whole pages (avtp_cache_copy) and the kept tokens of cached requests
// (avtp_cache_compact), to pages of their own or in place:
//   row(dst_table[r], j) = row(block_table[r], keep_idx[keep_cu[r] + j] - base_r),  row(t, p) = page t[p / P], row p % P
//
// Copies: 4 * Hkv * d bytes read and written a token bound them. Between different pages every row goes by
// itself: a warp finds the slots of 32 tokens, a lane each, and then moves them row by row, 16 bytes a lane.
//
// In place a row's destination may be another's source. Kept positions ascend and j <= keep_j - base, so that in their
// order a row is read before anything is written over it: what is written for tokens [a, b) lies before b, what is
// read for tokens from b on lies at b or behind. So a CTA takes a column of the request's rows (a slice of a head's keys or
// values) through all its tokens, a tile at a time, with a barrier between a tile's loads and its stores; columns are
// independent, and no CTA waits for another.
//
// What the calls record is found by a CTA of its own (the last one), the only writer of the status word; the
// others skip by the same rules. A request moved in place is checked as a whole by each of its CTAs before they move
// anything.
#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

__device__ __forceinline__ void write_status(DevStatus* st, int bad, int detail) {
  *st = DevStatus{bad ? static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT) : 0, bad ? 0 : 1, bad ? detail : 0, 0u};
}

// ---------------------------------------------------------------- whole pages
struct CopyDev {
  avtp_cache_t c;
  const int32_t *src, *dst;
  int64_t n;
  int64_t pieces;      // 16-byte pieces of a page of K, or of V
  int head_sh;         // log2 of a head's pieces
  int k_rows, v_rows;  // a page's rows in memory order: by token (0) or by head (1)
  DevStatus* st;
};

// Offset of piece i of a page, its rows in memory order.
__device__ __forceinline__ int64_t piece_offset(const CopyDev& d, int64_t i, int by_head, int64_t token_stride,
                                                int64_t head_stride) {
  const uint32_t row = static_cast<uint32_t>(i >> d.head_sh), in_row = static_cast<uint32_t>(i) & ((1u << d.head_sh) - 1);
  const uint32_t inner = by_head ? d.c.page_size : d.c.n_kv_heads, q = row / inner, m = row - q * inner;
  return (by_head ? m : q) * token_stride + (by_head ? q : m) * head_stride + in_row * 8;
}

__global__ void __launch_bounds__(kThreads) k_cache_copy(CopyDev d) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == gridDim.x - 1) {
    __shared__ int s_bad;
    if (threadIdx.x == 0) s_bad = 0x7fffffff;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < d.n; i += kThreads) {
      const int32_t s = d.src[i], t = d.dst[i];
      if (s < -1 || s >= d.c.n_pages || t < -1 || t >= d.c.n_pages) atomicMin(&s_bad, static_cast<int>(i));
    }
    __syncthreads();
    if (threadIdx.x == 0) write_status(d.st, s_bad != 0x7fffffff, s_bad);
    return;
  }
  // a CTA's share: kThreads * kUnroll pieces of a page of K or V
  const int64_t chunks = (d.pieces + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  const int64_t items = d.n * 2 * chunks;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x - 1) {
    const int64_t pair = item / (2 * chunks);
    const int64_t rest = item - pair * 2 * chunks;
    const bool is_v = rest >= chunks;
    const int64_t i0 = (rest - (is_v ? chunks : 0)) * kThreads * kUnroll + threadIdx.x;
    const int32_t from = d.src[pair], to = d.dst[pair];
    if (from < 0 || from >= d.c.n_pages || to < 0 || to >= d.c.n_pages) continue;
    __nv_bfloat16* pool = static_cast<__nv_bfloat16*>(is_v ? d.c.v : d.c.k);
    const int64_t page = is_v ? d.c.v_page_stride : d.c.k_page_stride;
    const int64_t token = is_v ? d.c.v_token_stride : d.c.k_token_stride, head = is_v ? d.c.v_head_stride : d.c.k_head_stride;
    const int by_head = is_v ? d.v_rows : d.k_rows;
    uint4 x[kUnroll];
    int64_t at[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * kThreads;
      if (i < d.pieces) {
        at[u] = piece_offset(d, i, by_head, token, head);
        x[u] = __ldcs(reinterpret_cast<const uint4*>(pool + from * page + at[u]));
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * kThreads < d.pieces) *reinterpret_cast<uint4*>(pool + to * page + at[u]) = x[u];
  }
}

// ---------------------------------------------------------------- kept tokens
struct CompactDev {
  avtp_cache_t c;
  avtp_cache_compact_args_t a;
  CachePages held;
  int each;     // to other pages: tokens of a warp at once, at most 32
  int lanes;    // to other pages: lanes of a row (a power of two, at most 32); pieces and head_sh as in the cache's write
  int pieces;
  int head_sh;
  int slice;    // in place: pieces of a head that a CTA takes; a power of two
  int slices;   // of a request, CTAs: Hkv * 2 * (pieces of a head / slice)
  DevStatus* st;
};

// Offsets in order, by all threads of the CTA.
__device__ bool offsets_fine(const avtp_cache_compact_args_t& a) {
  bool bad = threadIdx.x == 0 && a.keep_cu[0] != 0;
  for (int r = threadIdx.x; r < a.n_requests; r += kThreads) {
    const int64_t lo = a.keep_cu[r], hi = a.keep_cu[r + 1];
    bad = bad || lo < 0 || hi < lo || hi > a.n_kept;
  }
  return __syncthreads_or(bad) == 0;
}

// Slot of a request's row p; -1 where it lies outside the table or the pool, or (held) on a page let go of.
__device__ __forceinline__ int64_t slot_of(const avtp_cache_t& c, const int32_t* row, int max_pages, int64_t p,
                                           const CachePages* held, int32_t held_len) {
  const int64_t column = static_cast<uint32_t>(p) / static_cast<uint32_t>(c.page_size);
  if (p < 0 || p > 0x7fffffff || column >= max_pages) return -1;
  if (held != nullptr && !held->holds(static_cast<int32_t>(column), held_len)) return -1;
  const int32_t page = row[column];
  return page < 0 || page >= c.n_pages ? -1 : static_cast<int64_t>(page) * c.page_size + (p - column * c.page_size);
}

__device__ __forceinline__ int32_t held_len(const CompactDev& d, int r) { return d.a.window > 0 ? d.a.held_len[r] : 0; }

struct Move {
  int64_t from, to;  // slots; -1: not moved
  bool bad;
};
// Kept token i of request r, to other pages.
__device__ __forceinline__ Move move_of(const CompactDev& d, int r, int64_t i) {
  const avtp_cache_compact_args_t& a = d.a;
  const int64_t p = static_cast<int64_t>(a.keep_idx[i]) - (a.base_cu != nullptr ? a.base_cu[r] : 0);
  Move m;
  m.from = p >= a.seq_len[r] ? -1 : slot_of(d.c, a.block_table + r * a.table_stride, a.max_pages, p, &d.held, held_len(d, r));
  m.to = slot_of(d.c, a.dst_table + r * a.dst_stride, a.dst_max_pages, i - a.keep_cu[r], nullptr, 0);
  m.bad = m.from < 0 || m.to < 0;
  if (m.bad) m.from = m.to = -1;
  return m;
}
// What kept token j of n in place has wrong: its position or its order, its pages, or a page that others hold.
__device__ __forceinline__ bool bad_in_place(const CompactDev& d, int r, int64_t first, int64_t j) {
  const avtp_cache_compact_args_t& a = d.a;
  const int64_t base = a.base_cu != nullptr ? a.base_cu[r] : 0, p = a.keep_idx[first + j] - base;
  if (p < j || p >= a.seq_len[r] || (j > 0 && p <= a.keep_idx[first + j - 1] - base)) return true;
  const int32_t* row = a.block_table + r * a.table_stride;
  if (p == j) return false;
  const int64_t to = slot_of(d.c, row, a.max_pages, j, &d.held, held_len(d, r));
  if (to < 0 || slot_of(d.c, row, a.max_pages, p, &d.held, held_len(d, r)) < 0) return true;
  return a.shared != nullptr && a.shared[to / d.c.page_size] > 0;
}

// The CTA that records, and writes the new lengths.
__device__ void record(const CompactDev& d, bool in_place) {
  __shared__ int s_bad;
  if (threadIdx.x == 0) s_bad = 0x7fffffff;
  const avtp_cache_compact_args_t& a = d.a;
  if (!offsets_fine(a)) {
    if (threadIdx.x == 0) write_status(d.st, 1, -1);
    return;
  }
  const int64_t n = a.keep_cu[a.n_requests];
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const int r = upper_index(a.keep_cu, a.n_requests, i);
    if (in_place ? bad_in_place(d, r, a.keep_cu[r], i - a.keep_cu[r]) : move_of(d, r, i).bad) atomicMin(&s_bad, r);
  }
  if (a.len_out != nullptr)
    for (int r = threadIdx.x; r < a.n_requests; r += kThreads) a.len_out[r] = a.keep_cu[r + 1] - a.keep_cu[r];
  __syncthreads();
  if (threadIdx.x == 0) write_status(d.st, s_bad != 0x7fffffff, s_bad);
}

__global__ void __launch_bounds__(kThreads) k_cache_compact(CompactDev d) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == gridDim.x - 1) {
    record(d, false);
    return;
  }
  if (!offsets_fine(d.a)) return;
  const avtp_cache_compact_args_t& a = d.a;
  const int lane = threadIdx.x & 31, sub = lane & (d.lanes - 1), rows = 32 / d.lanes;
  const int64_t n = a.keep_cu[a.n_requests];
  const int64_t warps = static_cast<int64_t>(gridDim.x - 1) * (kThreads / 32);
  for (int64_t i0 = (static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + threadIdx.x / 32) * d.each; i0 < n;
       i0 += warps * d.each) {
    Move mine{-1, -1, false};
    if (lane < d.each && i0 + lane < n) mine = move_of(d, upper_index(a.keep_cu, a.n_requests, i0 + lane), i0 + lane);
    for (int k = 0; k < d.each; k += rows) {
      const int64_t from = __shfl_sync(0xffffffffu, mine.from, k + lane / d.lanes);
      const int64_t to = __shfl_sync(0xffffffffu, mine.to, k + lane / d.lanes);
      if (from < 0) continue;
      const uint32_t P = d.c.page_size;
      const uint32_t fp = static_cast<uint32_t>(from) / P, tp = static_cast<uint32_t>(to) / P;
      const int64_t fr = from - static_cast<int64_t>(fp) * P, tr = to - static_cast<int64_t>(tp) * P;
      __nv_bfloat16* kp = static_cast<__nv_bfloat16*>(d.c.k);
      __nv_bfloat16* vp = static_cast<__nv_bfloat16*>(d.c.v);
      const __nv_bfloat16* ks = kp + fp * d.c.k_page_stride + fr * d.c.k_token_stride;
      const __nv_bfloat16* vs = vp + fp * d.c.v_page_stride + fr * d.c.v_token_stride;
      __nv_bfloat16* kd = kp + tp * d.c.k_page_stride + tr * d.c.k_token_stride;
      __nv_bfloat16* vd = vp + tp * d.c.v_page_stride + tr * d.c.v_token_stride;
      for (int c0 = sub; c0 < d.pieces; c0 += d.lanes * kUnroll) {
        uint4 kx[kUnroll], vx[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int c = c0 + u * d.lanes;
          if (c < d.pieces) {
            const int64_t h = c >> d.head_sh;
            const int off = (c & ((1 << d.head_sh) - 1)) * 8;
            kx[u] = __ldcs(reinterpret_cast<const uint4*>(ks + h * d.c.k_head_stride + off));
            vx[u] = __ldcs(reinterpret_cast<const uint4*>(vs + h * d.c.v_head_stride + off));
          }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int c = c0 + u * d.lanes;
          if (c < d.pieces) {
            const int64_t h = c >> d.head_sh;
            const int off = (c & ((1 << d.head_sh) - 1)) * 8;
            *reinterpret_cast<uint4*>(kd + h * d.c.k_head_stride + off) = kx[u];
            *reinterpret_cast<uint4*>(vd + h * d.c.v_head_stride + off) = vx[u];
          }
        }
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads) k_cache_compact_in_place(CompactDev d) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == gridDim.x - 1) {
    record(d, true);
    return;
  }
  if (!offsets_fine(d.a)) return;
  const avtp_cache_compact_args_t& a = d.a;
  const int per_head = (1 << d.head_sh) / d.slice, sub = threadIdx.x & (d.slice - 1);
  const int rows = kThreads / d.slice;  // at once
  const int64_t items = static_cast<int64_t>(a.n_requests) * d.slices;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x - 1) {
    const int r = static_cast<int>(item / d.slices);
    int column = static_cast<int>(item - static_cast<int64_t>(r) * d.slices);
    const int64_t first = a.keep_cu[r], n = a.keep_cu[r + 1] - first;
    if (n == 0) continue;
    bool bad = false;
    for (int64_t j = threadIdx.x; j < n; j += kThreads) bad = bad || bad_in_place(d, r, first, j);
    if (__syncthreads_or(bad)) continue;
    const bool is_v = column >= d.c.n_kv_heads * per_head;
    if (is_v) column -= d.c.n_kv_heads * per_head;
    const int64_t page = is_v ? d.c.v_page_stride : d.c.k_page_stride;
    const int64_t token = is_v ? d.c.v_token_stride : d.c.k_token_stride;
    __nv_bfloat16* pool = static_cast<__nv_bfloat16*>(is_v ? d.c.v : d.c.k) +
                          (column / per_head) * (is_v ? d.c.v_head_stride : d.c.k_head_stride) +
                          ((column % per_head) * d.slice + sub) * 8;
    const int32_t* row = a.block_table + r * a.table_stride;
    const int64_t base = a.base_cu != nullptr ? a.base_cu[r] : 0;
    const uint32_t P = d.c.page_size;
    auto place = [&](int64_t p) {
      const uint32_t column = static_cast<uint32_t>(p) / P;
      return pool + row[column] * page + (p - static_cast<int64_t>(column) * P) * token;
    };
    constexpr int kRows = 8;  // of a thread, a tile
    for (int64_t j0 = threadIdx.x / d.slice; j0 - threadIdx.x / d.slice < n; j0 += rows * kRows) {
      uint4 x[kRows];
      __nv_bfloat16* to[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int64_t j = j0 + i * rows;
        to[i] = nullptr;
        if (j < n) {
          const int64_t p = a.keep_idx[first + j] - base;
          if (p != j) {
            to[i] = place(j);
            x[i] = *reinterpret_cast<const uint4*>(place(p));
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (to[i] != nullptr) *reinterpret_cast<uint4*>(to[i]) = x[i];
    }
  }
}

int head_shift(int d) { return d == 128 ? 4 : 3; }

}  // namespace

cudaError_t launch_cache_copy(const avtp_cache_t& c, const int32_t* src, const int32_t* dst, int64_t n, void* ws,
                              cudaStream_t s) {
  CopyDev d{};
  d.c = c;
  d.src = src;
  d.dst = dst;
  d.n = n;
  d.head_sh = head_shift(c.head_dim);
  d.pieces = static_cast<int64_t>(c.page_size) * c.n_kv_heads << d.head_sh;
  d.k_rows = c.k_head_stride > c.k_token_stride ? 1 : 0;
  d.v_rows = c.v_head_stride > c.v_token_stride ? 1 : 0;
  d.st = static_cast<DevStatus*>(ws);
  const int64_t want = n * 2 * ((d.pieces + kThreads * kUnroll - 1) / (kThreads * kUnroll));
  const int64_t most = 8 * static_cast<int64_t>(device_sm_count());
  return launch_kernel(k_cache_copy, dim3(static_cast<unsigned>((want < most ? want : most) + 1)), dim3(kThreads), 0, s,
                       /*pdl=*/true, d);
}

cudaError_t launch_cache_compact(const avtp_cache_t& c, const avtp_cache_compact_args_t& a, void* ws, cudaStream_t s) {
  CompactDev d{};
  d.c = c;
  d.a = a;
  d.head_sh = head_shift(c.head_dim);
  d.pieces = c.n_kv_heads << d.head_sh;
  d.lanes = 8;
  while (d.lanes < 32 && d.lanes < d.pieces) d.lanes *= 2;
  d.st = static_cast<DevStatus*>(ws);
  const int64_t sms = device_sm_count();
  d.held = CachePages::of(c.page_size, a.window, a.n_sinks);
  if (a.dst_table != nullptr) {
    d.each = 32;  // fewer where warps would be missing
    while (d.each > 32 / d.lanes && a.n_kept < d.each * 32 * sms) d.each /= 2;
    const int64_t per_cta = d.each * (kThreads / 32), want = (a.n_kept + per_cta - 1) / per_cta, most = 8 * sms;
    return launch_kernel(k_cache_compact, dim3(static_cast<unsigned>((want < most ? want : most) + 1)), dim3(kThreads), 0, s,
                         /*pdl=*/true, d);
  }
  d.slice = 1 << d.head_sh;
  d.slices = 2 * c.n_kv_heads * ((1 << d.head_sh) / d.slice);
  const int64_t want = static_cast<int64_t>(a.n_requests) * d.slices, most = 8 * sms;
  return launch_kernel(k_cache_compact_in_place, dim3(static_cast<unsigned>((want < most ? want : most) + 1)),
                       dim3(kThreads), 0, s, /*pdl=*/true, d);
}

}  // namespace avtp
