// Rows of the paged cache from place to place: whole pages (avtp_cache_copy) and the kept tokens of cached requests
// (avtp_cache_compact), to pages of their own or in place:
//   row(dst_table[r], j) = row(block_table[r], keep_idx[keep_cu[r] + j] - base_r),  row(t, p) = page t[p / P], row p % P
//
// Copies: 4 * Hkv * d bytes read and written a token bound them. Between different pages every row goes by itself: a
// warp finds the slots of as many tokens as leave all warps in one wave, a lane each, and then moves them row by row,
// 16 bytes a lane. 64 requests of 1000 kept tokens, 8 KV heads, d = 128: 90 us, 5.8 TB/s; four of 2900 20.5 us, 4.6
// TB/s, of which the way to the first row (offsets, position, two tables) and the launch take 4.
//
// In place a row's destination may be another's source. Kept positions ascend and j <= keep_j - base, so that in
// their order a row is read before anything is written over it: what is written for tokens [a, b) lies before b, what
// is read for tokens from b on lies at b or behind. So a CTA takes columns of the request's rows (slices of a head's
// keys or values) through all its tokens, a tile at a time, with a barrier between a tile's reads and its writes, and
// the next tiles' copies under way; columns are independent, and no CTA waits for another. 64 requests of 1000 of
// 3000 tokens 133-143 us, 3.7-3.9 TB/s; four of 2900 of 8600 29.7; one of 3000 of 9000 23.4, where twelve tiles one
// behind the other take 11 and the look at the positions 7 (to other pages 6.2).
//
// What is wrong is recorded where it is met, in a status word that a kernel beside this one clears. (A CTA that
// looked through all kept tokens instead took longer than the copies: 50 us for 11600 of them.) A request moved in
// place is checked as a whole by each of its CTAs before they move anything.
#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
constexpr int kWarpsOfSm = 24;  // that an SM holds of k_cache_compact (80 registers a thread)

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
  int checked;         // the pairs are checked by a CTA of its own, the status word's only writer
  DevStatus* st;
};
constexpr int64_t kCheckPairs = 2048;  // beyond, a kernel ahead clears the word and the copying CTAs record

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
  const int64_t workers = static_cast<int64_t>(gridDim.x) - d.checked;
  if (blockIdx.x == workers) {
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
  for (int64_t item = blockIdx.x; item < items; item += workers) {
    const int64_t pair = item / (2 * chunks);
    const int64_t rest = item - pair * 2 * chunks;
    const bool is_v = rest >= chunks;
    const int64_t i0 = (rest - (is_v ? chunks : 0)) * kThreads * kUnroll + threadIdx.x;
    const int32_t from = d.src[pair], to = d.dst[pair];
    if (!d.checked && threadIdx.x == 0 && (from < -1 || from >= d.c.n_pages || to < -1 || to >= d.c.n_pages))
      record_error(d.st, AVTP_ERR_DEVICE_INPUT, static_cast<int32_t>(pair));
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
  int slice;    // in place: pieces of a column, a power of two
  int columns;  // of a request: Hkv * 2 * (pieces of a head / slice)
  int parts;    // CTAs of a request, an equal share of its columns each
  int page_sh;  // log2 of the page size; -1: no power of two
  DevStatus* st;
};

// Table column of a request's row p; -1 where it lies outside the table, or (held) on a page let go of.
__device__ __forceinline__ int32_t column_of(const avtp_cache_t& c, int max_pages, int64_t p, const CachePages* held,
                                             int32_t held_len) {
  const int64_t column = static_cast<uint32_t>(p) / static_cast<uint32_t>(c.page_size);
  if (p < 0 || p > 0x7fffffff || column >= max_pages) return -1;
  return held == nullptr || held->holds(static_cast<int32_t>(column), held_len) ? static_cast<int32_t>(column) : -1;
}
// Its slot, on that column's page; -1 where that lies outside the pool.
__device__ __forceinline__ int64_t slot_on(const avtp_cache_t& c, int64_t p, int32_t column, int32_t page) {
  if (page < 0 || page >= c.n_pages) return -1;
  return static_cast<int64_t>(page) * c.page_size + (p - static_cast<int64_t>(column) * c.page_size);
}
__device__ __forceinline__ int64_t slot_of(const avtp_cache_t& c, const int32_t* row, int max_pages, int64_t p,
                                           const CachePages* held, int32_t held_len) {
  const int32_t column = column_of(c, max_pages, p, held, held_len);
  return column < 0 ? -1 : slot_on(c, p, column, row[column]);
}

__device__ __forceinline__ int32_t held_len(const CompactDev& d, int r) { return d.a.window > 0 ? d.a.held_len[r] : 0; }

struct Move {
  int64_t from, to;  // slots; -1: not moved
  bool bad;
};
// Kept token i of request r, whose first is token `first`, to other pages.
__device__ __forceinline__ Move move_of(const CompactDev& d, int r, int64_t i, int64_t first) {
  const avtp_cache_compact_args_t& a = d.a;
  const int64_t p = static_cast<int64_t>(a.keep_idx[i]) - (a.base_cu != nullptr ? a.base_cu[r] : 0);
  Move m;
  m.from = p >= a.seq_len[r] ? -1 : slot_of(d.c, a.block_table + r * a.table_stride, a.max_pages, p, &d.held, held_len(d, r));
  m.to = slot_of(d.c, a.dst_table + r * a.dst_stride, a.dst_max_pages, i - first, nullptr, 0);
  m.bad = m.from < 0 || m.to < 0;
  if (m.bad) m.from = m.to = -1;
  return m;
}
// Kept tokens j0 + thread, + kThreads, ... below j1 of a request in place, four at a time: f(j, where from, where
// to), slots, to -1 of one that stays. True if one is wrong: its position or its order, its pages, or a page that
// others hold.
template <class F>
__device__ bool look_in_place(const CompactDev& d, int r, int64_t first, int64_t j0, int64_t j1, F f) {
  constexpr int N = 4;
  const avtp_cache_compact_args_t& a = d.a;
  const int64_t base = a.base_cu != nullptr ? a.base_cu[r] : 0;
  const int32_t seq = a.seq_len[r], held = held_len(d, r);
  const int32_t* row = a.block_table + r * a.table_stride;
  bool bad = false;
  for (int64_t j = j0 + threadIdx.x; j < j1; j += N * kThreads) {
    int64_t p[N], before[N], from[N], to[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t k = j + i * kThreads;
      p[i] = k < j1 ? a.keep_idx[first + k] - base : k;
      before[i] = k < j1 && k > 0 ? a.keep_idx[first + k - 1] - base : -1;
    }
    // all looks into the table go out ahead of the first use of one
    int32_t c_to[N], c_from[N], p_to[N], p_from[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t k = j + i * kThreads;
      const bool fine = k < j1 && p[i] >= k && p[i] < seq && p[i] > before[i];
      bad = bad || (k < j1 && !fine);
      c_to[i] = fine ? column_of(d.c, a.max_pages, k, &d.held, held) : -1;
      c_from[i] = fine ? column_of(d.c, a.max_pages, p[i], &d.held, held) : -1;
      p_to[i] = c_to[i] >= 0 ? row[c_to[i]] : -1;
      p_from[i] = c_from[i] >= 0 ? row[c_from[i]] : -1;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t k = j + i * kThreads;
      to[i] = slot_on(d.c, k, c_to[i], p_to[i]);
      from[i] = slot_on(d.c, p[i], c_from[i], p_from[i]);
      bad = bad || (k < j1 && (to[i] < 0 || from[i] < 0));
      if (p[i] == k) to[i] = -1;  // stays, on a page that has to be the request's too
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t k = j + i * kThreads;
      if (a.shared != nullptr && to[i] >= 0 && a.shared[to[i] / d.c.page_size] > 0) bad = true;
      if (k < j1) f(k, from[i], to[i]);
    }
  }
  return bad;
}

constexpr int kStaged = 1024;  // requests whose offsets are kept in shared memory

// keep_cu, from shared memory where it fits; NULL where it is refused. All threads of the CTA.
__device__ const int32_t* offsets(const avtp_cache_compact_args_t& a, int32_t (&s_cu)[kStaged + 1]) {
  const bool staged = a.n_requests <= kStaged;
  bool bad = false;
  for (int r = threadIdx.x; r <= a.n_requests; r += kThreads) {
    const int64_t lo = r == 0 ? 0 : a.keep_cu[r - 1], hi = a.keep_cu[r];
    bad = bad || hi < lo || hi > a.n_kept || (r == 0 && hi != 0);
    if (staged) s_cu[r] = static_cast<int32_t>(hi);
  }
  if (__syncthreads_or(bad)) return nullptr;
  return staged ? s_cu : a.keep_cu;
}

// To other pages, by the call's first CTA: the new lengths.
__device__ void write_lengths(const avtp_cache_compact_args_t& a, const int32_t* cu) {
  if (blockIdx.x != 0 || a.len_out == nullptr) return;
  for (int r = threadIdx.x; r < a.n_requests; r += kThreads) a.len_out[r] = cu[r + 1] - cu[r];
}

__global__ void __launch_bounds__(kThreads) k_cache_compact(CompactDev d) {
  __shared__ int32_t s_cu[kStaged + 1];
  pdl_trigger();
  const avtp_cache_compact_args_t& a = d.a;
  const int32_t* cu = offsets(a, s_cu);
  int bad = cu != nullptr ? -1 : 0x7fffffff;
  if (cu != nullptr) {
    write_lengths(a, cu);
    const int lane = threadIdx.x & 31, sub = lane & (d.lanes - 1), rows = 32 / d.lanes;
    const int64_t n = cu[a.n_requests];
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
    for (int64_t i0 = (static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + threadIdx.x / 32) * d.each; i0 < n;
         i0 += warps * d.each) {
      Move mine{-1, -1, false};
      if (lane < d.each && i0 + lane < n) {
        const int r = upper_index(cu, a.n_requests, i0 + lane);
        mine = move_of(d, r, i0 + lane, cu[r]);
        if (mine.bad) bad = r;
      }
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
  pdl_wait();  // the status word is cleared by the kernel ahead
  if (bad >= 0) record_error(d.st, AVTP_ERR_DEVICE_INPUT, bad);
}

constexpr int kChunk = 4096;    // kept tokens whose slots are in shared memory
constexpr int kRows = 4;        // rows of a thread, a tile
constexpr int kTiles = 4;       // under way
constexpr int kColumnCtas = 2;  // of an SM
constexpr size_t kInPlaceSmem = kTiles * kRows * kThreads * 16 + 2 * kChunk * 4;

__global__ void __launch_bounds__(kThreads, kColumnCtas) k_cache_compact_in_place(CompactDev d) {
  extern __shared__ uint4 s_ring[];  // [kTiles][kRows][kThreads]: what a thread copies it reads itself
  __shared__ int32_t s_cu[kStaged + 1];
  int32_t* s_from = reinterpret_cast<int32_t*>(s_ring + kTiles * kRows * kThreads);  // slots; to -1: stays
  int32_t* s_to = s_from + kChunk;
  pdl_trigger();
  const avtp_cache_compact_args_t& a = d.a;
  const int32_t* cu = offsets(a, s_cu);
  int wrong = cu != nullptr ? -1 : 0x7fffffff;
  if (cu != nullptr) {
    const int per_head = (1 << d.head_sh) / d.slice, sub = threadIdx.x & (d.slice - 1);
    const int at_once = kThreads / d.slice, first_row = threadIdx.x / d.slice;
    const uint32_t P = d.c.page_size;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(s_ring)) + threadIdx.x * 16;
    const int64_t items = static_cast<int64_t>(a.n_requests) * d.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
      const int r = static_cast<int>(item / d.parts), part = static_cast<int>(item - static_cast<int64_t>(r) * d.parts);
      const int c0 = static_cast<int>(static_cast<int64_t>(part) * d.columns / d.parts);
      const int c1 = static_cast<int>(static_cast<int64_t>(part + 1) * d.columns / d.parts);
      const int64_t first = cu[r], n = cu[r + 1] - first;
      // A request's new length, by the CTA of its first columns behind the look: of one that stays as it was its old
      // one, so that whoever hands the lengths on gives none of its pages away.
      auto write_length = [&](int32_t len) {
        if (part == 0 && threadIdx.x == 0 && a.len_out != nullptr) a.len_out[r] = len;
      };
      if (n == 0) {
        write_length(0);
        continue;
      }
      auto look = [&](int64_t j0) {  // tokens j0 .. j0 + kChunk - 1
        return look_in_place(d, r, first, j0, min(n, j0 + kChunk), [&](int64_t j, int64_t from, int64_t to) {
          s_from[j - j0] = static_cast<int32_t>(from);
          s_to[j - j0] = static_cast<int32_t>(to);
        });
      };
      bool bad = look(0);
      // a new end inside a page that others hold: the request's next token would be written over theirs
      if (a.shared != nullptr && threadIdx.x == 0 && n < a.seq_len[r] && n % P != 0 && n / P < a.max_pages) {
        const int32_t page = a.block_table[r * a.table_stride + n / P];
        bad = bad || (page >= 0 && page < d.c.n_pages && a.shared[page] > 0);
      }
      if (n > kChunk) bad = look_in_place(d, r, first, kChunk, n, [](int64_t, int64_t, int64_t) {}) || bad;
      if (__syncthreads_or(bad)) {
        wrong = r;
        write_length(a.seq_len[r]);
        __syncthreads();
        continue;
      }
      write_length(static_cast<int32_t>(n));
      for (int64_t j0 = 0; j0 < n; j0 += kChunk) {
        if (j0 > 0) {
          __syncthreads();
          look(j0);
          __syncthreads();
        }
        const int rows = static_cast<int>(min(n - j0, static_cast<int64_t>(kChunk)));
        // Tiles, column by column. Copies run kTiles tiles ahead of the stores: a column's later rows lie behind all
        // that its earlier ones are written over, and columns do not meet.
        const int tiles = (rows + at_once * kRows - 1) / (at_once * kRows), all = tiles * (c1 - c0);
        struct Place {
          __nv_bfloat16* base;
          int64_t page, token;
          int row0;
        };
        auto tile_of = [&](int q) {
          const int c = q / tiles, col = c0 + c;
          const bool is_v = col >= d.c.n_kv_heads * per_head;
          const int within = is_v ? col - d.c.n_kv_heads * per_head : col;
          return Place{static_cast<__nv_bfloat16*>(is_v ? d.c.v : d.c.k) +
                           (within / per_head) * (is_v ? d.c.v_head_stride : d.c.k_head_stride) +
                           ((within % per_head) * d.slice + sub) * 8,
                       is_v ? d.c.v_page_stride : d.c.k_page_stride, is_v ? d.c.v_token_stride : d.c.k_token_stride,
                       (q - c * tiles) * at_once * kRows + first_row};
        };
        auto place = [&](const Place& t, int32_t slot) {
          const uint32_t p = d.page_sh >= 0 ? static_cast<uint32_t>(slot) >> d.page_sh : static_cast<uint32_t>(slot) / P;
          return t.base + p * t.page + (slot - p * P) * t.token;
        };
        auto issue = [&](int q) {
          if (q < all) {
            const Place t = tile_of(q);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
              const int j = t.row0 + i * at_once;
              if (j < rows && s_to[j] >= 0)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + (q % kTiles * kRows + i) * kThreads * 16),
                             "l"(place(t, s_from[j]))
                             : "memory");
            }
          }
          asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll 1
        for (int q = 0; q < kTiles; ++q) issue(q);
#pragma unroll 1
        for (int q = 0; q < all; ++q) {
          asm volatile("cp.async.wait_group %0;" ::"n"(kTiles - 1) : "memory");
          __syncthreads();  // the tile has been read
          const Place t = tile_of(q);
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            const int j = t.row0 + i * at_once;
            if (j < rows && s_to[j] >= 0)
              *reinterpret_cast<uint4*>(place(t, s_to[j])) = s_ring[(q % kTiles * kRows + i) * kThreads + threadIdx.x];
          }
          issue(q + kTiles);
        }
      }
      __syncthreads();
    }
  }
  pdl_wait();  // the status word is cleared by the kernel ahead
  if (wrong >= 0 && threadIdx.x == 0) record_error(d.st, AVTP_ERR_DEVICE_INPUT, wrong);
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
  d.checked = n <= kCheckPairs ? 1 : 0;
  if (!d.checked) {
    const cudaError_t e = launch_cache_status(d.st, s);
    if (e != cudaSuccess) return e;
  }
  return launch_kernel(k_cache_copy, dim3(static_cast<unsigned>((want < most ? want : most) + d.checked)), dim3(kThreads), 0,
                       s, /*pdl=*/true, d);
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
  const cudaError_t e = launch_cache_status(d.st, s);
  if (e != cudaSuccess) return e;
  if (a.dst_table != nullptr) {
    d.each = 32;  // fewer where that leaves all warps in one wave
    while (d.each > 32 / d.lanes && a.n_kept <= d.each / 2 * kWarpsOfSm * sms) d.each /= 2;
    const int64_t per_cta = d.each * (kThreads / 32), want = (a.n_kept + per_cta - 1) / per_cta, most = 8 * sms;
    const unsigned grid = static_cast<unsigned>(want < 1 ? 1 : (want < most ? want : most));
    return launch_kernel(k_cache_compact, dim3(grid), dim3(kThreads), 0, s, /*pdl=*/true, d);
  }
  static PerDevice attrs;
  const cudaError_t set = once_per_device(attrs, [](int, int*) {
    return cudaFuncSetAttribute(k_cache_compact_in_place, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(kInPlaceSmem));
  });
  if (set != cudaSuccess) return set;
  // Columns of a head's width, several a CTA where requests are many (they share the look at its tokens), or as
  // narrow as 64 bytes where CTAs would be missing.
  const int64_t most = kColumnCtas * sms, wanted = (most + a.n_requests - 1) / a.n_requests;
  d.slice = 1 << d.head_sh;
  while (d.slice > 4 && 2 * c.n_kv_heads * ((1 << d.head_sh) / d.slice) < wanted) d.slice /= 2;
  d.columns = 2 * c.n_kv_heads * ((1 << d.head_sh) / d.slice);
  d.parts = static_cast<int>(d.columns < wanted ? d.columns : wanted);
  d.page_sh = -1;
  if ((c.page_size & (c.page_size - 1)) == 0)
    for (d.page_sh = 0; (1 << d.page_sh) < c.page_size;) ++d.page_sh;
  const int64_t want = static_cast<int64_t>(a.n_requests) * d.parts;
  return launch_kernel(k_cache_compact_in_place, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(kThreads),
                       kInPlaceSmem, s, /*pdl=*/true, d);
}

}  // namespace avtp
