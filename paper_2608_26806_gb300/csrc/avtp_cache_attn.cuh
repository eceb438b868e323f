// Device code that the two kernels of avtp_cache_attention share (k_cache_attn.cu for few rows a
// request, k_cache_chunk.cu for many): the arguments, what a request asks for, and the cut of a
// call's work into equal runs.
#pragma once

#include "avtp_cache.cuh"
#include "avtp_tc.cuh"

namespace avtp {

struct CacheAttnDev {
  const __nv_bfloat16* q;
  int64_t q_stride;
  const int32_t* cu;
  const int32_t* seq;
  const int32_t* table;
  int64_t table_stride;
  int64_t n_tokens, n_pages;
  int R, max_new, max_pages, Hkv, G, page_size;
  int window, sinks;  // a query at place p sees u <= p with u > p - window or u < sinks (kernels of a window alone)
  int box;           // rows of a TMA box: a power of two that divides the page size, at most a tile
  int step_shift;    // see CachePlan
  int both;          // both kernels are at work and share the SMs (see cache_ctas)
  int64_t few_rows;  // requests of at most this many rows a KV head are k_cache_attn's, the others k_cache_chunk's
  float c2;
  __nv_bfloat16* o;
  int64_t o_stride;
  float* lse;
  int64_t lse_stride;
  DevStatus* st;
  int32_t* count;        // see CacheAttnWs
  float* part_o;
  float4* part_ml;
  float* chunk_o;
  float2* chunk_ml;
  CacheChunkSplit* split;
};

// A request's keys, at most: positions up to a block behind its last one are 32-bit numbers.
constexpr int32_t kCacheMostKeys = 0x7fffffff - 255;

struct CacheRequest {
  int32_t row0, n, seq;  // first packed row, new tokens, cached tokens
  // False for what validation refuses.
  __device__ __forceinline__ bool load(const CacheAttnDev& a, int r) {
    const int64_t lo = a.cu[r], hi = a.cu[r + 1];
    row0 = static_cast<int32_t>(lo);
    n = static_cast<int32_t>(hi - lo);
    seq = a.seq[r];
    return lo >= 0 && hi >= lo && hi <= a.n_tokens && hi - lo <= a.max_new && seq >= 0 &&
           seq <= kCacheMostKeys && seq <= static_cast<int64_t>(a.max_pages) * a.page_size && (r > 0 || lo == 0);
  }
  __device__ __forceinline__ int64_t rows(const CacheAttnDev& a) const { return static_cast<int64_t>(n) * a.G; }
};

// In a window, the first key behind the sinks that a token at place p sees (p negative: it sees nothing).
__device__ __forceinline__ int cache_low(const CacheAttnDev& a, int p) { return p < a.window ? 0 : p - a.window + 1; }
// The tiles between the sinks' and the first that a row block sees are left out: of those behind the sinks', tile j
// is the request's tile j + skip.
struct CacheSkip {
  int32_t sinks, skip;  // tiles
  // `first`: place of the row block's first new token
  __device__ __forceinline__ CacheSkip(const CacheAttnDev& a, int first, int tile_keys) {
    sinks = (a.sinks + tile_keys - 1) / tile_keys;
    skip = max(0, cache_low(a, first) / tile_keys - sinks);
  }
  __device__ __forceinline__ int tile(int j) const { return j < sinks ? j : j + skip; }
};

// The roles of a CTA share an instruction cache, which a second copy of their loops has cost more than
// half of a kernel's speed, and a first pass over code waits for it. So what is not a role's inner
// loop exists once a kernel: the waits (behind a first look), warp sums.
static __device__ __noinline__ bool cache_wait_on(uint64_t* bar, uint32_t parity) { return tc::mbar_wait(bar, parity); }
static __device__ __noinline__ bool cache_wait_warp_on(uint64_t* bar, uint32_t parity) {
  return tc::mbar_wait_warp(bar, parity);
}
__device__ __forceinline__ bool cache_wait(uint64_t* bar, uint32_t parity) {
  return tc::mbar_test_wait(bar, parity) || cache_wait_on(bar, parity);
}
__device__ __forceinline__ bool cache_wait_warp(uint64_t* bar, uint32_t parity) {
  return __all_sync(0xffffffffu, tc::mbar_test_wait(bar, parity)) || cache_wait_warp_on(bar, parity);
}
// Whether a CTA gives up, one answer for the calling warp.
__device__ __forceinline__ bool cache_raised(const volatile int* flag) { return __any_sync(0xffffffffu, *flag) != 0; }

// What a request costs k_cache_attn (x) and k_cache_chunk (y), in units of about 0.07 us of an SM: a tile
// of 64 keys 7, a block of 128 keys of a unit, or its beginning, 20 (a tile 6, 8 or 10: two chunks
// beside 22 single tokens 70, 65, 66 us, one of 2048 beside 63 255, 255, 289, one of 100 beside 63
// 270, 293, 369). Clamped so that the sum over the requests is a 32-bit number.
template <bool kWindow>
__device__ __forceinline__ int2 cache_weights(const CacheAttnDev& a, const CacheRequest& q) {
  const int64_t most = 0x7fffffff / a.R;
  // keys that a row block of so many tokens passes, at most
  auto keys = [&](int all, int tokens) {
    if (!kWindow) return all;
    return static_cast<int>(min(static_cast<int64_t>(all), static_cast<int64_t>(a.window) + a.sinks + tokens));
  };
  if (q.rows(a) <= a.few_rows)
    return make_int2(static_cast<int>(min(most, int64_t(7) * a.Hkv * ((keys(q.seq, q.n) + 63) / 64))), 0);
  const int rows = 2 * (kChunkRows / 2 / a.G);
  const int64_t units = static_cast<int64_t>((q.n + rows - 1) / rows) * a.Hkv;
  return make_int2(0, static_cast<int>(min(most, 20 * units * (2 + keys(max(0, q.seq - q.n / 2), rows) / 128))));
}
// The CTAs that work in k_cache_attn (`few`) or k_cache_chunk, of the grid's. The first is bound by
// memory, the second by the tensor cores, and a CTA of either fills an SM: where a call needs both
// they share the SMs by their work, and the second kernel's CTAs start on those that the first
// leaves. (One behind the other, each on all SMs: 74, 292 and 293 us for the three above.)
__device__ __forceinline__ int cache_ctas(const CacheAttnDev& a, int2 w, bool few) {
  const int grid = static_cast<int>(gridDim.x);
  if (!a.both || w.x == 0 || w.y == 0) return grid;
  const float part = static_cast<float>(w.x) / (static_cast<float>(w.x) + static_cast<float>(w.y));
  const int n = max(1, min(grid - 1, static_cast<int>(part * grid + 0.5f)));
  return few ? n : grid - n;
}

// Inclusive sums over a warp.
static __device__ __noinline__ int cache_scan(int x) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// A call's work as one line of steps, request by request, row block by row block (rows served by one pass
// over their keys: a request's of a KV head in k_cache_attn, a unit in k_cache_chunk), cut into equal
// runs. A step is 2^step_shift tiles of keys of a row block (0 but for calls whose bounds would let the
// line pass 2^31 steps). Every CTA forms the cut for itself, its loading warp alone for up to 32 requests
// (a lane each), else all its threads (NT of them, equal shares of the requests; pre[i] is the steps before
// thread i's share).
constexpr int kNearRequests = 32;
template <int NT>
struct CachePlan {
  int32_t pre[NT + 1];
  int32_t total, most, ok;
  int32_t few, chunk;  // summed cache_weights

  __device__ __forceinline__ static int share(const CacheAttnDev& a) { return (a.R + NT - 1) / NT; }
  // For more than kNearRequests requests, all threads: steps(request, most) gives a request's steps,
  // with those of its longest row block in `most`. NT is a multiple of 32.
  template <bool kWindow, class F>
  __device__ void form(const CacheAttnDev& a, F steps) {
    const int tid = threadIdx.x, lane = tid & 31, each = share(a);
    if (tid == 0) {
      most = 1;
      ok = 1;
      few = chunk = 0;
    }
    __syncthreads();
    int sum = 0, longest = 1;
    bool fine = true;
#pragma unroll 1
    for (int r = tid * each; r < min(a.R, (tid + 1) * each); ++r) {
      CacheRequest q;
      fine = q.load(a, r) && fine;
      if (fine) {
        sum += steps(q, longest);
        if (a.both) {
          const int2 w = cache_weights<kWindow>(a, q);
          atomicAdd(&few, w.x);
          atomicAdd(&chunk, w.y);
        }
      }
    }
    if (!fine) ok = 0;
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == 0 && longest > 1) atomicMax(&most, longest);
    pre[tid + 1] = sum;
    __syncthreads();
    if (tid < 32) {
      int carry = 0;
      const int used = min(NT, a.R);  // threads with a share
#pragma unroll 1
      for (int b = 0; b < used; b += 32) {
        const int x = cache_scan(pre[b + lane + 1]) + carry;
        pre[b + lane + 1] = x;
        carry = __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) {
        pre[0] = 0;
        total = carry;
      }
    }
    __syncthreads();
  }
};
// The loading warp's view of the line.
template <bool kWindow>
struct CacheLine {
  int total;  // 0 if validation refuses a length
  int most;   // steps of the longest row block (a row block's steps are one after the other on the line)
  int incl;   // up to kNearRequests requests: steps up to this lane's, its own included
  int2 weights;
  bool fine;  // up to kNearRequests requests: validation refuses none

  CacheLine() = default;
  template <int NT, class F>
  __device__ __forceinline__ CacheLine(const CacheAttnDev& a, const CachePlan<NT>& plan, const CacheRequest& mine,
                                       bool mine_ok, F steps) {
    if (a.R > kNearRequests) {
      total = plan.ok ? plan.total : 0;
      most = plan.most;
      incl = 0;
      weights = make_int2(plan.few, plan.chunk);
    } else {
      const int lane = threadIdx.x & 31;
      int longest = 1;
      incl = lane < a.R && mine_ok ? steps(mine, longest) : 0;
      incl = a.R > 1 ? cache_scan(incl) : __shfl_sync(0xffffffffu, incl, 0);
      most = __reduce_max_sync(0xffffffffu, longest);
      fine = __all_sync(0xffffffffu, mine_ok || lane >= a.R);
      total = fine ? __shfl_sync(0xffffffffu, incl, 31) : 0;
      weights = make_int2(0, 0);
      if (a.both) {
        const int2 w = lane < a.R && mine_ok ? cache_weights<kWindow>(a, mine) : make_int2(0, 0);
        weights = make_int2(__reduce_add_sync(0xffffffffu, w.x), __reduce_add_sync(0xffffffffu, w.y));
      }
    }
  }
  // Request r, by the whole warp: of up to kNearRequests a lane holds it (a load takes 800 cycles).
  __device__ __forceinline__ CacheRequest request(const CacheAttnDev& a, const CacheRequest& mine, int r) const {
    CacheRequest q;
    if (a.R <= kNearRequests) {
      q.row0 = __shfl_sync(0xffffffffu, mine.row0, r);
      q.n = __shfl_sync(0xffffffffu, mine.n, r);
      q.seq = __shfl_sync(0xffffffffu, mine.seq, r);
    } else {
      q.load(a, r);
    }
    return q;
  }
  // A request at or before that of step t, t < total, and the steps before it.
  template <int NT>
  __device__ __forceinline__ int find(const CacheAttnDev& a, const CachePlan<NT>& plan, int t, int* before) const {
    if (a.R <= kNearRequests) {
      const int r = __popc(__ballot_sync(0xffffffffu, incl <= t));
      const int x = __shfl_sync(0xffffffffu, incl, r > 0 ? r - 1 : 0);
      *before = r > 0 ? x : 0;
      return r;
    }
    int lo = 0, hi = min(NT, a.R);
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.pre[mid] <= t) lo = mid; else hi = mid;
    }
    *before = plan.pre[lo];
    return lo * CachePlan<NT>::share(a);
  }
};

// The runs: N of them, the first total % N a step longer than the others. N is as many as there are
// CTAs, fewer where a run would be shorter than `least` steps or a block would be in more than
// kCacheMaxPieces pieces.
struct CacheRuns {
  int total, each, longer;  // steps of a run, runs of one step more
  int N;
  CacheRuns() = default;
  __device__ __forceinline__ CacheRuns(int total_, int most, int least, int ctas) : total(total_) {
    const int run = max((most + kCacheMaxPieces - 3) / (kCacheMaxPieces - 2), least);
    N = max(1, min(ctas, static_cast<int>(static_cast<uint32_t>(total) / static_cast<uint32_t>(run))));
    each = static_cast<uint32_t>(total) / static_cast<uint32_t>(N);
    longer = total - each * N;
  }
  __device__ __forceinline__ int begin(int c) const { return c < N ? c * each + min(c, longer) : total; }
  // the run of step t
  __device__ __forceinline__ int run(int t) const {
    const int edge = longer * (each + 1);
    return t < edge ? static_cast<uint32_t>(t) / static_cast<uint32_t>(each + 1)
                    : longer + static_cast<uint32_t>(t - edge) / static_cast<uint32_t>(each);
  }
};
// Where a run leaves a piece of a block: a block that began in an earlier run in its even place, one
// that goes on in the next run in its odd one. A run has at most one of either kind.
__device__ __forceinline__ int piece_place(int run, bool begins) { return 2 * run + (begins ? 1 : 0); }

// Where a request's boxes of keys lie, 32 of them at a time: a warp looks them up in the block table, a
// lane a box, and one thread issues their copies. Box i holds keys i * box ..
struct CacheBoxes {
  int2 at[32];  // page, row of the page
  // Boxes i0 .. i0 + 31 (i0 a multiple of 32) of a request of `seq` tokens; true if a page lies outside the pool:
  // page 0 then stands in its place. In a window no page is looked up for boxes behind the sinks that end at or
  // before key `low`, for it may have been let go of: their copies read behind the pool, and bring zeros.
  template <bool kWindow>
  __device__ __forceinline__ bool load(const CacheAttnDev& a, const int32_t* row, int seq, int i0, int low = 0) {
    const int lane = threadIdx.x & 31;
    const uint32_t i = static_cast<uint32_t>(i0 + lane), in_page = static_cast<uint32_t>(a.page_size / a.box);
    const uint32_t p = i / in_page;
    int page = 0;
    const int64_t key = static_cast<int64_t>(i) * a.box;
    const bool seen = !kWindow || key < a.sinks || key + a.box > low;
    if (key < seq && seen) page = row[p];
    const bool bad = page < 0 || page >= a.n_pages;
    __syncwarp();  // the boxes before have been used
    at[lane] = make_int2(!seen ? static_cast<int>(a.n_pages) : bad ? 0 : page, static_cast<int>(i - p * in_page) * a.box);
    __syncwarp();
    return __any_sync(0xffffffffu, bad);
  }
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::
          "r"(tc::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(tc::smem_u32(bar))
      : "memory");
}

}  // namespace avtp
