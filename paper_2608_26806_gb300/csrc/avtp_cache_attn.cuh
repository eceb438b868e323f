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
  int R, max_new, max_pages, Hq, Hkv, G, page_size;
  int box;           // rows of a TMA box: a power of two that divides the page size, at most a tile
  int64_t few_rows;  // requests of at most this many rows a KV head are k_cache_attn's, the others k_cache_chunk's
  float c2;
  __nv_bfloat16* o;
  int64_t o_stride;
  float* lse;
  int64_t lse_stride;
  DevStatus* st;
  int32_t* count;        // see CacheAttnWs
  float* part_o;
  float2* part_ml;
  float* chunk_o;
  float2* chunk_ml;
  CacheChunkSplit* split;
};

struct CacheRequest {
  int32_t row0, n, seq;  // first packed row, new tokens, cached tokens
  // False for what validation refuses.
  __device__ __forceinline__ bool load(const CacheAttnDev& a, int r) {
    const int64_t lo = a.cu[r], hi = a.cu[r + 1];
    row0 = static_cast<int32_t>(lo);
    n = static_cast<int32_t>(hi - lo);
    seq = a.seq[r];
    return lo >= 0 && hi >= lo && hi <= a.n_tokens && hi - lo <= a.max_new && seq >= 0 &&
           seq <= static_cast<int64_t>(a.max_pages) * a.page_size && (r > 0 || lo == 0);
  }
  __device__ __forceinline__ int64_t rows(const CacheAttnDev& a) const { return static_cast<int64_t>(n) * a.G; }
};

// A call's work as one line of steps, request by request, cut into equal runs. Every CTA forms the
// cut for itself: NT threads take equal shares of the requests, pre[i] is the steps before thread
// i's share and pre[NT] all of them (0 if validation refuses a length).
template <int NT>
struct CachePlan {
  int64_t pre[NT + 1];
  int32_t most;  // steps of the longest row block (a row block's steps are one after the other on the line)
  int32_t ok;

  // steps(request, most): its steps, with the longest block's in `most`. All NT threads; ends with
  // a barrier. NT is a multiple of 32.
  template <class F>
  __device__ void form(const CacheAttnDev& a, F steps) {
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) {
      most = 1;
      ok = 1;
      pre[0] = 0;
    }
    __syncthreads();
    const int share = (a.R + NT - 1) / NT;
    int64_t sum = 0;
    int longest = 1;
    bool fine = true;
    for (int r = tid * share; r < min(a.R, (tid + 1) * share); ++r) {
      CacheRequest q;
      fine = q.load(a, r) && fine;
      if (fine) sum += steps(q, longest);
    }
    if (!fine) ok = 0;
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == 0 && longest > 1) atomicMax(&most, longest);
    pre[tid + 1] = sum;
    __syncthreads();
    if (tid < 32) {
      int64_t carry = 0;
      for (int b = 0; b < NT; b += 32) {
        int64_t x = pre[b + lane + 1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        x += carry;
        pre[b + lane + 1] = ok ? x : 0;
        carry = __shfl_sync(0xffffffffu, x, 31);
      }
    }
    __syncthreads();
  }
  // The first request of the share that step t lies in, and the steps before it.
  __device__ __forceinline__ int find(const CacheAttnDev& a, int64_t t, int64_t* before) const {
    int lo = 0, hi = NT;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] <= t) lo = mid; else hi = mid;
    }
    *before = pre[lo];
    return lo * ((a.R + NT - 1) / NT);
  }
};

// The runs: CTA c of N takes steps [c total / N, (c + 1) total / N). N is as many CTAs as there are,
// fewer where a run would be shorter than `least` steps or a block would have more than
// kCacheMaxPieces pieces.
struct CacheRuns {
  int64_t total, N;
  __device__ __forceinline__ CacheRuns(int64_t total_, int most, int least) : total(total_) {
    const int64_t run = max((most + kCacheMaxPieces - 3) / (kCacheMaxPieces - 2), least);
    N = max(int64_t(1), min(static_cast<int64_t>(gridDim.x), total / run));
  }
  __device__ __forceinline__ int64_t begin(int64_t c) const { return c < N ? c * total / N : total; }
  // the CTA of step t: the last whose run begins at or before it
  __device__ __forceinline__ int cta(int64_t t) const { return static_cast<int>(((t + 1) * N - 1) / total); }
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::
          "r"(tc::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(tc::smem_u32(bar))
      : "memory");
}

}  // namespace avtp
