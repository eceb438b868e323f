// Host-side declarations of the paged cache's kernels (k_cache_*.cu).
#pragma once

#include <cuda.h>

#include "avtp_internal.cuh"

namespace avtp {

// ---------------------------------------------------------------- slots
struct SlotsWs {
  size_t status;  // DevStatus
  size_t past;    // int32 [R]: past_len as it was (seq_len may overwrite it)
  size_t first;   // int32 [R]: entry of the free list of a request's first new page
  size_t total;
};
cudaError_t launch_cache_slots(const avtp_cache_slots_args_t& a, void* ws, const SlotsWs& p, cudaStream_t s);

// ---------------------------------------------------------------- write
// Clears a status word. The kernel behind it starts beside it, behind everything ahead of both, and waits for it
// (pdl_wait) before it records.
cudaError_t launch_cache_status(DevStatus* st, cudaStream_t s);
cudaError_t launch_cache_write(const avtp_cache_t& c, const avtp_cache_write_args_t& a, void* ws, cudaStream_t s);

// ---------------------------------------------------------------- rotary positions
cudaError_t launch_rope(const avtp_rope_args_t& a, const avtp_cache_t* c, void* ws, cudaStream_t s);

// ---------------------------------------------------------------- pages
// Which pages a request of n tokens holds (see avtp.h): columns j < up(n) with j < sinks or j >= left(held_len).
struct CachePages {
  int32_t P, window, sinks;  // page size, window, pages of the sinks
  static CachePages of(int32_t page_size, int32_t window, int32_t n_sinks) {
    return {page_size, window, window > 0 ? static_cast<int32_t>((int64_t(n_sinks) + page_size - 1) / page_size) : 0};
  }
  __device__ __forceinline__ int32_t up(int32_t n) const { return (static_cast<uint32_t>(n) + P - 1u) / P; }
  // the first page that the window of token n needs
  __device__ __forceinline__ int32_t left(int32_t n) const {
    return window > 0 && n >= window ? (n - window + 1) / P : 0;
  }
  __device__ __forceinline__ bool holds(int32_t column, int32_t held) const {
    return column < sinks || column >= left(held);
  }
  // Whether n tokens need a page that a request held at `held` tokens has let go of. (Not those whose pages are all the
  // sinks', nor where the sinks reach what is held.)
  __device__ __forceinline__ bool lacks(int32_t n, int32_t held) const {
    return max(sinks, left(n)) < min(left(held), up(n));
  }
};

struct FreeWs {
  size_t status, first, rel, last, total;  // see FreeDev
};
cudaError_t launch_cache_free(const avtp_cache_free_args_t& a, void* ws, const FreeWs& p, cudaStream_t s);

struct ForkWs {
  size_t status, first, fresh, mark, total;  // see ForkDev
};
cudaError_t launch_cache_fork(const avtp_cache_fork_args_t& a, void* ws, const ForkWs& p, cudaStream_t s);

cudaError_t launch_cache_copy(const avtp_cache_t& c, const int32_t* src, const int32_t* dst, int64_t n, void* ws,
                              cudaStream_t s);
cudaError_t launch_cache_compact(const avtp_cache_t& c, const avtp_cache_compact_args_t& a, void* ws, cudaStream_t s);

// ---------------------------------------------------------------- attention
// Rows of a (request, KV head) are its (new token, head of the group) pairs, token by token.
constexpr int kCacheMaxPieces = 32;   // pieces that a row block's keys are split into, at most
constexpr int kChunkRows = 256;       // rows of a unit of k_cache_chunk, two slots of 128
constexpr int kChunkKeys = 128;       // keys of its blocks
// Requests of at most kCacheFewRows rows a KV head are k_cache_attn's, when no request of the call can
// have more; beside larger ones (max_new is the call's bound) those of at most kCacheFewMixed, one
// warp's. Sixteen requests of 700-4000 tokens, four heads a group, us a call there and in
// k_cache_chunk: 20 rows 34.9 / 41.7, 32 rows 37.6 / 42.1, 36 rows (by four warps a slice of keys) 49.0 /
// 42.4, 64 rows 55.4 / 42.8.
constexpr int kCacheFewRows = 32;
constexpr int kCacheFewMixed = 16;

// A unit of k_cache_chunk in several pieces, for the kernel that joins them; c1 < c0: none.
struct CacheChunkSplit {
  int32_t row0, n, head, unit;  // request's first packed row and new tokens, KV head, unit of the request
  int32_t c0, c1;               // runs of the first and the last piece
};

struct CacheAttnWs {
  size_t status;    // DevStatus
  size_t count;     // int32 [grid]: pieces done of the row block whose first piece is the CTA's last
  size_t part_o;    // float [2 * grid][rows][d]: a piece's O, not yet divided by its sum
  size_t part_ml;   // float4 [2 * grid][rows]: a piece's reference (log2 units), sum of P, of its rounded values
  // of k_cache_chunk, when max_new allows a request for it
  size_t chunk_o;   // float4 [2 * grid][2 slots][d / 4][128 rows]
  size_t chunk_ml;  // float2 [2 * grid][2 slots][128 rows]
  size_t split;     // CacheChunkSplit [grid]
  size_t total;
};
CacheAttnWs plan_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a);
// window 0: none
cudaError_t launch_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a, const avtp_cache_window_t& w,
                                   void* ws, const CacheAttnWs& p, cudaStream_t s);
// False: a windowed call of more work than its kernels count.
bool cache_attention_fits(const avtp_cache_t& c, const avtp_cache_attn_args_t& a, const avtp_cache_window_t& w);

struct CacheAttnDev;
cudaError_t launch_cache_chunk(int head_dim, bool in_window, int grid, const CUtensorMap& mq, const CUtensorMap& mk,
                               const CUtensorMap& mv, const CacheAttnDev& a, cudaStream_t s);

}  // namespace avtp
