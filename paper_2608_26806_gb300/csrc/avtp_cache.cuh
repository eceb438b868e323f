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
cudaError_t launch_cache_write(const avtp_cache_t& c, const avtp_cache_write_args_t& a, void* ws, cudaStream_t s);

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
cudaError_t launch_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a, void* ws,
                                   const CacheAttnWs& p, cudaStream_t s);

struct CacheAttnDev;
cudaError_t launch_cache_chunk(int head_dim, int grid, const CUtensorMap& mq, const CUtensorMap& mk,
                               const CUtensorMap& mv, const CacheAttnDev& a, cudaStream_t s);

}  // namespace avtp
