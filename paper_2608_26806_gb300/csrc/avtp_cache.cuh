// Host-side declarations of the paged cache's kernels (k_cache_*.cu).
#pragma once

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
constexpr int kCacheTile = 64;        // keys of a tile
constexpr int kCacheMaxPieces = 32;   // pieces a row block's keys are split into, at most
struct CacheAttnWs {
  size_t status;   // DevStatus
  size_t count;    // int32 [grid]: pieces done of the row block whose first piece is the CTA's last
  size_t part_o;   // float [2 * grid][rows][d]: a piece's O, not yet divided by its sum
  size_t part_ml;  // float2 [2 * grid][rows]: a piece's reference and sum (log2 units)
  size_t total;
};
CacheAttnWs plan_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a);
cudaError_t launch_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a, void* ws,
                                   const CacheAttnWs& p, cudaStream_t s);

}  // namespace avtp
