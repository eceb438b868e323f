// C ABI of the paged cache: argument validation, workspace plans and launches of
// avtp_cache_slots, avtp_cache_write and avtp_cache_attention.
#include <math.h>

#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kInt32Max = 0x7fffffff;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }
avtp_status_t from_cuda(cudaError_t e) { return e == cudaSuccess ? AVTP_OK : AVTP_ERR_CUDA; }

avtp_status_t check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & (kAlign - 1)) != 0 || ws_bytes < need)
    return AVTP_ERR_WORKSPACE;
  return AVTP_OK;
}

avtp_status_t check_pool_size(int64_t n_pages, int32_t page_size) {
  if (n_pages < 1 || page_size < 1) return AVTP_ERR_INVALID_ARG;
  if (n_pages > kInt32Max / page_size) return AVTP_ERR_RANGE;
  return AVTP_OK;
}

avtp_status_t check_cache(const avtp_cache_t* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->n_kv_heads < 1) return AVTP_ERR_INVALID_ARG;
  const avtp_status_t st = check_pool_size(c->n_pages, c->page_size);
  if (st != AVTP_OK) return st;
  if (c->head_dim != 64 && c->head_dim != 128) return AVTP_ERR_UNSUPPORTED;
  if (c->n_kv_heads > 65536) return AVTP_ERR_RANGE;
  if (!aligned16(c->k) || !aligned16(c->v)) return AVTP_ERR_UNSUPPORTED;
  const int64_t strides[2][3] = {{c->k_page_stride, c->k_token_stride, c->k_head_stride},
                                 {c->v_page_stride, c->v_token_stride, c->v_head_stride}};
  for (const auto& s : strides) {
    for (int64_t x : s) {
      if (x < c->head_dim) return AVTP_ERR_INVALID_ARG;
      if (x % 8 != 0) return AVTP_ERR_UNSUPPORTED;
      if (x >= (int64_t(1) << 39)) return AVTP_ERR_RANGE;  // a tensor map's stride is below 2^40 bytes
    }
    if (s[0] < s[1] || s[0] < s[2]) return AVTP_ERR_UNSUPPORTED;
  }
  return AVTP_OK;
}

avtp_status_t check_slots(const avtp_cache_slots_args_t* a) {
  if (a == nullptr || a->n_requests < 1 || a->n_tokens < 0 || a->max_pages < 1) return AVTP_ERR_INVALID_ARG;
  const avtp_status_t st = check_pool_size(a->n_pages, a->page_size);
  if (st != AVTP_OK) return st;
  if (a->n_tokens > kInt32Max || a->n_free > kInt32Max) return AVTP_ERR_RANGE;
  // the kernel's 32-bit loops over the requests step 1024 at a time, past the last
  if (a->n_requests > kInt32Max - 1024) return AVTP_ERR_RANGE;
  if (a->n_free < 0 || a->table_stride < a->max_pages) return AVTP_ERR_INVALID_ARG;
  if (a->cu_new == nullptr || a->block_table == nullptr || a->seq_len == nullptr) return AVTP_ERR_INVALID_ARG;
  if ((a->n_tokens > 0 && a->slot_map == nullptr) || (a->n_free > 0 && a->free_pages == nullptr))
    return AVTP_ERR_INVALID_ARG;
  return AVTP_OK;
}

SlotsWs plan_slots(const avtp_cache_slots_args_t& a) {
  SlotsWs p{};
  const size_t R = static_cast<size_t>(a.n_requests);
  p.status = 0;
  p.past = align_up(sizeof(DevStatus));
  p.first = p.past + align_up(R * 4);
  p.total = p.first + align_up(R * 4);
  return p;
}

avtp_status_t check_attn(const avtp_cache_t* c, const avtp_cache_attn_args_t* a) {
  avtp_status_t st = check_cache(c);
  if (st != AVTP_OK) return st;
  if (c->page_size % 16 != 0) return AVTP_ERR_UNSUPPORTED;
  if (a == nullptr || a->n_requests < 1 || a->n_tokens < 0 || a->max_new < 0 || a->max_pages < 1 || a->n_q_heads < 1)
    return AVTP_ERR_INVALID_ARG;
  if (a->n_tokens > kInt32Max) return AVTP_ERR_RANGE;
  if (a->n_q_heads % c->n_kv_heads != 0 || a->n_q_heads / c->n_kv_heads > kAttnMaxGroupHeads)
    return AVTP_ERR_UNSUPPORTED;
  // rows of a KV head, and new tokens beside cached ones, are 32-bit numbers
  if (static_cast<int64_t>(a->max_new) * (a->n_q_heads / c->n_kv_heads) > kInt32Max) return AVTP_ERR_RANGE;
  // so are the blocks of rows that the requests may have, with a few steps each (see CachePlan)
  const int64_t slot = kChunkRows / 2 / (a->n_q_heads / c->n_kv_heads);
  if (a->n_requests + a->n_tokens / (2 * slot) > (int64_t(1) << 27) / c->n_kv_heads) return AVTP_ERR_RANGE;
  if (a->cu_new == nullptr || a->seq_len == nullptr || a->block_table == nullptr) return AVTP_ERR_INVALID_ARG;
  if (a->n_tokens > 0 && (a->q == nullptr || a->o == nullptr)) return AVTP_ERR_INVALID_ARG;
  if (a->table_stride < a->max_pages) return AVTP_ERR_INVALID_ARG;
  const int64_t row = static_cast<int64_t>(a->n_q_heads) * c->head_dim;
  if (a->q_stride < row || a->o_stride < row) return AVTP_ERR_INVALID_ARG;
  if (a->q_stride % 8 != 0 || a->o_stride % 8 != 0) return AVTP_ERR_UNSUPPORTED;
  if (!aligned16(a->q) || !aligned16(a->o)) return AVTP_ERR_UNSUPPORTED;
  if (a->lse != nullptr && a->lse_stride < a->n_tokens) return AVTP_ERR_INVALID_ARG;
  if (!(a->softmax_scale > 0.f) || !isfinite(a->softmax_scale)) return AVTP_ERR_INVALID_ARG;
  return AVTP_OK;
}

}  // namespace
}  // namespace avtp

using namespace avtp;

extern "C" {

avtp_status_t avtp_cache_slots_workspace_size(const avtp_cache_slots_args_t* args, size_t* bytes) {
  const avtp_status_t st = check_slots(args);
  if (st != AVTP_OK) return st;
  if (bytes == nullptr) return AVTP_ERR_INVALID_ARG;
  *bytes = plan_slots(*args).total;
  return AVTP_OK;
}

avtp_status_t avtp_cache_slots(const avtp_cache_slots_args_t* args, void* workspace, size_t workspace_bytes,
                               avtp_stream_t stream) {
  avtp_status_t st = check_slots(args);
  if (st != AVTP_OK) return st;
  const SlotsWs p = plan_slots(*args);
  if ((st = check_ws(workspace, workspace_bytes, p.total)) != AVTP_OK) return st;
  return from_cuda(launch_cache_slots(*args, workspace, p, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_write(const avtp_cache_t* cache, const avtp_cache_write_args_t* args, void* workspace,
                               size_t workspace_bytes, avtp_stream_t stream) {
  avtp_status_t st = check_cache(cache);
  if (st != AVTP_OK) return st;
  if (args == nullptr || args->n < 0 || args->n_rows < 0) return AVTP_ERR_INVALID_ARG;
  if (args->n > kInt32Max || args->n_rows > kInt32Max) return AVTP_ERR_RANGE;
  if (args->n > 0 && (args->k == nullptr || args->v == nullptr || args->slot_map == nullptr))
    return AVTP_ERR_INVALID_ARG;
  const int64_t row = static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim;
  if (args->k_stride < row || args->v_stride < row) return AVTP_ERR_INVALID_ARG;
  if (args->k_stride % 8 != 0 || args->v_stride % 8 != 0) return AVTP_ERR_UNSUPPORTED;
  if (!aligned16(args->k) || !aligned16(args->v)) return AVTP_ERR_UNSUPPORTED;
  if ((st = check_ws(workspace, workspace_bytes, sizeof(DevStatus))) != AVTP_OK) return st;
  return from_cuda(launch_cache_write(*cache, *args, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_attention_workspace_size(const avtp_cache_t* cache, const avtp_cache_attn_args_t* args,
                                                  size_t* bytes) {
  const avtp_status_t st = check_attn(cache, args);
  if (st != AVTP_OK) return st;
  if (bytes == nullptr) return AVTP_ERR_INVALID_ARG;
  *bytes = plan_cache_attention(*cache, *args).total;
  return AVTP_OK;
}

avtp_status_t avtp_cache_attention(const avtp_cache_t* cache, const avtp_cache_attn_args_t* args, void* workspace,
                                   size_t workspace_bytes, avtp_stream_t stream) {
  avtp_status_t st = check_attn(cache, args);
  if (st != AVTP_OK) return st;
  const CacheAttnWs p = plan_cache_attention(*cache, *args);
  if ((st = check_ws(workspace, workspace_bytes, p.total)) != AVTP_OK) return st;
  return from_cuda(launch_cache_attention(*cache, *args, workspace, p, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
