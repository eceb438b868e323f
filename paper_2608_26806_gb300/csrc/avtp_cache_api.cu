// C ABI of the paged cache: argument validation, workspace plans and launches of
// avtp_cache_slots, avtp_cache_write, avtp_rope, avtp_cache_attention (and _window_attention) and the upkeep of pages
// (avtp_cache_compact, _copy, _fork, _free); the frequencies of avtp_rope.
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

// One tensor of rows: head_dim elements a head, contiguous heads.
avtp_status_t check_rows(const void* p, int64_t stride, int64_t row) {
  if (p == nullptr || stride < row) return AVTP_ERR_INVALID_ARG;
  return aligned16(p) && stride % 8 == 0 ? AVTP_OK : AVTP_ERR_UNSUPPORTED;
}

avtp_status_t check_rope(const avtp_rope_args_t* a, const avtp_cache_t* c) {
  if (a == nullptr || a->n_tokens < 0 || a->n_q_heads < 0 || a->n_kv_heads < 0) return AVTP_ERR_INVALID_ARG;
  if (a->n_tokens > kInt32Max || a->n_q_heads > 65536 || a->n_kv_heads > 65536) return AVTP_ERR_RANGE;
  if (a->head_dim != 64 && a->head_dim != 128) return AVTP_ERR_UNSUPPORTED;
  if (a->rot_dim < 0 || a->rot_dim > a->head_dim) return AVTP_ERR_INVALID_ARG;
  if (a->rot_dim % 8 != 0) return AVTP_ERR_UNSUPPORTED;
  if (a->style != AVTP_ROPE_HALF && a->style != AVTP_ROPE_INTERLEAVED) return AVTP_ERR_INVALID_ARG;
  if (!isfinite(a->attn_factor) || !isfinite(a->eps) || a->eps < 0.f) return AVTP_ERR_INVALID_ARG;
  if (c != nullptr) {
    const avtp_status_t st = check_cache(c);
    if (st != AVTP_OK) return st;
    if (c->n_kv_heads != a->n_kv_heads || c->head_dim != a->head_dim) return AVTP_ERR_INVALID_ARG;
  }
  if (a->n_tokens == 0) return AVTP_OK;
  const int64_t d = a->head_dim;
  struct Rows {
    const void* p;
    int64_t stride, heads;
    bool wanted;
  } const rows[5] = {{a->q, a->q_stride, a->n_q_heads, true},
                     {a->q_out, a->q_out_stride, a->n_q_heads, true},
                     {a->k, a->k_stride, a->n_kv_heads, true},
                     {a->k_out, a->k_out_stride, a->n_kv_heads, c == nullptr || a->k_out != nullptr},
                     {a->v, a->v_stride, a->n_kv_heads, c != nullptr}};
  for (const Rows& r : rows) {
    if (r.heads == 0 || !r.wanted) continue;
    const avtp_status_t st = check_rows(r.p, r.stride, r.heads * d);
    if (st != AVTP_OK) return st;
  }
  if (c != nullptr && a->slot_map == nullptr) return AVTP_ERR_INVALID_ARG;
  if (a->rot_dim > 0 && (a->inv_freq == nullptr || a->pos == nullptr || a->n_planes < 1 || a->pos_stride < a->n_tokens))
    return AVTP_ERR_INVALID_ARG;
  if (!aligned16(a->q_norm) || !aligned16(a->k_norm)) return AVTP_ERR_UNSUPPORTED;
  return AVTP_OK;
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

avtp_status_t check_window_attn(const avtp_cache_t* c, const avtp_cache_attn_args_t* a, const avtp_cache_window_t* w) {
  const avtp_status_t st = check_attn(c, a);
  if (st != AVTP_OK) return st;
  if (w == nullptr || w->window < 1 || w->n_sinks < 0) return AVTP_ERR_INVALID_ARG;
  return cache_attention_fits(*c, *a, *w) ? AVTP_OK : AVTP_ERR_RANGE;
}

// The kernels' 32-bit loops over requests or children step 1024 at a time, past the last.
bool countable(int64_t n) { return n <= kInt32Max - 1024; }

avtp_status_t check_table(const int32_t* table, int32_t max_pages, int64_t stride) {
  return table != nullptr && max_pages >= 1 && stride >= max_pages ? AVTP_OK : AVTP_ERR_INVALID_ARG;
}

avtp_status_t check_window(int32_t window, int32_t n_sinks, const void* held_len) {
  return window >= 0 && n_sinks >= 0 && (window == 0 || held_len != nullptr) ? AVTP_OK : AVTP_ERR_INVALID_ARG;
}

avtp_status_t check_compact(const avtp_cache_t* c, const avtp_cache_compact_args_t* a) {
  avtp_status_t st = check_cache(c);
  if (st != AVTP_OK) return st;
  if (a == nullptr || a->n_requests < 1 || a->n_kept < 0) return AVTP_ERR_INVALID_ARG;
  if (a->n_kept > kInt32Max || !countable(a->n_requests)) return AVTP_ERR_RANGE;
  if (a->keep_cu == nullptr || a->seq_len == nullptr || (a->n_kept > 0 && a->keep_idx == nullptr)) return AVTP_ERR_INVALID_ARG;
  if ((st = check_table(a->block_table, a->max_pages, a->table_stride)) != AVTP_OK) return st;
  if (a->dst_table != nullptr && (st = check_table(a->dst_table, a->dst_max_pages, a->dst_stride)) != AVTP_OK) return st;
  if (a->len_out == a->seq_len) return AVTP_ERR_INVALID_ARG;
  return check_window(a->window, a->n_sinks, a->held_len);
}

avtp_status_t check_fork(const avtp_cache_fork_args_t* a) {
  if (a == nullptr || a->n_requests < 1 || a->n_children < 0) return AVTP_ERR_INVALID_ARG;
  avtp_status_t st = check_pool_size(a->n_pages, a->page_size);
  if (st != AVTP_OK) return st;
  if (!countable(a->n_requests) || !countable(a->n_children) || a->n_free > kInt32Max) return AVTP_ERR_RANGE;
  if (a->n_free < 0 || (a->n_free > 0 && a->free_pages == nullptr)) return AVTP_ERR_INVALID_ARG;
  if ((st = check_table(a->block_table, a->max_pages, a->table_stride)) != AVTP_OK) return st;
  if (a->seq_len == nullptr || a->shared == nullptr) return AVTP_ERR_INVALID_ARG;
  if (a->n_children > 0 && (a->parent == nullptr || a->child == nullptr || a->copy_src == nullptr || a->copy_dst == nullptr))
    return AVTP_ERR_INVALID_ARG;
  return check_window(a->window, a->n_sinks, a->held_len);
}

ForkWs plan_fork(const avtp_cache_fork_args_t& a) {
  ForkWs p{};
  const size_t R = static_cast<size_t>(a.n_requests), C = static_cast<size_t>(a.n_children);
  p.status = 0;
  p.first = align_up(sizeof(DevStatus));
  p.fresh = p.first + align_up((C + 1) * 4);
  p.mark = p.fresh + align_up(C * 4);
  p.total = p.mark + align_up(R * 4);
  return p;
}

avtp_status_t check_free(const avtp_cache_free_args_t* a) {
  if (a == nullptr || a->n_requests < 1) return AVTP_ERR_INVALID_ARG;
  avtp_status_t st = check_pool_size(a->n_pages, a->page_size);
  if (st != AVTP_OK) return st;
  if (!countable(a->n_requests) || a->n_free > kInt32Max) return AVTP_ERR_RANGE;
  if (a->n_free < 0 || (a->n_free > 0 && a->free_pages == nullptr)) return AVTP_ERR_INVALID_ARG;
  if ((st = check_table(a->block_table, a->max_pages, a->table_stride)) != AVTP_OK) return st;
  if (a->seq_len == nullptr || a->new_len == nullptr || a->free_head == nullptr || a->seq_len_out == nullptr ||
      a->free_head_out == nullptr || (a->window > 0 && a->held_len_out == nullptr))
    return AVTP_ERR_INVALID_ARG;
  return check_window(a->window, a->n_sinks, a->held_len);
}

FreeWs plan_free(const avtp_cache_free_args_t& a) {
  FreeWs p{};
  const size_t R = static_cast<size_t>(a.n_requests), n = static_cast<size_t>(a.n_pages);
  p.status = 0;
  p.first = align_up(sizeof(DevStatus));
  p.rel = p.first + align_up((R + 1) * 4);
  p.last = p.rel + (a.shared != nullptr ? align_up(n * 4) : 0);
  p.total = p.last + align_up(n * 4);
  return p;
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

avtp_status_t avtp_rope(const avtp_rope_args_t* args, const avtp_cache_t* cache, void* workspace, size_t workspace_bytes,
                        avtp_stream_t stream) {
  avtp_status_t st = check_rope(args, cache);
  if (st != AVTP_OK) return st;
  if ((st = check_ws(workspace, workspace_bytes, sizeof(DevStatus))) != AVTP_OK) return st;
  return from_cuda(launch_rope(*args, cache, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_rope_frequencies(const avtp_rope_freq_args_t* a, float* inv_freq, float* attn_factor) {
  if (a == nullptr || inv_freq == nullptr || a->rot_dim < 2 || a->rot_dim % 2 != 0 || !(a->base > 1.0) ||
      !isfinite(a->base) || a->scale < AVTP_ROPE_SCALE_NONE || a->scale > AVTP_ROPE_SCALE_YARN)
    return AVTP_ERR_INVALID_ARG;
  const bool yarn = a->scale == AVTP_ROPE_SCALE_YARN;
  if (a->scale != AVTP_ROPE_SCALE_NONE && (!(a->factor >= 1.0) || !isfinite(a->factor))) return AVTP_ERR_INVALID_ARG;
  if (a->scale == AVTP_ROPE_SCALE_NTK && a->rot_dim < 4) return AVTP_ERR_INVALID_ARG;
  if (yarn && (!(a->original_len > 0.0) || !isfinite(a->original_len) || !(a->slow >= 0.0) || !(a->slow < a->fast) ||
               !isfinite(a->fast)))
    return AVTP_ERR_INVALID_ARG;
  const double n = a->rot_dim;
  const double base = a->scale == AVTP_ROPE_SCALE_NTK ? a->base * pow(a->factor, n / (n - 2.0)) : a->base;
  for (int32_t i = 0; i < a->rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / n);
    if (a->scale == AVTP_ROPE_SCALE_LINEAR) f /= a->factor;
    if (yarn) {
      const double turns = a->original_len * f / 6.283185307179586;
      const double g = fmin(fmax((turns - a->slow) / (a->fast - a->slow), 0.0), 1.0);
      f = (1.0 - g) * f / a->factor + g * f;
    }
    inv_freq[i] = static_cast<float>(f);
  }
  if (attn_factor != nullptr) *attn_factor = yarn ? static_cast<float>(0.1 * log(a->factor) + 1.0) : 1.f;
  return AVTP_OK;
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
  return from_cuda(launch_cache_attention(*cache, *args, avtp_cache_window_t{0, 0}, workspace, p,
                                          reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_window_attention_workspace_size(const avtp_cache_t* cache, const avtp_cache_attn_args_t* args,
                                                         const avtp_cache_window_t* window, size_t* bytes) {
  const avtp_status_t st = check_window_attn(cache, args, window);
  if (st != AVTP_OK) return st;
  if (bytes == nullptr) return AVTP_ERR_INVALID_ARG;
  *bytes = plan_cache_attention(*cache, *args).total;
  return AVTP_OK;
}

avtp_status_t avtp_cache_window_attention(const avtp_cache_t* cache, const avtp_cache_attn_args_t* args,
                                          const avtp_cache_window_t* window, void* workspace, size_t workspace_bytes,
                                          avtp_stream_t stream) {
  avtp_status_t st = check_window_attn(cache, args, window);
  if (st != AVTP_OK) return st;
  const CacheAttnWs p = plan_cache_attention(*cache, *args);
  if ((st = check_ws(workspace, workspace_bytes, p.total)) != AVTP_OK) return st;
  return from_cuda(
      launch_cache_attention(*cache, *args, *window, workspace, p, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_compact(const avtp_cache_t* cache, const avtp_cache_compact_args_t* args, void* workspace,
                                 size_t workspace_bytes, avtp_stream_t stream) {
  avtp_status_t st = check_compact(cache, args);
  if (st != AVTP_OK) return st;
  if ((st = check_ws(workspace, workspace_bytes, sizeof(DevStatus))) != AVTP_OK) return st;
  return from_cuda(launch_cache_compact(*cache, *args, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_copy(const avtp_cache_t* cache, const int32_t* src, const int32_t* dst, int64_t n, void* workspace,
                              size_t workspace_bytes, avtp_stream_t stream) {
  avtp_status_t st = check_cache(cache);
  if (st != AVTP_OK) return st;
  if (n < 0 || (n > 0 && (src == nullptr || dst == nullptr))) return AVTP_ERR_INVALID_ARG;
  if (n > kInt32Max) return AVTP_ERR_RANGE;
  if ((st = check_ws(workspace, workspace_bytes, sizeof(DevStatus))) != AVTP_OK) return st;
  return from_cuda(launch_cache_copy(*cache, src, dst, n, workspace, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_fork_workspace_size(const avtp_cache_fork_args_t* args, size_t* bytes) {
  const avtp_status_t st = check_fork(args);
  if (st != AVTP_OK) return st;
  if (bytes == nullptr) return AVTP_ERR_INVALID_ARG;
  *bytes = plan_fork(*args).total;
  return AVTP_OK;
}

avtp_status_t avtp_cache_fork(const avtp_cache_fork_args_t* args, void* workspace, size_t workspace_bytes,
                              avtp_stream_t stream) {
  avtp_status_t st = check_fork(args);
  if (st != AVTP_OK) return st;
  const ForkWs p = plan_fork(*args);
  if ((st = check_ws(workspace, workspace_bytes, p.total)) != AVTP_OK) return st;
  return from_cuda(launch_cache_fork(*args, workspace, p, reinterpret_cast<cudaStream_t>(stream)));
}

avtp_status_t avtp_cache_free_workspace_size(const avtp_cache_free_args_t* args, size_t* bytes) {
  const avtp_status_t st = check_free(args);
  if (st != AVTP_OK) return st;
  if (bytes == nullptr) return AVTP_ERR_INVALID_ARG;
  *bytes = plan_free(*args).total;
  return AVTP_OK;
}

avtp_status_t avtp_cache_free(const avtp_cache_free_args_t* args, void* workspace, size_t workspace_bytes,
                              avtp_stream_t stream) {
  avtp_status_t st = check_free(args);
  if (st != AVTP_OK) return st;
  const FreeWs p = plan_free(*args);
  if ((st = check_ws(workspace, workspace_bytes, p.total)) != AVTP_OK) return st;
  return from_cuda(launch_cache_free(*args, workspace, p, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
