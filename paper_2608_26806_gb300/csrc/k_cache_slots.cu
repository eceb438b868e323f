// Block tables and slot maps of a step's new tokens in the paged cache, from lengths that only
// the device knows (the pruned offsets of avtp_prune). With P = page_size:
//   have_r = ceil(past_r / P),  need_r = ceil((past_r + new_r) / P),  take_r = need_r - have_r
//   first_r = head + sum_{s < r} take_s
//   table[r][j] = free[first_r + j - have_r]                      have_r <= j < need_r
//   slot[t] = table[r][p / P] * P + p % P,  p = past_r + t - cu_r  cu_r <= t < cu_{r+1}
//   seq_len_r = past_r + new_r,  head' = head + sum_r take_r;  slot = -1 behind the last token.
//
// One CTA checks everything before anything is written (offsets, lengths, the free list's end and
// every page that will be used), so a refused call changes nothing. It keeps past_r and first_r
// in the workspace: seq_len and free_head_out may be past_len and free_head themselves. Up to
// kOneCtaTokens tokens the same CTA writes the maps; beyond, a second kernel over the whole GPU.
#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 1024;
constexpr int kMapThreads = 256;
constexpr int64_t kOneCtaTokens = 8192;

struct SlotsDev {
  avtp_cache_slots_args_t a;
  DevStatus* st;
  int32_t* past;   // workspace copies, see SlotsWs
  int32_t* first;
};

__device__ __forceinline__ int64_t ceil_div(int64_t x, int64_t p) { return (x + p - 1) / p; }

// New pages of request r into its table row; the lanes of a group of n threads share them.
__device__ __forceinline__ void write_pages(const SlotsDev& d, int r, int lane, int n) {
  const int64_t past = d.past[r], len = past + d.a.cu_new[r + 1] - d.a.cu_new[r];
  const int64_t have = ceil_div(past, d.a.page_size), need = ceil_div(len, d.a.page_size);
  int32_t* row = d.a.block_table + r * d.a.table_stride;
  const int32_t* src = d.a.free_pages + d.first[r];
  for (int64_t j = have + lane; j < need; j += n) row[j] = src[j - have];
}

// The slot of token t, which belongs to request r. New pages are read from the free list (their
// table entries may be another thread's to write).
__device__ __forceinline__ int32_t slot_of(const SlotsDev& d, int r, int64_t t) {
  const int64_t past = d.past[r];
  const int64_t pos = past + t - d.a.cu_new[r];
  const int32_t page = static_cast<int32_t>(pos / d.a.page_size);
  const int32_t have = static_cast<int32_t>(ceil_div(past, d.a.page_size));
  const int32_t id = page < have ? d.a.block_table[r * d.a.table_stride + page] : d.a.free_pages[d.first[r] + page - have];
  return id * d.a.page_size + static_cast<int32_t>(pos - static_cast<int64_t>(page) * d.a.page_size);
}

// Slots of tokens t, t + step, ... A thread's requests only go up, so it searches for the first
// and walks to the next.
__device__ void write_slots(const SlotsDev& d, int64_t t, int64_t step) {
  const int R = d.a.n_requests;
  const int64_t live = d.a.cu_new[R];
  int r = -1;
  for (; t < d.a.n_tokens; t += step) {
    if (t >= live) {
      d.a.slot_map[t] = -1;
      continue;
    }
    if (r < 0 || t >= d.a.cu_new[r + 1]) r = upper_index(d.a.cu_new, R, t);
    d.a.slot_map[t] = slot_of(d, r, t);
  }
}

__global__ void __launch_bounds__(kThreads) k_cache_slots(SlotsDev d, int write_all) {
  __shared__ int s_err, s_detail;
  __shared__ int64_t s_warp[32], s_carry;
  pdl_wait();
  pdl_trigger();
  const avtp_cache_slots_args_t& a = d.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int R = a.n_requests;
  const int64_t P = a.page_size;
  const int64_t head = a.free_head != nullptr ? *a.free_head : 0;
  if (tid == 0) {
    s_err = (head < 0 || a.cu_new[0] != 0) ? 1 : 0;
    s_detail = -1;
    s_carry = 0;
  }
  __syncthreads();
  auto fail = [&](int detail) {
    if (atomicExch(&s_err, 1) == 0) s_detail = detail;
  };
  for (int base = 0; base < R; base += kThreads) {
    const int r = base + tid;
    int64_t past = 0, take = 0;
    if (r < R) {
      const int64_t lo = a.cu_new[r], hi = a.cu_new[r + 1];
      past = a.past_len != nullptr ? a.past_len[r] : 0;
      if (lo < 0 || hi < lo || hi > a.n_tokens || past < 0 || past + hi - lo > a.max_pages * P ||
          past + hi - lo > 0x7fffffff) {
        fail(r);
      } else {
        take = ceil_div(past + hi - lo, P) - ceil_div(past, P);
        if (hi > lo && past % P != 0) {  // the page that the new tokens begin in
          const int32_t id = a.block_table[r * a.table_stride + past / P];
          if (id < 0 || id >= a.n_pages) fail(r);
        }
      }
    }
    int64_t incl = take;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int64_t before = s_carry;
    for (int w = 0; w < warp; ++w) before += s_warp[w];
    if (r < R) {
      // below n_free (checked before it is used), which is below 2^31
      const int64_t first = head + before + incl - take;
      d.past[r] = static_cast<int32_t>(past);
      d.first[r] = static_cast<int32_t>(first < a.n_free ? first : a.n_free);
    }
    __syncthreads();
    if (tid == kThreads - 1) s_carry = before + incl;
    __syncthreads();
  }
  const int64_t total = s_carry;
  if (tid == 0 && head + total > a.n_free) fail(R);
  __syncthreads();
  if (!s_err) {
    for (int64_t j = tid; j < total; j += kThreads) {
      const int32_t id = a.free_pages[head + j];
      if (id < 0 || id >= a.n_pages) fail(R);
    }
  }
  __syncthreads();
  const bool ok = s_err == 0;
  if (tid == 0) {
    *d.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, s_detail, 0u};
    if (ok && a.free_head_out != nullptr) *a.free_head_out = static_cast<int32_t>(head + total);
  }
  if (!ok) return;
  for (int r = tid; r < R; r += kThreads)
    a.seq_len[r] = d.past[r] + a.cu_new[r + 1] - a.cu_new[r];
  if (!write_all) return;
  for (int r = warp; r < R; r += kThreads / 32) write_pages(d, r, lane, 32);
  write_slots(d, tid, kThreads);
}

__global__ void __launch_bounds__(kMapThreads) k_cache_slots_map(SlotsDev d) {
  pdl_wait();
  pdl_trigger();
  if (!d.st->layout_ok) return;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kMapThreads + threadIdx.x;
  const int64_t threads = static_cast<int64_t>(gridDim.x) * kMapThreads;
  for (int64_t r = at >> 5; r < d.a.n_requests; r += threads >> 5)
    write_pages(d, static_cast<int>(r), threadIdx.x & 31, 32);
  write_slots(d, at, threads);
}

}  // namespace

cudaError_t launch_cache_slots(const avtp_cache_slots_args_t& a, void* ws, const SlotsWs& p, cudaStream_t s) {
  SlotsDev d{a, ws_at<DevStatus>(ws, p.status), ws_at<int32_t>(ws, p.past), ws_at<int32_t>(ws, p.first)};
  const bool one = a.n_tokens <= kOneCtaTokens;
  const cudaError_t e = launch_kernel(k_cache_slots, dim3(1), dim3(kThreads), 0, s, /*pdl=*/true, d, one ? 1 : 0);
  if (e != cudaSuccess || one) return e;
  const int64_t want = (a.n_tokens + kMapThreads - 1) / kMapThreads, most = 4 * static_cast<int64_t>(device_sm_count());
  return launch_kernel(k_cache_slots_map, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(kMapThreads), 0, s,
                       /*pdl=*/true, d);
}

}  // namespace avtp
