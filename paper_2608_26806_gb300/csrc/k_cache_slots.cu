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
// kOneCtaTokens tokens the same CTA writes the maps; beyond, a second kernel over the whole GPU. What
// bounds either is latency, a chain of dependent loads: a step of 8 requests 4.0-4.5 us a call, of 256
// 4.6-5.1, of 1024 6.7; 2000 tokens of 64 requests 6.3 in one CTA, 2100 6.3 in two kernels, 5815 7.8 and 6.1,
// 15938 17.3 and 6.6, 142331 8.9 in two.
#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 1024;
constexpr int kMapThreads = 256;
constexpr int64_t kOneCtaTokens = 2048;

// Requests whose lengths are kept in shared memory. (2000 requests, a token each, 11.0 us and 11.3 when they are
// not, ten each 12.5 and 13.7.)
constexpr int kStaged = 2048;

struct SlotsDev {
  avtp_cache_slots_args_t a;
  DevStatus* st;
  int32_t* past;   // workspace copies, see SlotsWs
  int32_t* first;
};

// Per request: offset, cached tokens, entry of its first new page in the free list. In shared memory
// for up to kStaged requests: a token's request is then found by eleven quick loads, not eleven trips to L2.
struct Lengths {
  const int32_t *cu, *past, *first;
};

__device__ __forceinline__ int64_t ceil_div(int64_t x, int64_t p) { return (x + p - 1) / p; }

// New pages k, k + step, ... of `total`, from entry `head` of the free list on. (Page by page, not
// request by request: a step brings 256 requests a page or none each, a prefill eight of them hundreds.)
__device__ __forceinline__ void write_pages(const SlotsDev& d, const Lengths& l, int64_t head, int64_t total, int64_t k,
                                            int64_t step) {
  for (; k < total; k += step) {
    const int r = upper_index(l.first, d.a.n_requests, head + k);
    const int64_t have = ceil_div(l.past[r], d.a.page_size);
    d.a.block_table[r * d.a.table_stride + have + head + k - l.first[r]] = d.a.free_pages[head + k];
  }
}

// Slots of tokens t, t + step, ... New pages are read from the free list (their table entries may
// be another thread's to write).
__device__ __forceinline__ void write_slots(const SlotsDev& d, const Lengths& l, int64_t t, int64_t step) {
  const int R = d.a.n_requests, P = d.a.page_size;
  const int64_t live = l.cu[R];
  int r = -1;
  for (; t < d.a.n_tokens; t += step) {
    if (t >= live) {
      d.a.slot_map[t] = -1;
      continue;
    }
    if (r < 0 || t >= l.cu[r + 1]) r = upper_index(l.cu, R, t);
    // a request's length is a 32-bit number
    const uint32_t past = l.past[r], pos = past + static_cast<uint32_t>(t - l.cu[r]);
    const uint32_t page = pos / P, have = (past + P - 1u) / P;
    const int32_t id = page < have ? d.a.block_table[r * d.a.table_stride + page] : d.a.free_pages[l.first[r] + page - have];
    d.a.slot_map[t] = id * P + static_cast<int32_t>(pos - page * P);
  }
}

__global__ void __launch_bounds__(kThreads) k_cache_slots(SlotsDev d, int write_all) {
  __shared__ int s_err, s_detail;
  __shared__ int64_t s_warp[32], s_carry;
  __shared__ int32_t s_cu[kStaged + 1], s_past[kStaged], s_first[kStaged];
  pdl_wait();
  pdl_trigger();
  const avtp_cache_slots_args_t& a = d.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int R = a.n_requests;
  const int64_t P = a.page_size;
  const bool staged = R <= kStaged;
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
      const int32_t f = static_cast<int32_t>(first < a.n_free ? first : a.n_free);
      if (staged) {
        s_cu[r] = a.cu_new[r];
        s_past[r] = static_cast<int32_t>(past);
        s_first[r] = f;
        if (r == R - 1) s_cu[R] = a.cu_new[R];
      }
      if (!staged || !write_all) {
        d.past[r] = static_cast<int32_t>(past);
        d.first[r] = f;
      }
    }
    __syncthreads();
    if (tid == kThreads - 1) s_carry = before + incl;
    __syncthreads();
  }
  const int64_t total = s_carry;
  if (tid == 0 && head + total > a.n_free) fail(R);
  __syncthreads();
  if (!s_err) {
    // eight loads at a time: 8900 pages one after the other had taken 3 us
    bool bad = false;
    for (int64_t j0 = tid; j0 < total; j0 += 8 * kThreads) {
      int32_t id[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) id[i] = j0 + i * kThreads < total ? a.free_pages[head + j0 + i * kThreads] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) bad = bad || id[i] < 0 || id[i] >= a.n_pages;
    }
    if (bad) fail(R);
  }
  __syncthreads();
  const bool ok = s_err == 0;
  if (tid == 0) {
    *d.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, s_detail, 0u};
    if (ok && a.free_head_out != nullptr) *a.free_head_out = static_cast<int32_t>(head + total);
  }
  if (!ok) return;
  const Lengths l = staged ? Lengths{s_cu, s_past, s_first} : Lengths{a.cu_new, d.past, d.first};
  for (int r = tid; r < R; r += kThreads) a.seq_len[r] = l.past[r] + l.cu[r + 1] - l.cu[r];
  if (!write_all) return;
  write_pages(d, l, head, total, tid, kThreads);
  write_slots(d, l, tid, kThreads);
}

// The maps of a call whose lengths k_cache_slots has checked.
__global__ void __launch_bounds__(kMapThreads) k_cache_slots_map(SlotsDev d) {
  __shared__ int32_t s_cu[kStaged + 1], s_past[kStaged], s_first[kStaged];
  const int R = d.a.n_requests;
  const bool staged = R <= kStaged;
  if (staged)  // an input: it need not wait for the kernel ahead
    for (int i = threadIdx.x; i <= R; i += kMapThreads) s_cu[i] = d.a.cu_new[i];
  pdl_wait();
  pdl_trigger();
  if (!d.st->layout_ok) return;
  if (staged) {
    for (int i = threadIdx.x; i < R; i += kMapThreads) {
      s_past[i] = d.past[i];
      s_first[i] = d.first[i];
    }
    __syncthreads();
  }
  const Lengths l = staged ? Lengths{s_cu, s_past, s_first} : Lengths{d.a.cu_new, d.past, d.first};
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kMapThreads + threadIdx.x;
  const int64_t threads = static_cast<int64_t>(gridDim.x) * kMapThreads;
  const int64_t head = l.first[0];
  // the last request's pages end the list's part
  const int64_t past = l.past[R - 1], len = past + l.cu[R] - l.cu[R - 1];
  const int64_t total = l.first[R - 1] + ceil_div(len, d.a.page_size) - ceil_div(past, d.a.page_size) - head;
  write_pages(d, l, head, total, at, threads);
  write_slots(d, l, at, threads);
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
