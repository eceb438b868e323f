// Rotary positions of queries and keys, behind the norm of each head where there is one, with the keys and
// values going to their slots of the paged cache:
//   y = x rsqrt(mean(x^2) + eps) w                    (x itself without a norm)
//   z_a = f (y_a cos t - y_b sin t),  z_b = f (y_b cos t + y_a sin t),  t = pos[plane_i] inv_freq_i
// for the pairs (a, b) = (i, i + rot/2) or (2i, 2i + 1) of a head's first rot elements; the others are y.
//
// What bounds it: bytes. Each q, k and v row is read and written once, and a head's norm and rotation are
// between. A head is D/16 lanes of 16 elements each, held as two pieces of V elements (or twice two of four) that
// turn into one another: piece u and piece u + rot/(2V) of the half style, two neighbours of the interleaved one, so
// that neither style moves elements between lanes and a call may write over its inputs. The norm's sum is three (D =
// 128) or two shuffles.
//
// Angles: far positions leave a 32-bit product no fraction. inv_freq / 2 pi is held as a 64-bit fraction of
// a turn, so that pos times it, modulo 2^64, is the angle modulo a turn in integers: its error is that of the fraction, 2^-53
// of inv_freq, times pos (position 2^31: 4e-7 rad). The top 32 bits go to sincospif. A lane forms one or two of the
// token's cosines and sines for its warp, which shuffles hand round: a warp serves a token's heads one group
// after the other, or a share of them where there are few tokens.
#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBatch = 3;       // groups of heads that a warp has under way
constexpr int kWarpsOfSm = 24;  // warps of an SM that a call's work is spread over, at least

struct RopeDev {
  avtp_rope_args_t a;
  avtp_cache_t c;   // k NULL: no cache
  int slices;       // shares of a token's heads, a warp each
  int iq, ik, iv;   // groups of heads of q, k and v
  DevStatus* st;
};

// Positions in turns: inv_freq / 2 pi modulo 1 as a fraction of 2^64.
__device__ __forceinline__ uint64_t turn_fraction(float inv_freq) {
  const double f = static_cast<double>(inv_freq) * 0.15915494309189533577;
  return __double2ull_rn((f - floor(f)) * 18446744073709551616.0);
}

template <int V>
struct Piece;
template <>
struct Piece<8> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void load_near(const __nv_bfloat16* p) { w = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ uint32_t& part(int i) { return i == 0 ? w.x : (i == 1 ? w.y : (i == 2 ? w.z : w.w)); }
};
template <>
struct Piece<4> {
  uint2 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void load_near(const __nv_bfloat16* p) { w = __ldg(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint2*>(p) = w; }
  __device__ __forceinline__ uint32_t& part(int i) { return i == 0 ? w.x : w.y; }
};
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

// The call's tables and slots, by a CTA of its own: the others skip what it records, so that the status word
// has one writer and the call is one launch.
__device__ void check(const RopeDev& d) {
  __shared__ int s_bad;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  bool bad = false;
  for (int i = threadIdx.x; i < d.a.rot_dim / 2; i += kThreads) {
    bad = bad || !isfinite(d.a.inv_freq[i]);
    if (d.a.pair_plane != nullptr) bad = bad || d.a.pair_plane[i] < 0 || d.a.pair_plane[i] >= d.a.n_planes;
  }
  if (d.c.k != nullptr) {
    const int64_t slots = d.c.n_pages * d.c.page_size;
    for (int64_t t0 = threadIdx.x; t0 < d.a.n_tokens; t0 += 8 * kThreads) {
      int32_t s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = t0 + i * kThreads < d.a.n_tokens ? d.a.slot_map[t0 + i * kThreads] : -1;
#pragma unroll
      for (int i = 0; i < 8; ++i) bad = bad || s[i] < -1 || s[i] >= slots;
    }
  }
  if (bad) s_bad = 1;
  __syncthreads();
  if (threadIdx.x == 0) *d.st = DevStatus{s_bad ? static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT) : 0, s_bad ? 0 : 1, 0, 0u};
}

template <int D, int V>
__global__ void __launch_bounds__(kThreads) k_rope(RopeDev d) {
  constexpr int kLanes = D / 16;      // of a head
  constexpr int kHeads = 32 / kLanes;  // of a group
  constexpr int kUnits = 8 / V;       // pairs of pieces a lane
  constexpr int kMine = D / 64;       // pairs whose cosine and sine a lane forms
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == gridDim.x - 1) {
    check(d);
    return;
  }
  const avtp_rope_args_t& a = d.a;
  const int lane = threadIdx.x & 31, sub = lane % kLanes, group = lane / kLanes;
  const bool apart = a.style == AVTP_ROPE_HALF;
  const int turning = a.rot_dim / 2;
  // pair e of a lane (of eight) is pair V (sub + kLanes (e / V)) + e % V of the head
  auto pair_of = [&](int e) { return V * (sub + kLanes * (e / V)) + e % V; };
  // its pieces' first elements, and whether four of its pairs turn (rot is a multiple of eight)
  int at[kUnits][2];
  bool turns[2];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = sub + kLanes * i, n = turning / V;
    at[i][0] = apart ? (u < n ? u * V : 2 * u * V) : 2 * u * V;
    at[i][1] = apart && u < n ? u * V + turning : at[i][0] + V;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) turns[i] = pair_of(4 * i) < turning;
  uint64_t freq[kMine];
  const int32_t* where[kMine];
  bool fine = true;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int p = pair_of(group * kMine + i);
    freq[i] = 0;
    where[i] = a.pos;
    if (p < turning) {
      const float f = a.inv_freq[p];
      const int plane = a.pair_plane != nullptr ? a.pair_plane[p] : 0;
      fine = fine && isfinite(f) && plane >= 0 && plane < a.n_planes;
      freq[i] = fine ? turn_fraction(f) : 0;
      where[i] += fine ? plane * a.pos_stride : 0;
    }
  }
  if (!__all_sync(0xffffffffu, fine)) return;  // recorded by check()

  const int groups = d.iq + d.ik + d.iv;
  const int64_t items = a.n_tokens * d.slices, step = static_cast<int64_t>(gridDim.x - 1) * kWarps;
  const uint32_t slots = static_cast<uint32_t>(d.c.n_pages * d.c.page_size);
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + threadIdx.x / 32; item < items; item += step) {
    const int64_t t = item / d.slices;
    const int slice = static_cast<int>(item - t * d.slices);
    int32_t pos[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) pos[i] = turning > 0 ? where[i][t] : 0;
    int64_t page = -1, in_page = 0;
    if (d.c.k != nullptr) {
      const int32_t slot = a.slot_map[t];
      if (slot >= 0 && static_cast<uint32_t>(slot) < slots) {
        page = static_cast<uint32_t>(slot) / static_cast<uint32_t>(d.c.page_size);
        in_page = slot - page * d.c.page_size;
      }
    }
    float cs[8], sn[8];
    bool formed = false;
    for (int g0 = slice; g0 < groups; g0 += kBatch * d.slices) {
      Piece<V> x[kBatch][kUnits][2];
      int head[kBatch], what[kBatch];  // 0: a query's, 1: a key's, 2: a value's; -1: none
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int g = g0 + b * d.slices;
        const bool is_q = g < d.iq, is_k = !is_q && g < d.iq + d.ik;
        head[b] = (g - (is_q ? 0 : (is_k ? d.iq : d.iq + d.ik))) * kHeads + group;
        what[b] = g >= groups || head[b] >= (is_q ? a.n_q_heads : a.n_kv_heads) ? -1 : (is_q ? 0 : (is_k ? 1 : 2));
        if (what[b] < 0) continue;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_q ? a.q : (is_k ? a.k : a.v)) +
                                   t * (is_q ? a.q_stride : (is_k ? a.k_stride : a.v_stride)) + head[b] * D;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
          x[b][i][0].load(src + at[i][0]);
          x[b][i][1].load(src + at[i][1]);
        }
      }
      if (!formed && turning > 0) {
        formed = true;
        float c[kMine], s[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const uint64_t phase = freq[i] * static_cast<uint64_t>(static_cast<int64_t>(pos[i]));
          // half turns, -1 .. 1
          sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &s[i], &c[i]);
          c[i] *= a.attn_factor;
          s[i] *= a.attn_factor;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          cs[e] = __shfl_sync(0xffffffffu, c[e % kMine], e / kMine * kLanes + sub);
          sn[e] = __shfl_sync(0xffffffffu, s[e % kMine], e / kMine * kLanes + sub);
        }
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int g = g0 + b * d.slices;
        if (g >= groups) break;
        const bool is_v = g >= d.iq + d.ik;
        const void* norm = g < d.iq ? a.q_norm : a.k_norm;
        if (!is_v && (norm != nullptr || turning > 0)) {
          // first and second of the lane's pairs, pair e = 2 i .. : (a, b) of the half style lie in two pieces
          float y[kUnits][2][V];
#pragma unroll
          for (int i = 0; i < kUnits; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < V / 2; ++e) {
                const uint32_t w = what[b] < 0 ? 0u : x[b][i][h].part(e);
                y[i][h][2 * e] = low(w);
                y[i][h][2 * e + 1] = high(w);
              }
          if (norm != nullptr) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kUnits; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < V; ++e) sum = fmaf(y[i][h][e], y[i][h][e], sum);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float inv = rsqrtf(fmaf(sum, 1.f / D, a.eps));
#pragma unroll
            for (int i = 0; i < kUnits; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                Piece<V> w;
                w.load_near(static_cast<const __nv_bfloat16*>(norm) + at[i][h]);
#pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                  y[i][h][2 * e] *= inv * low(w.part(e));
                  y[i][h][2 * e + 1] *= inv * high(w.part(e));
                }
              }
          }
          auto turn = [&](float& p, float& q, int e) {
            const float first = p * cs[e] - q * sn[e];
            q = q * cs[e] + p * sn[e];
            p = first;
          };
          if (apart) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (turns[e / 4]) turn(y[e / V][0][e % V], y[e / V][1][e % V], e);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              constexpr int kPairs = V / 2;  // of a piece
              const int i = e / V, h = e / kPairs % 2, k = e % kPairs;
              if (turns[e / 4]) turn(y[i][h][2 * k], y[i][h][2 * k + 1], e);
            }
          }
          // (elements that neither are normed nor turn keep their bits, a NaN's among them)
#pragma unroll
          for (int i = 0; i < kUnits; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (norm != nullptr || turns[kUnits == 2 ? i : (apart ? 0 : h)]) {
#pragma unroll
                for (int e = 0; e < V / 2; ++e) x[b][i][h].part(e) = pack(y[i][h][2 * e], y[i][h][2 * e + 1]);
              }
        }
        auto store = [&](__nv_bfloat16* to) {
#pragma unroll
          for (int i = 0; i < kUnits; ++i) {
            x[b][i][0].store(to + at[i][0]);
            x[b][i][1].store(to + at[i][1]);
          }
        };
        if (what[b] == 0) {
          store(static_cast<__nv_bfloat16*>(a.q_out) + t * a.q_out_stride + head[b] * D);
        } else if (what[b] > 0) {
          if (what[b] == 1 && a.k_out != nullptr)
            store(static_cast<__nv_bfloat16*>(a.k_out) + t * a.k_out_stride + head[b] * D);
          if (page >= 0) {
            if (what[b] == 1)
              store(static_cast<__nv_bfloat16*>(d.c.k) + page * d.c.k_page_stride + in_page * d.c.k_token_stride +
                    head[b] * d.c.k_head_stride);
            else
              store(static_cast<__nv_bfloat16*>(d.c.v) + page * d.c.v_page_stride + in_page * d.c.v_token_stride +
                    head[b] * d.c.v_head_stride);
          }
        }
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope(const avtp_rope_args_t& a, const avtp_cache_t* c, void* ws, cudaStream_t s) {
  RopeDev d{};
  d.a = a;
  if (c != nullptr) d.c = *c;
  const int heads = 512 / a.head_dim;
  d.iq = (a.n_q_heads + heads - 1) / heads;
  d.ik = (a.n_kv_heads + heads - 1) / heads;
  d.iv = c != nullptr ? d.ik : 0;
  d.st = static_cast<DevStatus*>(ws);
  const int groups = d.iq + d.ik + d.iv, sms = device_sm_count();
  d.slices = 1;
  while (d.slices * kBatch < groups && a.n_tokens * d.slices < static_cast<int64_t>(sms) * kWarpsOfSm) ++d.slices;
  const int64_t want = (a.n_tokens * d.slices + kWarps - 1) / kWarps, most = static_cast<int64_t>(sms) * 8;
  const unsigned grid = static_cast<unsigned>((want < most ? want : most) + 1);
  // half-style pairs whose halves begin inside a piece of eight are held as pieces of four
  const bool fours = a.style == AVTP_ROPE_HALF && a.rot_dim % 16 != 0;
  auto kernel = a.head_dim == 128 ? (fours ? k_rope<128, 4> : k_rope<128, 8>) : (fours ? k_rope<64, 4> : k_rope<64, 8>);
  return launch_kernel(kernel, dim3(grid), dim3(kThreads), 0, s, /*pdl=*/true, d);
}

}  // namespace avtp
