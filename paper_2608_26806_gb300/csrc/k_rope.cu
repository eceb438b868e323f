// Rotary positions of queries and keys, behind the norm of each head where there is one, with the keys and
// values going to their slots of the paged cache:
//   y = x rsqrt(mean(x^2) + eps) w                    (x itself without a norm)
//   z_a = f (y_a cos t - y_b sin t),  z_b = f (y_b cos t + y_a sin t),  t = pos[plane_i] inv_freq_i
// for the pairs (a, b) = (i, i + rot/2) or (2i, 2i + 1) of a head's first rot elements; the others are y.
//
// What bounds it: bytes. Each q, k and v row is read and written once, and a head's norm and rotation are between. A
// head is D/16 lanes of 16 elements each, held as two pieces of V elements (or twice two of four) that turn into one
// another: piece u and piece u + rot/(2V) of the half style, two neighbours of the interleaved one, so that neither
// style moves elements between lanes and a call may write over its inputs. The norm's sum is three (D = 128) or two
// shuffles.
//
// Angles: far positions leave a 32-bit product no fraction. inv_freq / 2 pi is held as a 64-bit fraction of a turn,
// so that pos times it, modulo 2^64, is the angle modulo a turn in integers: its error is that of the fraction (2^-61
// of inv_freq, 2^-64 of a turn), times pos. The top 32 bits go to sincospif. A lane forms one or two of the token's
// cosines and sines for its warp; with the norm's weights they become 16 pairs of factors a lane, so that a word of
// two elements takes two packed products.
//
// A warp takes tokens and, where there are few of these, a share of their heads. Its rows come by asynchronous copies
// into shared memory that run four groups of heads ahead of the work, on into the next token's; what a lane copies it
// reads itself, so that nothing waits but the lane. (Rows loaded into registers, two groups at a time: 48 us for 9856
// tokens, now 42-44; the first form, a warp's 150 registers holding three groups and the weights read for each head,
// 127.)
//
// Measured, in a graph, with norms and the cache as destination: 32 query heads, 8 KV heads, d = 128: 64 tokens 3.6
// us, 1024 8.1, 9856 42.5, 20000 81.7, 6.0 TB/s; 16 and 16 heads of 64, whose rows go by 64 bytes: 9856 25.5, 4.8
// TB/s.
#include <type_traits>

#include "avtp_cache.cuh"
#include "avtp_tc.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kAhead = 4;       // groups of heads whose rows a warp has under way, a KiB each (three 43.2 us, six 42.5)
constexpr int kCtasOfSm = 4;    // up to 128 registers a thread (9856 tokens 42.5 us; five CTAs, 96 and spills 44.6, six 48.3)
constexpr int64_t kCheckTokens = 4096;
constexpr int kWarpsOfSm = 16;  // warps of an SM that a call's work is spread over, at least

struct RopeDev {
  avtp_rope_args_t a;
  avtp_cache_t c;   // k NULL: no cache
  int iq, ik;       // groups of heads of q, and of k or v
  int checked;      // a CTA of its own checks tables and slots
  DevStatus* st;
};

// inv_freq / 2 pi modulo 1 as a fraction of 2^64, by integers (in 64-bit floating point, scarce on this part, a
// prompt of 9856 tokens took 0.7 us more and a step of 64 0.2): inv_freq = m 2^-s with a 24-bit m, and m times 2^64 /
// 2 pi, shifted.
__device__ __forceinline__ uint64_t turn_fraction(float inv_freq) {
  constexpr uint64_t kTurn = 0x28be60db9391054aull;  // 2^64 / 2 pi
  const uint32_t b = __float_as_uint(inv_freq), e = (b >> 23) & 0xffu;
  const uint64_t m = (b & 0x7fffffu) | (e != 0 ? 0x800000u : 0u);
  const int s = 150 - static_cast<int>(e != 0 ? e : 1u);
  const uint64_t lo = m * kTurn, hi = __umul64hi(m, kTurn);
  uint64_t f = 0;
  if (s <= 0) f = s > -64 ? lo << -s : 0;
  else if (s < 64) f = (lo >> s) | (hi << (64 - s));
  else if (s < 128) f = hi >> (s - 64);
  return b >> 31 ? 0 - f : f;
}

// V elements of a row in registers.
template <int V>
struct Piece;
template <>
struct Piece<8> {
  uint4 w;
  __device__ __forceinline__ void load(const void* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ uint32_t& part(int i) { return i == 0 ? w.x : (i == 1 ? w.y : (i == 2 ? w.z : w.w)); }
};
template <>
struct Piece<4> {
  uint2 w;
  __device__ __forceinline__ void load(const void* p) { w = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint2*>(p) = w; }
  __device__ __forceinline__ uint32_t& part(int i) { return i == 0 ? w.x : w.y; }
};
template <int V>
__device__ __forceinline__ void copy_ahead(uint32_t to, const __nv_bfloat16* from) {
  if (V == 8) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// The call's tables and slots, by a CTA of its own: the others skip what it records, so that the status word has one
// writer and the call is one launch. Of more tokens than kCheckTokens, which one CTA would take longer to look
// through than the others to rotate (a million tokens of 4 + 2 heads of 64: 1.37 ms instead of 0.86), the warps
// record what they meet themselves, in a status word that a kernel ahead has cleared.
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
    constexpr int N = 16;
    for (int64_t t0 = threadIdx.x; t0 < d.a.n_tokens; t0 += N * kThreads) {
      int32_t s[N];
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = t0 + i * kThreads < d.a.n_tokens ? d.a.slot_map[t0 + i * kThreads] : -1;
#pragma unroll
      for (int i = 0; i < N; ++i) bad = bad || s[i] < -1 || s[i] >= slots;
    }
  }
  if (bad) s_bad = 1;
  __syncthreads();
  if (threadIdx.x == 0) *d.st = DevStatus{s_bad ? static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT) : 0, s_bad ? 0 : 1, 0, 0u};
}

template <int D, int V, bool kApart>
__global__ void __launch_bounds__(kThreads, kCtasOfSm) k_rope(RopeDev d) {
  constexpr int kLanes = D / 16;       // of a head
  constexpr int kHeads = 32 / kLanes;  // of a group
  constexpr int kUnits = 8 / V;        // pairs of pieces a lane
  constexpr int kMine = D / 64;        // pairs whose cosine and sine a lane forms
  static_assert(kApart || V == 8, "neighbours turn within pieces of eight");
  constexpr int kPieceBytes = 2 * V;
  // a lane's pieces of the groups under way: what a lane copies it reads itself
  __shared__ __align__(16) float s_turn[kWarps][2][D / 2];  // the token's cosines and sines, pair by pair
  __shared__ __align__(16) unsigned char s_ahead[kWarps][kAhead][kUnits][2][32 * kPieceBytes];
  pdl_wait();
  pdl_trigger();
  const int workers = static_cast<int>(gridDim.x) - d.checked;
  if (static_cast<int>(blockIdx.x) == workers) {
    if (blockIdx.y == 0) check(d);
    return;
  }
  const avtp_rope_args_t& a = d.a;
  const int lane = threadIdx.x & 31, sub = lane % kLanes, group = lane / kLanes;
  const int turning = a.rot_dim / 2;
  const bool part = a.rot_dim < D;  // some elements do not turn
  // pair e of a lane (of eight) is pair V (sub + kLanes (e / V)) + e % V of the head
  auto pair_of = [&](int e) { return V * (sub + kLanes * (e / V)) + e % V; };
  // its pieces' first elements, and whether four of its pairs turn (rot is a multiple of eight)
  int at[kUnits][2];
  bool turns[2];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = sub + kLanes * i, n = turning / V;
    at[i][0] = kApart ? (u < n ? u * V : 2 * u * V) : 2 * u * V;
    at[i][1] = kApart && u < n ? u * V + turning : at[i][0] + V;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) turns[i] = pair_of(4 * i) < turning;
  // whether the words of a piece turn
  auto turned = [&](int i, int h) { return turns[kUnits == 2 ? i : (kApart ? 0 : h)]; };

  // Tokens t, t + step, ... with a share (slice) of their groups of heads, its queries', keys' and values' in this
  // order: n of them, each of heads (slice + j slices) kHeads ... Copies run kAhead groups ahead of the work, through
  // a token's rows of every kind and on into the next token's.
  int64_t t = static_cast<int64_t>(blockIdx.x) * kWarps + threadIdx.x / 32;
  const int64_t step = static_cast<int64_t>(workers) * kWarps;
  const int slice = blockIdx.y, slices = gridDim.y;
  const int nq = slice < d.iq ? (d.iq - 1 - slice) / slices + 1 : 0, nk = slice < d.ik ? (d.ik - 1 - slice) / slices + 1 : 0;
  const int n = nq + nk + (d.c.k != nullptr ? nk : 0);
  if (n == 0) return;
  const uint32_t buffer = tc::smem_u32(s_ahead[threadIdx.x / 32][0][0][0]) + lane * kPieceBytes;
  int64_t ahead_t = t;
  int ahead_j = 0, ahead_stage = 0, stage = 0;
  auto issue = [&]() {
    if (ahead_t < a.n_tokens) {
      const bool is_q = ahead_j < nq, is_k = !is_q && ahead_j < nq + nk;
      const int head = (slice + (ahead_j - (is_q ? 0 : (is_k ? nq : nq + nk))) * slices) * kHeads + group;
      if (head < (is_q ? a.n_q_heads : a.n_kv_heads)) {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_q ? a.q : (is_k ? a.k : a.v)) +
                                   ahead_t * (is_q ? a.q_stride : (is_k ? a.k_stride : a.v_stride)) + head * D;
        const uint32_t to = buffer + ahead_stage * (kUnits * 2 * 32 * kPieceBytes);
#pragma unroll
        for (int i = 0; i < kUnits; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) copy_ahead<V>(to + (i * 2 + h) * 32 * kPieceBytes, src + at[i][h]);
      }
      if (++ahead_j == n) {
        ahead_j = 0;
        ahead_t += step;
      }
    }
    ahead_stage = ahead_stage + 1 == kAhead ? 0 : ahead_stage + 1;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // The next group, heads of a tensor of `heads`: `change` what was read, by the whole warp, and `store` it.
  auto pass = [&](int head, int heads, auto&& change, auto&& store) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    Piece<V> x[kUnits][2];
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) x[i][h].load(&s_ahead[threadIdx.x / 32][stage][i][h][lane * kPieceBytes]);
    change(x);
    stage = stage + 1 == kAhead ? 0 : stage + 1;
    issue();
    if (head < heads) store(x, head);
  };
  auto write = [&](const Piece<V> (&x)[kUnits][2], __nv_bfloat16* to) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      x[i][0].store(to + at[i][0]);
      x[i][1].store(to + at[i][1]);
    }
  };
  auto keep = [](Piece<V> (&)[kUnits][2]) {};
#pragma unroll 1
  for (int j = 0; j < kAhead; ++j) issue();

  // this lane's pairs: frequency and plane
  uint64_t freq[kMine];
  const int32_t* where[kMine];
  bool fine = true;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int p = pair_of(group * kMine + i);
    freq[i] = 0;
    where[i] = nullptr;
    if (p < turning) {
      const float f = a.inv_freq[p];
      const int plane = a.pair_plane != nullptr ? a.pair_plane[p] : 0;
      if (isfinite(f) && plane >= 0 && plane < a.n_planes) {
        freq[i] = turn_fraction(f);
        where[i] = a.pos + plane * a.pos_stride;
      } else {
        fine = false;
      }
    }
  }
  if (!__all_sync(0xffffffffu, fine)) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!d.checked && lane == 0) record_error(d.st, AVTP_ERR_DEVICE_INPUT, -1);
    return;
  }
  int32_t pos[kMine], slot = -1;  // of the next token
  auto look = [&](int64_t at_t) {
    if (at_t >= a.n_tokens) return;
#pragma unroll
    for (int i = 0; i < kMine; ++i) pos[i] = where[i] != nullptr ? where[i][at_t] : 0;
    if (d.c.k != nullptr) slot = a.slot_map[at_t];
  };
  look(t);

#pragma unroll 1
  for (; t < a.n_tokens; t += step) {
    __syncwarp();  // the token before has been set up
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const uint64_t phase = freq[i] * static_cast<uint64_t>(static_cast<int64_t>(pos[i]));
      float c, s;
      // half turns, -1 .. 1
      sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &s, &c);
      // (1 and 0 of pairs that do not turn)
      const int p = pair_of(group * kMine + i);
      s_turn[threadIdx.x / 32][0][p] = where[i] != nullptr ? c * a.attn_factor : 1.f;
      s_turn[threadIdx.x / 32][1][p] = where[i] != nullptr ? s * a.attn_factor : 0.f;
    }
    __syncwarp();
    int64_t page = -1, in_page = 0;
    if (!d.checked && lane == 0 && (slot < -1 || slot >= d.c.n_pages * d.c.page_size))
      record_error(d.st, AVTP_ERR_DEVICE_INPUT, static_cast<int32_t>(t));
    if (slot >= 0 && slot < d.c.n_pages * d.c.page_size) {
      page = static_cast<uint32_t>(slot) / static_cast<uint32_t>(d.c.page_size);
      in_page = slot - page * d.c.page_size;
    }
    look(t + step);

    // `count` groups, of queries or of keys, with their norm.
    auto turn = [&](int count, int heads, const void* norm, auto&& store) {
      if (norm == nullptr && turning == 0) {
#pragma unroll 1
        for (int j = 0; j < count; ++j) pass((slice + j * slices) * kHeads + group, heads, keep, store);
        return;
      }
      // what the two elements of a lane's word i (of eight) become: x * c[i] + partner * s[i], the norm's weights in
      // both
      float2 factor_c[8], factor_s[8];
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        Piece<V> w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (norm != nullptr) {
            w[h].load(static_cast<const __nv_bfloat16*>(norm) + at[i][h]);
          } else {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) w[h].part(e) = 0x3f803f80u;  // ones
          }
        }
        // the unit's pairs, two by two
        float2 cosines[V / 2], sines[V / 2];
#pragma unroll
        for (int e = 0; e < V / 2; e += 2) {
          const float4 c = *reinterpret_cast<const float4*>(&s_turn[threadIdx.x / 32][0][pair_of(i * V + 2 * e)]);
          const float4 s = *reinterpret_cast<const float4*>(&s_turn[threadIdx.x / 32][1][pair_of(i * V + 2 * e)]);
          cosines[e] = make_float2(c.x, c.y);
          cosines[e + 1] = make_float2(c.z, c.w);
          sines[e] = make_float2(s.x, s.y);
          sines[e + 1] = make_float2(s.z, s.w);
        }
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          // words e of the two pieces
          const int one = i * V + e, two = one + V / 2;
          const float2 w0 = make_float2(low(w[0].part(e)), high(w[0].part(e)));
          const float2 w1 = make_float2(low(w[1].part(e)), high(w[1].part(e)));
          if (kApart) {  // two pairs, their second elements in the second piece
            const float2 c = cosines[e], s = sines[e];
            factor_c[one] = tc::mul2(w0, c);
            factor_s[one] = tc::mul2(w1, make_float2(-s.x, -s.y));
            factor_c[two] = tc::mul2(w1, c);
            factor_s[two] = tc::mul2(w0, s);
          } else {  // pair e of the first piece, and of the second
            const float c = e & 1 ? cosines[e / 2].y : cosines[e / 2].x, s = e & 1 ? sines[e / 2].y : sines[e / 2].x;
            const float cc = e & 1 ? cosines[2 + e / 2].y : cosines[2 + e / 2].x;
            const float ss = e & 1 ? sines[2 + e / 2].y : sines[2 + e / 2].x;
            factor_c[one] = tc::mul2(w0, make_float2(c, c));
            factor_s[one] = tc::mul2(make_float2(w0.y, w0.x), make_float2(-s, s));
            factor_c[two] = tc::mul2(w1, make_float2(cc, cc));
            factor_s[two] = tc::mul2(make_float2(w1.y, w1.x), make_float2(-ss, ss));
          }
        }
      }
      auto change = [&](Piece<V> (&x)[kUnits][2]) {
        float2 y[8];
#pragma unroll
        for (int i = 0; i < kUnits; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < V / 2; ++e)
              y[i * V + h * (V / 2) + e] = make_float2(low(x[i][h].part(e)), high(x[i][h].part(e)));
        if (norm != nullptr) {
          float2 sq = make_float2(0.f, 0.f);
#pragma unroll
          for (int i = 0; i < 8; ++i) sq = tc::ffma2(y[i], y[i], sq);
          float sum = sq.x + sq.y;
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          const float inv = rsqrtf(fmaf(sum, 1.f / D, a.eps));
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = tc::mul2(y[i], make_float2(inv, inv));
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
              const int me = i * V + h * (V / 2) + e;
              float2 v = kApart ? y[i * V + (1 - h) * (V / 2) + e] : make_float2(y[me].y, y[me].x);
              if (part && !turned(i, h)) v = make_float2(0.f, 0.f);  // whatever it is, an infinity too
              const float2 z = tc::ffma2(y[me], factor_c[me], tc::mul2(v, factor_s[me]));
              // (elements that neither are normed nor turn keep their bits, a NaN's among them)
              if (!part || norm != nullptr || turned(i, h)) x[i][h].part(e) = tc::pack_bf16x2(z.x, z.y);
            }
      };
#pragma unroll 1
      for (int j = 0; j < count; ++j) pass((slice + j * slices) * kHeads + group, heads, change, store);
    };

    if (nq > 0) {
      __nv_bfloat16* row = static_cast<__nv_bfloat16*>(a.q_out) + t * a.q_out_stride;
      turn(nq, a.n_q_heads, a.q_norm, [&](const Piece<V> (&x)[kUnits][2], int head) { write(x, row + head * D); });
    }
    if (nk > 0) {
      __nv_bfloat16* row = static_cast<__nv_bfloat16*>(a.k_out) + t * a.k_out_stride;
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(d.c.k) + page * d.c.k_page_stride + in_page * d.c.k_token_stride;
      turn(nk, a.n_kv_heads, a.k_norm, [&](const Piece<V> (&x)[kUnits][2], int head) {
        if (a.k_out != nullptr) write(x, row + head * D);
        if (page >= 0) write(x, to + head * d.c.k_head_stride);
      });
    }
    if (n > nq + nk) {
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(d.c.v) + page * d.c.v_page_stride + in_page * d.c.v_token_stride;
#pragma unroll 1
      for (int j = 0; j < nk; ++j)
        pass((slice + j * slices) * kHeads + group, page >= 0 ? a.n_kv_heads : 0, keep,
             [&](const Piece<V> (&x)[kUnits][2], int head) { write(x, to + head * d.c.v_head_stride); });
    }
  }
}

}  // namespace

cudaError_t launch_rope(const avtp_rope_args_t& a, const avtp_cache_t* c, void* ws, cudaStream_t s) {
  RopeDev d{};
  d.a = a;
  if (a.n_tokens == 0) d.a.rot_dim = 0;  // its tables may be missing
  if (c != nullptr) d.c = *c;
  d.st = static_cast<DevStatus*>(ws);
  // warps share a token's groups of heads where there are few tokens
  const int heads = 512 / a.head_dim, most = a.n_q_heads > a.n_kv_heads ? a.n_q_heads : a.n_kv_heads;
  const int groups = (most + heads - 1) / heads;
  d.iq = (a.n_q_heads + heads - 1) / heads;
  d.ik = (a.n_kv_heads + heads - 1) / heads;
  int slices = 1;
  while (slices < groups && a.n_tokens * slices < static_cast<int64_t>(device_sm_count()) * kWarpsOfSm) ++slices;
  const int64_t want = (a.n_tokens + kWarps - 1) / kWarps, fit = static_cast<int64_t>(device_sm_count()) * kCtasOfSm / slices;
  d.checked = c == nullptr || a.n_tokens <= kCheckTokens ? 1 : 0;
  if (!d.checked) {
    const cudaError_t e = launch_cache_status(d.st, s);
    if (e != cudaSuccess) return e;
  }
  const dim3 grid(static_cast<unsigned>((slices == 1 && want > fit ? fit : want) + d.checked),
                  static_cast<unsigned>(slices));
  const bool apart = a.style == AVTP_ROPE_HALF;
  // half-style pairs whose halves begin inside a piece of eight are held as pieces of four
  const bool fours = apart && a.rot_dim % 16 != 0;
  auto pick = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    return fours ? k_rope<D, 4, true> : (apart ? k_rope<D, 8, true> : k_rope<D, 8, false>);
  };
  auto kernel = a.head_dim == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
  return launch_kernel(kernel, grid, dim3(kThreads), 0, s, /*pdl=*/true, d);
}

}  // namespace avtp
