// Causal attention of a step's new tokens over the paged cache, keys split over CTAs:
//   O[t, h]   = sum_u softmax_u(scale * q[t, h] . k[u, g(h)]) v[u, g(h)]
//   lse[h, t] = ln sum_u exp(scale * q[t, h] . k[u, g(h)]),  u < seq_len - n + i + 1
// for the i-th of the request's n new tokens. Rows of a (request, KV head): its (new token, head
// of the group) pairs, token by token; they share the head's keys and values, which are read once
// for a block of 16 kWM rows.
//
// What bounds it: the cache's bytes. A tile of keys and values is 32 KiB (64 keys at d = 128, 128 at d = 64),
// 1400 cycles of an SM's share of HBM; its products, by warp-level mma.sync (32 rows are too few for a tcgen05
// tile), take less up to 16 rows and about as long for 32. So everything serves the stream of loads: a CTA per
// SM, a ring of tiles filled by TMA (a box per page piece, the pages' numbers looked up 32 boxes at a time),
// and the whole call's tiles, taken as one line (request, KV head, tile), cut into equal runs, one a CTA, none
// shorter than a thirtieth of the longest head's (kCacheMaxPieces). A run that begins or ends inside a KV
// head's keys leaves a piece (O, reference, sums) in the workspace; the CTA that finishes a head's last piece
// joins them, in their order, so results do not depend on who came last.
//
// Per tile and warp: S = Q K^T on the warp's kTile kWM / 4 keys and 16 rows, P = exp2(c2 S - m)
// against the row's reference m, in bf16 straight from S's registers as the A operand of P V, and
// the sum l of P. The warps' shares meet at the end of a segment. m, l and O are fp32. P is
// rounded to bf16 for its product (at most 2^-8 of a weight), O once at the end; O is divided by the sum of
// the rounded P, which one more product with a column of ones gives, so that a row that one key
// dominates loses nothing to the rounding (error of O against 64 bits, 2-norm, one request of 3425
// tokens with some sharp queries: 2.5e-3 divided by l, 1.9e-3 so; 1.6e-3 is O's own rounding), and the
// LSE takes l.
//
// Measured, calls one behind the other (d = 128, a token a request): four requests of 50000 tokens, 8 KV heads,
// 124-127 us, 6.5 TB/s; 64 of 200-8000, 4 KV heads, pages of 16, 98-102 us, 5.8 TB/s, the cache's bytes read
// once and nothing else. 64 of 700-4000 with 16 heads of 64: 146 us, 4.3 TB/s, where the pages hold a head's
// rows 128 bytes at a time among the others' (of the 256 bytes that a fetch brings, half have left L2 when the
// other head wants them: 1.43 times the keys and values come from DRAM); 111 us, 5.7 TB/s where they hold them
// one behind the other. One request of 3425 tokens, 8 KV heads, 9.2 us: 5700 cycles to the first load, two
// tiles in 3600, 2500 for the piece and its count, 3500 for the join.
//
// Warps 0-3 compute, warp 4 makes segments and loads keys, warp 5 values (one warp for both: one request of
// 3425 tokens 9.3 us instead of 9.05, four of 50000 124.3 instead of 123.6). Every wait is bounded; a CTA whose
// wait gives up records AVTP_ERR_TIMEOUT and leaves. Keys behind a request's last are masked by selection and
// their values cleared in registers, so nothing there (an infinity, a NaN) reaches a row.
#include <cudaTypedefs.h>

#include <type_traits>

#include "avtp_cache_attn.cuh"

namespace avtp {
namespace {

constexpr int kWarps = 4;  // that compute
constexpr int kConsumers = 32 * kWarps;
constexpr int kKeyWarp = kWarps;  // and the one behind it for the values
constexpr int kThreads = kConsumers + 64;
constexpr int kConsumerBar = 1;  // named barrier of the computing warps
constexpr int kPrepThreads = 256;
// A tile's share of a row's sum above kRescaleSum moves the row's reference, if its maximum exceeds
// the reference by more than kRescaleTau (log2 units).
constexpr float kRescaleSum = 16384.f;
constexpr float kRescaleTau = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// A run's part of one row block.
struct Segment {
  int32_t row0;        // the request's first packed row
  int32_t n, seq;      // its new tokens and cached tokens
  int32_t head;        // KV head (-1: no more)
  int32_t tile0, tile1;
  int32_t c0, c1;      // CTAs of the block's first and last piece
  int32_t req;
};

// Keys of a tile, 32 KiB of K and V either way. (Tiles of 64 at d = 64: 64 requests of 700-4000 tokens, 16
// heads, 154 us instead of 140; what a tile costs beside its bytes is the same.)
__host__ __device__ constexpr int tile_keys(int d) { return d == 128 ? 64 : 128; }
__host__ __device__ constexpr uint32_t stage_bytes(int d) { return 2u * tile_keys(d) * d * 2; }
constexpr int kStages = 5;
// A warp's O on its way to the others: 16 rows of d floats, 8 floats of padding so that the eight
// rows of an accumulator's column pair fall into different banks.
__host__ __device__ constexpr int out_row(int d) { return d + 8; }
__host__ __device__ constexpr size_t smem_bytes(int d) {
  return 1024 + static_cast<size_t>(kStages) * stage_bytes(d) + kWarps * 16 * out_row(d) * 4;
}
template <int D>
struct Shared {
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint64_t seg_full[2], seg_empty[2];
  Segment seg[2];
  CachePlan<kThreads> plan;
  CacheWindow window[2];  // of the keys' warp, of the values'
  float m[kWarps][16], l[kWarps][16], w[kWarps][16];  // reference, sum of P, of its rounded values
  int32_t last;
  int abort, bad_page;
};
constexpr size_t kMostShared = 227 * 1024;  // of a CTA
static_assert(smem_bytes(128) + sizeof(Shared<128>) <= kMostShared && smem_bytes(64) + sizeof(Shared<64>) <= kMostShared,
              "shared memory of one CTA");

// ---------------------------------------------------------------- validation
// The first kernel of a call: the status word, the counters, and what the lengths have wrong. The
// attention runs beside it and waits for it before its first use of either.
__global__ void __launch_bounds__(kPrepThreads) k_cache_prep(CacheAttnDev a, int counters) {
  __shared__ int s_bad;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) s_bad = 0x7fffffff;
  __syncthreads();
  for (int i = threadIdx.x; i < counters; i += kPrepThreads) a.count[i] = 0;
  for (int r = threadIdx.x; r < a.R; r += kPrepThreads) {
    CacheRequest q;
    if (!q.load(a, r)) atomicMin(&s_bad, r);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool ok = s_bad == 0x7fffffff;
    *a.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, ok ? 0 : s_bad, 0u};
  }
}

// ---------------------------------------------------------------- building blocks
__device__ __forceinline__ void bar_consumers() {
  asm volatile("bar.sync %0, %1;" ::"n"(kConsumerBar), "n"(kConsumers) : "memory");
}
// The same, and whether x holds for any of them: what decides whether they go on has to be one answer
// for all, or some would wait for others that have left.
__device__ __forceinline__ bool bar_consumers_any(bool x) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(x ? 1u : 0u), "n"(kConsumerBar), "n"(kConsumers)
      : "memory");
  return any != 0;
}
__device__ __forceinline__ void tma_load_5d(void* dst, const CUtensorMap* map, int row, int head, int page, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], [%6];" ::
          "r"(tc::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(head), "r"(page), "r"(tc::smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Over the four lanes of a row. (The maximum passes a NaN over; its exponential is NaN all the
// same and takes the row's sum with it.)
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

// A row's result, four columns a lane: O divided by its sum and rounded, and the LSE.
template <int D>
__device__ __forceinline__ void store_row(const CacheAttnDev& a, const Segment& g, int row, int col, float4 v, float m, float l,
                                          float w) {
  const int tok = row / a.G, head = g.head * a.G + (row - tok * a.G);
  const int64_t t = static_cast<int64_t>(g.row0) + tok;
  const float inv = w == 0.f ? 0.f : 1.f / w;  // no key visible: zeros
  const uint2 x = make_uint2(tc::pack_bf16x2(v.x * inv, v.y * inv), tc::pack_bf16x2(v.z * inv, v.w * inv));
  *reinterpret_cast<uint2*>(a.o + t * a.o_stride + static_cast<int64_t>(head) * D + col) = x;
  if (col == 0 && a.lse != nullptr) a.lse[head * a.lse_stride + t] = (m + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- attention
// Tiles of a row block: one for an empty cache, whose rows are zeros; none for requests without new
// tokens, or with more rows than this kernel takes.
template <int D>
__device__ __forceinline__ int tiles_of(const CacheAttnDev& a, const CacheRequest& q) {
  return q.n == 0 || q.rows(a) > a.few_rows ? 0 : max(1, (q.seq - 1) / tile_keys(D) + 1);
}

__device__ __forceinline__ int steps_of(const CacheAttnDev& a, int tiles) {
  return (tiles + (1 << a.step_shift) - 1) >> a.step_shift;
}

// A wait looks at one bit of a barrier's phase, so a warp may be at most one phase behind what it waits for.
// Every computing warp therefore waits for every tile of the ring, in order, and both loading warps for every
// release. (Warps that took tiles in turn, each waiting for its own alone, could find the ring's turn before
// still on its way, pass, release the stage early and have the loader arrive on a phase with no arrival left.)
//
// mapK, mapV: the cache as {64 elements, row of the page, panel of 64, head, page}, box of `box` rows
// and all panels of one head and page: one TMA instruction a page piece. (One a panel, at pages of 16
// rows 16 of them a tile, issued too slowly: 4.4 TB/s.) kWM warps share the keys of a slice of the tile, 16
// rows each: two from 17 rows on.
template <int D, int kWM>
__global__ void __launch_bounds__(kThreads, 1)
k_cache_attn(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, CacheAttnDev a) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ Shared<D> sh;
  constexpr int kRows = 16 * kWM;
  constexpr int kSlices = kWarps / kWM;       // slices of a tile's keys
  constexpr int kTile = tile_keys(D);
  constexpr int kKeys = kTile / kSlices;      // keys of a slice
  static_assert(kWarps % kWM == 0 && kKeys % 16 == 0 && kConsumers % (D / 4) == 0, "the computing warps' shares");
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* s_out = reinterpret_cast<float*>(smem + kStages * stage_bytes(D));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&sh.kv_full[s], 2);  // the keys' copies and the values'
      tc::mbar_init(&sh.kv_empty[s], kWarps);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&sh.seg_full[s], 1);
      tc::mbar_init(&sh.seg_empty[s], kWarps + 1);  // and the values' warp
    }
    sh.abort = 0;
    sh.bad_page = -1;
    tc::fence_mbar_init();
    tc::tma_prefetch_map(&mapK);
    tc::tma_prefetch_map(&mapV);
  }
  CacheRequest mine{};  // a lane's request of a call of few: on its way while the barriers are made
  bool mine_ok = true;
  if (warp == kKeyWarp && lane < a.R) mine_ok = mine.load(a, lane);
  pdl_trigger();
  __syncthreads();
  auto steps = [&](const CacheRequest& q, int& most) {
    const int t = steps_of(a, tiles_of<D>(a, q));
    most = max(most, t);
    return t * a.Hkv;
  };
  if (a.R > kNearRequests) sh.plan.form(a, steps);
  volatile int* abort_flag = &sh.abort;

  if (warp >= kKeyWarp) {
    // ------------------------------------------------------------ segments and keys; values
    const int kv = warp == kKeyWarp ? 0 : 1;
    const CUtensorMap* map = kv ? &mapV : &mapK;
    const int per_tile = kTile / a.box;
    CacheLine line;
    CacheRuns runs;
    int t = 0, t1 = 0, pre = 0, r = 0;  // steps: next, the run's end, before request r
    if (kv == 0) {
      line = CacheLine(a, sh.plan, mine, mine_ok, steps);
      runs = CacheRuns(line.total, line.most, 1, cache_ctas(a, line.weights, true));
      t = runs.begin(blockIdx.x);
      t1 = runs.begin(blockIdx.x + 1);
      if (t < t1) r = line.find(a, sh.plan, t, &pre);
    }
    int n = 0;
    bool fine = true;
#pragma unroll 1
    for (int sc = 0; fine; ++sc) {
      Segment g{};
      if (kv == 1) {
        fine = cache_wait_warp(&sh.seg_full[sc & 1], (sc >> 1) & 1);
        if (!fine) break;
        g = sh.seg[sc & 1];
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sh.seg_empty[sc & 1]);
      } else {
        g.head = -1;
        int end = t;
        if (t < t1) {
          CacheRequest q;
          int tiles, len;  // tiles and steps of a row block
#pragma unroll 1
          for (;; ++r) {
            q = line.request(a, mine, r);
            tiles = tiles_of<D>(a, q);
            len = steps_of(a, tiles);
            if (t < pre + len * a.Hkv) break;
            pre += len * a.Hkv;
          }
          g.head = static_cast<int>(static_cast<uint32_t>(t - pre) / static_cast<uint32_t>(len));
          const int s = pre + g.head * len;  // the block's first step
          end = min(t1, s + len);
          g.row0 = q.row0;
          g.n = q.n;
          g.seq = q.seq;
          g.tile0 = (t - s) << a.step_shift;
          g.tile1 = min(tiles, (end - s) << a.step_shift);
          g.c0 = t == s ? static_cast<int>(blockIdx.x) : runs.run(s);
          g.c1 = end == s + len ? static_cast<int>(blockIdx.x) : runs.run(s + len - 1);
          g.req = r;
        }
        if (sc >= 2) fine = cache_wait_warp(&sh.seg_empty[sc & 1], ((sc >> 1) - 1) & 1);
        if (!fine) break;
        if (lane == 0) {
          sh.seg[sc & 1] = g;
          tc::mbar_arrive(&sh.seg_full[sc & 1]);
        }
        __syncwarp();
        t = end;
      }
      if (g.head < 0) break;
      const int32_t* row = a.table + g.req * a.table_stride;
      for (int tile = g.tile0; tile < g.tile1 && !cache_raised(abort_flag); ++tile, ++n) {
        const int i0 = tile * per_tile, sb = n % kStages;
        if (tile == g.tile0 || (i0 & 31) == 0)
          if (sh.window[kv].load(a, row, g.seq, i0 & ~31)) sh.bad_page = g.req;
        const int keys = min(kTile, g.seq - tile * kTile);  // none: an empty cache
        const int boxes = keys <= 0 ? 0 : (keys + a.box - 1) / a.box;
        if (tc::elect_one()) {
          if (n >= kStages && !cache_wait(&sh.kv_empty[sb], (n / kStages - 1) & 1)) {
            *abort_flag = 1;
          } else {
            tc::mbar_arrive_expect_tx(&sh.kv_full[sb], boxes * a.box * D * 2);
            unsigned char* dst = smem + sb * stage_bytes(D) + kv * (stage_bytes(D) / 2);
#pragma unroll 1
            for (int b = 0; b < boxes; ++b, dst += a.box * D * 2) {
              const int2 at = sh.window[kv].at[(i0 + b) & 31];
              tma_load_5d(dst, map, at.y, g.head, at.x, &sh.kv_full[sb]);
            }
          }
        }
        __syncwarp();
      }
      fine = !cache_raised(abort_flag);
    }
    if (!fine && lane == 0) *abort_flag = 1;
    // let the copies in flight land before the CTA may exit
    for (int k = (n >= kStages ? n - kStages : 0); k < n; ++k)
      cache_wait_warp(&sh.kv_full[k % kStages], (k / kStages) & 1);
  } else {
    // ------------------------------------------------------------ products, softmax, output
    const int wm = warp % kWM, slice = warp / kWM;
    const int gr = lane >> 2, tq = lane & 3;  // this lane's row pair and column pair of an MMA
    const uint32_t base = tc::smem_u32(smem);
    const float c2 = a.c2;
    int n = 0;
    for (int sc = 0;; ++sc) {
      if (!cache_wait_warp(&sh.seg_full[sc & 1], (sc >> 1) & 1)) *abort_flag = 1;
      if (bar_consumers_any(*abort_flag != 0)) break;
      const Segment g = sh.seg[sc & 1];
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sh.seg_empty[sc & 1]);
      if (g.head < 0) break;
      const int rows = g.n * a.G;
      // Q as the A operand; keys visible to this lane's two rows
      uint32_t qa[D / 16][4];
      int limit[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = wm * 16 + gr + 8 * i;
        const int at = min(row, rows - 1);
        const int tok = at / a.G, head = g.head * a.G + (at - tok * a.G);
        limit[i] = min(g.seq, g.seq - g.n + tok + 1);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (static_cast<int64_t>(g.row0) + tok) * a.q_stride +
                                                                static_cast<int64_t>(head) * D);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          qa[ks][i] = row < rows ? src[ks * 8 + tq] : 0u;
          qa[ks][i + 2] = row < rows ? src[ks * 8 + tq + 4] : 0u;
        }
        // A row that is not stored: q = 0. It sees no more than the others, or 0 x NaN behind the request's
        // last key would have its warp look for the maximum and move stored rows' references.
        if (row >= rows) limit[i] = g.seq;
      }
      const int all_see = g.seq - g.n + 1;  // keys that every row sees

      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      float rs[4] = {0.f, 0.f, 0.f, 0.f};  // P times ones: rows gr and gr + 8 in rs[0] and rs[2]
      float o[D / 8][4];
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

      for (int tile = g.tile0; tile < g.tile1; ++tile, ++n) {
        const int sb = n % kStages;
        if (!cache_wait_warp(&sh.kv_full[sb], (n / kStages) & 1)) {
          *abort_flag = 1;
          break;
        }
        const int key0 = tile * kTile + slice * kKeys;
        if (key0 < g.seq) {
          // a box is its D / 64 panels of 128-byte rows one behind the other
          const uint32_t kb = base + sb * stage_bytes(D), vb = kb + stage_bytes(D) / 2, panel = a.box * 128;
          auto sixteen = [&](int kk) {  // 16 keys of the slice
            const int key = slice * kKeys + kk * 16;
            return static_cast<uint32_t>(key & ~(a.box - 1)) * (D * 2) + static_cast<uint32_t>(key & (a.box - 1)) * 128;
          };
          // S: two chains of products a tile of 8 keys, so that no product waits long for another
          float s[kKeys / 8][4];
          uint32_t f[D / 16][4];  // K, then V fragments of 16 keys
#pragma unroll
          for (int kk = 0; kk < kKeys / 16; ++kk) {
            const int key = ((lane >> 4) << 3) + (lane & 7);
            const uint32_t at = kb + sixteen(kk) + key * 128;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const int chunk = (ks & 3) * 2 + ((lane >> 3) & 1);
              ldsm4(at + (ks >> 2) * panel + ((chunk ^ (key & 7)) << 4), f[ks]);
            }
            float e[2][4] = {}, o2[2][4] = {};
#pragma unroll
            for (int ks = 0; ks < D / 16; ks += 2) {
              mma_16816(e[0], qa[ks], f[ks][0], f[ks][1]);
              mma_16816(e[1], qa[ks], f[ks][2], f[ks][3]);
              mma_16816(o2[0], qa[ks + 1], f[ks + 1][0], f[ks + 1][1]);
              mma_16816(o2[1], qa[ks + 1], f[ks + 1][2], f[ks + 1][3]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int x = 0; x < 4; ++x) s[2 * kk + i][x] = e[i][x] + o2[i][x];
          }
          auto load_v = [&](int kk) {
            const int key = lane & 15;
            const uint32_t at = vb + sixteen(kk) + key * 128;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
              const int chunk = (c & 3) * 2 + (lane >> 4);
              ldsm4_t(at + (c >> 2) * panel + ((chunk ^ (key & 7)) << 4), f[c]);
            }
          };
          load_v(0);
          if (key0 + kKeys > all_see) {
#pragma unroll
            for (int i = 0; i < kKeys / 8; ++i) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (key0 + i * 8 + 2 * tq + (e & 1) >= limit[e >> 1]) s[i][e] = -INFINITY;
            }
          }
          // P against the rows' references, and its sums. Only a sum above kRescaleSum, a row
          // without a reference, or a NaN makes the warp take the maximum, move the references
          // and compute P again.
          uint32_t p[kKeys / 16][4];
          float sum[2];
          auto exps = [&]() {
            const float m0 = m[0] == -INFINITY ? 0.f : m[0], m1 = m[1] == -INFINITY ? 0.f : m[1];
            sum[0] = sum[1] = 0.f;
#pragma unroll
            for (int i = 0; i < kKeys / 8; ++i) {
              const float p0 = tc::ex2(fmaf(s[i][0], c2, -m0)), p1 = tc::ex2(fmaf(s[i][1], c2, -m0));
              const float p2 = tc::ex2(fmaf(s[i][2], c2, -m1)), p3 = tc::ex2(fmaf(s[i][3], c2, -m1));
              sum[0] += p0 + p1;
              sum[1] += p2 + p3;
              p[i >> 1][(i & 1) * 2] = tc::pack_bf16x2(p0, p1);
              p[i >> 1][(i & 1) * 2 + 1] = tc::pack_bf16x2(p2, p3);
            }
          };
          exps();
          if (__any_sync(0xffffffffu, m[0] == -INFINITY || m[1] == -INFINITY || !(sum[0] <= kRescaleSum) ||
                                          !(sum[1] <= kRescaleSum))) {
            float f2[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float mx = -INFINITY;
#pragma unroll
              for (int k = 0; k < kKeys / 8; ++k) mx = fmaxf(mx, fmaxf(s[k][2 * i], s[k][2 * i + 1]));
              const float mb = quad_max(mx) * c2;  // -inf when nothing is visible
              f2[i] = 1.f;
              if (mb > m[i] + kRescaleTau) {
                f2[i] = m[i] == -INFINITY ? 0.f : tc::ex2(m[i] - mb);
                m[i] = mb;
              }
              l[i] *= f2[i];
              rs[2 * i] *= f2[i];
              rs[2 * i + 1] *= f2[i];
            }
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
              o[i][0] *= f2[0];
              o[i][1] *= f2[0];
              o[i][2] *= f2[1];
              o[i][3] *= f2[1];
            }
            exps();
          }
          l[0] += sum[0];
          l[1] += sum[1];
          const bool tail = key0 + kKeys > g.seq;
#pragma unroll
          for (int kk = 0; kk < kKeys / 16; ++kk) {
            if (kk > 0) load_v(kk);
            if (tail) {
              // values behind the request's last key: cleared, so that P = 0 meets no infinity
              const int left = g.seq - (key0 + kk * 16 + 2 * tq);
              const uint32_t k0 = left > 1 ? 0xffffffffu : (left == 1 ? 0xffffu : 0u);
              const uint32_t k1 = left > 9 ? 0xffffffffu : (left == 9 ? 0xffffu : 0u);
#pragma unroll
              for (int c = 0; c < D / 16; ++c) {
                f[c][0] &= k0;
                f[c][1] &= k1;
                f[c][2] &= k0;
                f[c][3] &= k1;
              }
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
              mma_16816(o[2 * c], p[kk], f[c][0], f[c][1]);
              mma_16816(o[2 * c + 1], p[kk], f[c][2], f[c][3]);
            }
            mma_16816(rs, p[kk], 0x3f803f80u, 0x3f803f80u);
          }
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sh.kv_empty[sb]);
      }

      // ---- the four warps' shares meet in shared memory
      float* mine = s_out + warp * 16 * out_row(D);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        *reinterpret_cast<float2*>(mine + gr * out_row(D) + i * 8 + 2 * tq) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(mine + (gr + 8) * out_row(D) + i * 8 + 2 * tq) = make_float2(o[i][2], o[i][3]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float sum = quad_sum(l[i]);
        if (tq == 0) {
          sh.m[warp][gr + 8 * i] = m[i];
          sh.l[warp][gr + 8 * i] = sum;
          sh.w[warp][gr + 8 * i] = rs[2 * i];
        }
      }
      if (bar_consumers_any(*abort_flag != 0)) break;
      const int pieces = g.c1 - g.c0 + 1;
      constexpr int kLanes = D / 4;               // lanes of a row, four columns each
      constexpr int kAtOnce = kConsumers / kLanes;  // rows at once
      const int sub = tid % kLanes, col = sub * 4;
      for (int row = tid / kLanes; row < rows; row += kAtOnce) {
        const int w = row / 16, rr = row % 16;
        float M = -INFINITY;
#pragma unroll
        for (int s = 0; s < kSlices; ++s) M = fmaxf(M, sh.m[s * kWM + w][rr]);
        float L = 0.f, W = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int s = 0; s < kSlices; ++s) {
          const float ms = sh.m[s * kWM + w][rr];
          const float f = ms == -INFINITY ? 0.f : tc::ex2(ms - M);
          const float4 x = *reinterpret_cast<const float4*>(s_out + ((s * kWM + w) * 16 + rr) * out_row(D) + col);
          L += f * sh.l[s * kWM + w][rr];
          W += f * sh.w[s * kWM + w][rr];
          v.x = fmaf(f, x.x, v.x);
          v.y = fmaf(f, x.y, v.y);
          v.z = fmaf(f, x.z, v.z);
          v.w = fmaf(f, x.w, v.w);
        }
        if (pieces == 1) {
          store_row<D>(a, g, row, col, v, M, L, W);
        } else {
          const int64_t at = static_cast<int64_t>(piece_place(blockIdx.x, g.tile0 == 0)) * kRows + row;
          __stcg(reinterpret_cast<float4*>(a.part_o + at * D + col), v);
          if (sub == 0) __stcg(a.part_ml + at, make_float4(M, L, W, 0.f));
        }
      }
      if (pieces == 1) continue;

      // ---- a piece: the last of the block's to arrive joins them
      bar_consumers();
      if (tid == 0) {
        pdl_wait();  // the counters are cleared by the kernel ahead
        // behind this CTA's piece, ahead of its reads of the others' (0.4 us less than two fences)
        int before;
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(a.count + g.c0) : "memory");
        sh.last = before == pieces - 1;
      }
      bar_consumers();
      if (!sh.last) continue;
      // Eight pieces of a row at a time or two of four rows, whichever takes fewer turns, each of which is one
      // trip to L2; a row's reference moves between turns. (One request of 3425 tokens, 7 rows a head in 27
      // pieces: 12.6 us the one way, 14.6 the other; 16 of 700-4000, 16 rows in 2 or 3: 39.5 and 37.9.) Beyond
      // 16 pieces, join_many: the first 11.0 us so, five tokens of 32 heads 18.7 -> 16.5. (For the second, and
      // for ten pieces a head, it would take 0.3 to 1.2 us more.)
      auto join = [&](auto rows_at_once) {
        constexpr int N = decltype(rows_at_once)::value, P = 8 / N;
        for (int row0 = tid / kLanes; row0 < rows; row0 += kAtOnce * N) {
          float M[N], L[N], W[N];
          float4 v[N];
#pragma unroll
          for (int i = 0; i < N; ++i) {
            M[i] = -INFINITY;
            L[i] = W[i] = 0.f;
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          }
#pragma unroll 1
          for (int k0 = 0; k0 < pieces; k0 += P) {
            float4 ml[N][P];
            float4 x[N][P];
#pragma unroll
            for (int k = 0; k < P; ++k) {
              const int64_t at = static_cast<int64_t>(piece_place(g.c0 + k0 + k, k0 + k == 0)) * kRows + row0;
#pragma unroll
              for (int i = 0; i < N; ++i) {
                ml[i][k] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
                x[i][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k0 + k < pieces && row0 + i * kAtOnce < rows) {
                  ml[i][k] = __ldcg(a.part_ml + at + i * kAtOnce);
                  x[i][k] = __ldcg(reinterpret_cast<const float4*>(a.part_o + (at + i * kAtOnce) * D + col));
                }
              }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
              float mn = M[i];
#pragma unroll
              for (int k = 0; k < P; ++k) mn = fmaxf(mn, ml[i][k].x);
              const float old = M[i] == -INFINITY ? 0.f : tc::ex2(M[i] - mn);
              M[i] = mn;
              L[i] *= old;
              W[i] *= old;
              v[i] = make_float4(v[i].x * old, v[i].y * old, v[i].z * old, v[i].w * old);
#pragma unroll
              for (int k = 0; k < P; ++k) {
                const float f = ml[i][k].x == -INFINITY ? 0.f : tc::ex2(ml[i][k].x - mn);
                L[i] = fmaf(f, ml[i][k].y, L[i]);
                W[i] = fmaf(f, ml[i][k].z, W[i]);
                v[i].x = fmaf(f, x[i][k].x, v[i].x);
                v[i].y = fmaf(f, x[i][k].y, v[i].y);
                v[i].z = fmaf(f, x[i][k].z, v[i].z);
                v[i].w = fmaf(f, x[i][k].w, v[i].w);
              }
            }
          }
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (row0 + i * kAtOnce < rows) store_row<D>(a, g, row0 + i * kAtOnce, col, v[i], M[i], L[i], W[i]);
        }
      };
      // A row in many pieces: their references and sums lie with the row's lanes, one or two a lane, and the
      // weights are formed once, while the first sixteen pieces' rows are on their way.
      auto join_many = [&]() {
        constexpr int P = 16, E = kCacheMaxPieces / kLanes;
        auto place = [&](int piece, int row) {
          return piece_place(g.c0 + piece, piece == 0) * static_cast<int64_t>(kRows) + row;
        };
        // the warp stays together: row0 of its first lanes
#pragma unroll 1
        for (int row0 = warp * 32 / kLanes; row0 < rows; row0 += kAtOnce) {
          const int row = row0 + lane / kLanes;
          const bool here = row < rows;
          float4 ml[E];
          float weight[E];
          float M = -INFINITY, L = 0.f, W = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int piece = sub + e * kLanes;
            ml[e] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
            if (piece < pieces && here) ml[e] = __ldcg(a.part_ml + place(piece, row));
          }
#pragma unroll 1
          for (int k0 = 0; k0 < pieces; k0 += P) {
            float4 x[P];
#pragma unroll
            for (int k = 0; k < P; ++k) {
              x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (k0 + k < pieces && here)
                x[k] = __ldcg(reinterpret_cast<const float4*>(a.part_o + place(k0 + k, row) * D + col));
            }
            if (k0 == 0) {
#pragma unroll
              for (int e = 0; e < E; ++e) M = fmaxf(M, ml[e].x);
#pragma unroll 1
              for (int o = kLanes / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
              for (int e = 0; e < E; ++e) {
                weight[e] = ml[e].x == -INFINITY ? 0.f : tc::ex2(ml[e].x - M);
                L = fmaf(weight[e], ml[e].y, L);
                W = fmaf(weight[e], ml[e].z, W);
              }
#pragma unroll 1
              for (int o = kLanes / 2; o > 0; o >>= 1) {
                L += __shfl_xor_sync(0xffffffffu, L, o);
                W += __shfl_xor_sync(0xffffffffu, W, o);
              }
            }
#pragma unroll
            for (int k = 0; k < P; ++k) {
              const float mine = E == 2 && k0 + k >= kLanes ? weight[E - 1] : weight[0];
              const float f = __shfl_sync(0xffffffffu, mine, k0 + k, kLanes);
              v.x = fmaf(f, x[k].x, v.x);
              v.y = fmaf(f, x[k].y, v.y);
              v.z = fmaf(f, x[k].z, v.z);
              v.w = fmaf(f, x[k].w, v.w);
            }
          }
          if (here) store_row<D>(a, g, row, col, v, M, L, W);
        }
      };
      const int turns = (rows + kAtOnce - 1) / kAtOnce;  // of one row a thread
      const int few = (turns + 3) / 4 * ((pieces + 1) / 2);
      if (pieces > 16 && turns * 2 < few) join_many();
      else if (few < turns * ((pieces + 7) / 8)) join(std::integral_constant<int, 4>{});
      else join(std::integral_constant<int, 1>{});
    }
  }
  pdl_wait();  // this grid's end implies the validation kernel's, which resets the status word
  __syncthreads();
  if (tid == 0) {
    if (sh.abort) record_error(a.st, AVTP_ERR_TIMEOUT, static_cast<int32_t>(blockIdx.x));
    if (sh.bad_page >= 0) record_error(a.st, AVTP_ERR_DEVICE_INPUT, sh.bad_page);
  }
}

// ---------------------------------------------------------------- host side
PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}

bool encode(CUtensorMap* m, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
            const cuuint32_t* box) {
  auto fn = encode_fn();
  const cuuint32_t es[5] = {1, 1, 1, 1, 1};
  return fn != nullptr && fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, es,
                             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Pool {  // one tensor of the cache; strides in bytes
  const void* base;
  cuuint64_t page, token, head;
};

// Whole rows, for k_cache_attn.
bool rows_map(CUtensorMap* m, const Pool& t, const avtp_cache_t& c, int box) {
  const cuuint64_t panels = static_cast<cuuint64_t>(c.head_dim) / 64;
  const cuuint64_t dims[5] = {64, static_cast<cuuint64_t>(c.page_size), panels, static_cast<cuuint64_t>(c.n_kv_heads),
                              static_cast<cuuint64_t>(c.n_pages)};
  const cuuint64_t strides[4] = {t.token, 128, t.head, t.page};
  const cuuint32_t boxes[5] = {64, static_cast<cuuint32_t>(box), static_cast<cuuint32_t>(panels), 1, 1};
  return encode(m, 5, t.base, dims, strides, boxes);
}
// A panel of 64 elements, for k_cache_chunk, whose operands want a tile's panels whole.
bool panel_map(CUtensorMap* m, const Pool& t, const avtp_cache_t& c, int box) {
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c.head_dim), static_cast<cuuint64_t>(c.page_size),
                              static_cast<cuuint64_t>(c.n_kv_heads), static_cast<cuuint64_t>(c.n_pages)};
  const cuuint64_t strides[3] = {t.token, t.head, t.page};
  const cuuint32_t boxes[4] = {64, static_cast<cuuint32_t>(box), 1, 1};
  return encode(m, 4, t.base, dims, strides, boxes);
}
// q as {d, head, token}, box of 64 elements, a group's heads, as many tokens as fit into 128 rows.
bool query_map(CUtensorMap* m, const avtp_cache_attn_args_t& a, int d, int G) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(a.n_q_heads),
                              static_cast<cuuint64_t>(a.n_tokens)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(d) * 2, static_cast<cuuint64_t>(a.q_stride) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(G), static_cast<cuuint32_t>(kChunkRows / 2 / G)};
  return encode(m, 3, a.q, dims, strides, box);
}

template <int D, int kWM>
cudaError_t launch_attn(int grid, const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttnDev& a, cudaStream_t s) {
  static PerDevice attrs;
  const cudaError_t e = once_per_device(attrs, [](int, int*) {
    return cudaFuncSetAttribute(k_cache_attn<D, kWM>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(smem_bytes(D)));
  });
  if (e != cudaSuccess) return e;
  return launch_kernel(k_cache_attn<D, kWM>, dim3(grid), dim3(kThreads), smem_bytes(D), s, /*pdl=*/true, mk, mv, a);
}

// What the call's bounds leave to each kernel.
struct Shape {
  int64_t rows;      // of a request's KV head, at most
  bool few, chunks;  // k_cache_attn, k_cache_chunk
  int64_t few_rows;
  int row_warps;     // of k_cache_attn: 16 rows each
};
Shape shape_of(const avtp_cache_t& c, const avtp_cache_attn_args_t& a) {
  Shape s{};
  s.rows = static_cast<int64_t>(a.max_new) * (a.n_q_heads / c.n_kv_heads);
  s.chunks = s.rows > kCacheFewRows;
  s.few = !s.chunks || a.n_requests > 1;
  s.few_rows = !s.few ? 0 : (s.chunks ? kCacheFewMixed : kCacheFewRows);
  const int64_t most = s.rows < s.few_rows ? s.rows : s.few_rows;
  s.row_warps = most <= 16 ? 1 : 2;
  return s;
}

}  // namespace

CacheAttnWs plan_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a) {
  CacheAttnWs p{};
  const Shape sh = shape_of(c, a);
  const size_t grid = static_cast<size_t>(device_sm_count()), d = static_cast<size_t>(c.head_dim);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~static_cast<size_t>(255);
    return at;
  };
  p.status = take(sizeof(DevStatus));
  p.count = take(grid * 4);
  if (sh.few) {
    const size_t rows = 16 * static_cast<size_t>(sh.row_warps);
    p.part_o = take(2 * grid * rows * d * 4);
    p.part_ml = take(2 * grid * rows * 16);
  }
  if (sh.chunks) {
    p.chunk_o = take(2 * grid * kChunkRows * d * 4);
    p.chunk_ml = take(2 * grid * kChunkRows * 8);
    p.split = take(grid * sizeof(CacheChunkSplit));
  }
  p.total = off;
  return p;
}

cudaError_t launch_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a, void* ws,
                                   const CacheAttnWs& p, cudaStream_t s) {
  const Shape sh = shape_of(c, a);
  CacheAttnDev d{};
  d.q = static_cast<const __nv_bfloat16*>(a.q);
  d.q_stride = a.q_stride;
  d.cu = a.cu_new;
  d.seq = a.seq_len;
  d.table = a.block_table;
  d.table_stride = a.table_stride;
  d.n_tokens = a.n_tokens;
  d.n_pages = c.n_pages;
  d.R = a.n_requests;
  d.max_new = a.max_new;
  d.max_pages = a.max_pages;
  d.Hkv = c.n_kv_heads;
  d.G = a.n_q_heads / c.n_kv_heads;
  d.page_size = c.page_size;
  d.few_rows = sh.few_rows;
  d.both = sh.few && sh.chunks ? 1 : 0;
  d.c2 = a.softmax_scale * kLog2e;
  d.o = static_cast<__nv_bfloat16*>(a.o);
  d.o_stride = a.o_stride;
  d.lse = a.lse;
  d.lse_stride = a.lse_stride;
  d.st = ws_at<DevStatus>(ws, p.status);
  d.count = ws_at<int32_t>(ws, p.count);
  d.part_o = ws_at<float>(ws, p.part_o);
  d.part_ml = ws_at<float4>(ws, p.part_ml);
  d.chunk_o = ws_at<float>(ws, p.chunk_o);
  d.chunk_ml = ws_at<float2>(ws, p.chunk_ml);
  d.split = ws_at<CacheChunkSplit>(ws, p.split);
  // steps of the longest line the bounds allow, below 2^31
  auto shift = [&](int64_t blocks, int64_t tiles) {
    int sft = 0;
    while (static_cast<double>(blocks) * static_cast<double>((tiles >> sft) + 4) * c.n_kv_heads >= 2147483648.0) ++sft;
    return sft;
  };
  // a request's keys, at most (CacheRequest refuses more)
  const int64_t table = static_cast<int64_t>(a.max_pages) * c.page_size, keys = table < kCacheMostKeys ? table : kCacheMostKeys;
  const int grid = device_sm_count();
  cudaError_t e = launch_kernel(k_cache_prep, dim3(1), dim3(kPrepThreads), 0, s, /*pdl=*/true, d, grid);
  if (e != cudaSuccess || a.n_tokens == 0) return e;
  const Pool pk{c.k, static_cast<cuuint64_t>(c.k_page_stride) * 2, static_cast<cuuint64_t>(c.k_token_stride) * 2,
                static_cast<cuuint64_t>(c.k_head_stride) * 2};
  const Pool pv{c.v, static_cast<cuuint64_t>(c.v_page_stride) * 2, static_cast<cuuint64_t>(c.v_token_stride) * 2,
                static_cast<cuuint64_t>(c.v_head_stride) * 2};
  // boxes no longer than a kernel's tile, and whole in a page
  auto box = [&](int tile) {
    int b = 16;
    while (b < tile && c.page_size % (2 * b) == 0) b *= 2;
    return b;
  };
  CUtensorMap mk, mv, mq;
  if (sh.few) {
    d.box = box(tile_keys(c.head_dim));
    d.step_shift = shift(a.n_requests, keys / tile_keys(c.head_dim));
    if (!rows_map(&mk, pk, c, d.box) || !rows_map(&mv, pv, c, d.box)) return cudaErrorInvalidValue;
    auto launch = c.head_dim == 128 ? (sh.row_warps == 1 ? launch_attn<128, 1> : launch_attn<128, 2>)
                                    : (sh.row_warps == 1 ? launch_attn<64, 1> : launch_attn<64, 2>);
    if ((e = launch(grid, mk, mv, d, s)) != cudaSuccess) return e;
  }
  if (!sh.chunks) return cudaSuccess;
  d.box = box(kChunkKeys);
  d.step_shift = shift(a.n_tokens / (2 * (kChunkRows / 2 / d.G)) + a.n_requests, keys / kChunkKeys);
  if (!panel_map(&mk, pk, c, d.box) || !panel_map(&mv, pv, c, d.box) || !query_map(&mq, a, c.head_dim, d.G))
    return cudaErrorInvalidValue;
  return launch_cache_chunk(c.head_dim, grid, mq, mk, mv, d, s);
}

}  // namespace avtp
