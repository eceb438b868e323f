// Causal attention of a step's new tokens over the paged cache, keys split over CTAs:
//   O[t, h]   = sum_u softmax_u(scale * q[t, h] . k[u, g(h)]) v[u, g(h)]
//   lse[h, t] = ln sum_u exp(scale * q[t, h] . k[u, g(h)]),  u < seq_len - n + i + 1
// for the i-th of the request's n new tokens. Rows of a (request, KV head): its (new token, head
// of the group) pairs, token by token; they share the head's keys and values, which are read once
// for a block of 16 kWM rows.
//
// What bounds it: the cache's bytes. A tile of 64 keys is 32 KiB at d = 128, 1400 cycles of an
// SM's share of HBM; its products, by warp-level mma.sync (16 rows are too few for a tcgen05
// tile), take a fraction of that. So everything serves the stream of loads: a CTA per SM, a ring
// of tiles filled by TMA (a box per page piece, the pages' numbers looked up a tile ahead), and
// the whole call's tiles, taken as one line (request, KV head, row block, tile), cut into equal
// runs, one a CTA, whatever the requests' lengths. A run that begins or ends inside a row block
// leaves a piece (O, reference, sum) in the workspace; the CTA that finishes a block's last
// piece joins them, in their order, so results do not depend on who came last.
//
// Per tile and warp: S = Q K^T on the warp's 64 / (4 / kWM) keys and 16 rows, the running
// maximum m and sum l of exp2(c2 S - m) per row in registers, P in bf16 straight from S's
// registers as the A operand of P V. Rows' values are summed over the four warps' keys at the end
// of a row block. m, l and O are fp32; P is rounded to bf16 as the tensor core takes it (2^-9 of
// a weight, averaged over the keys), O once at the end.
//
// Warps 0-3 compute, warp 4 loads. Every wait is bounded; a CTA whose wait gives up records
// AVTP_ERR_TIMEOUT and leaves. Keys behind a request's last are masked by selection and their
// values cleared in registers, so nothing there (an infinity, a NaN) reaches a row.
#include <cudaTypedefs.h>

#include "avtp_cache.cuh"
#include "avtp_tc.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 160;
constexpr int kConsumers = 128;
constexpr int kLoadWarp = 4;
constexpr int kPrepThreads = 256;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

struct AttnDev {
  const __nv_bfloat16* q;
  int64_t q_stride;
  const int32_t* cu;
  const int32_t* seq;
  const int32_t* table;
  int64_t table_stride;
  int64_t n_tokens, n_pages;
  int R, max_new, max_pages, Hq, Hkv, G, page_size;
  int box;        // rows of a TMA box: a power of two that divides the page size, at most a tile
  int k_tok, v_tok;  // the map's second dimension is the row of the page, its third the head (else the reverse)
  float c2;
  __nv_bfloat16* o;
  int64_t o_stride;
  float* lse;
  int64_t lse_stride;
  DevStatus* st;
  int32_t* count;
  float* part_o;
  float2* part_ml;
};

// A run's part of one row block.
struct Segment {
  int32_t row0;        // the request's first packed row
  int32_t n, seq;      // its new tokens and cached tokens
  int32_t head, block; // KV head (-1: no more), row block
  int32_t tile0, tile1, tiles;
  int32_t c0, c1;      // CTAs of the block's first and last piece
  int32_t slot, slot0; // where this piece goes, when there are several, and the block's first
  int32_t req;
};

__host__ __device__ constexpr uint32_t stage_bytes(int d) { return 2u * kCacheTile * d * 2; }
__host__ __device__ constexpr int stages(int d) { return d == 128 ? 5 : 10; }
// A warp's O on its way to the others: 16 rows of d floats, 8 floats of padding so that the eight
// rows of an accumulator's column pair fall into different banks.
__host__ __device__ constexpr int out_row(int d) { return d + 8; }
__host__ __device__ constexpr size_t smem_bytes(int d) {
  return 1024 + static_cast<size_t>(stages(d)) * stage_bytes(d) + 4 * 16 * out_row(d) * 4;
}
static_assert(smem_bytes(128) <= 200 * 1024 && smem_bytes(64) <= 200 * 1024, "shared memory of one CTA");

template <int D>
struct Shared {
  uint64_t kv_full[stages(D)], kv_empty[stages(D)];
  uint64_t seg_full[2], seg_empty[2];
  Segment seg[2];
  int64_t pre[kThreads + 1];  // tiles before each thread's share of the requests
  float m[4][16], l[4][16];
  int32_t most;               // tiles of the longest row block
  int32_t last;
  int abort, bad_page;
};

// ---------------------------------------------------------------- what a request asks
struct Request {
  int32_t row0, n, seq;
  __device__ __forceinline__ bool load(const AttnDev& a, int r) {
    const int64_t lo = a.cu[r], hi = a.cu[r + 1];
    row0 = static_cast<int32_t>(lo);
    n = static_cast<int32_t>(hi - lo);
    seq = a.seq[r];
    return lo >= 0 && hi >= lo && hi <= a.n_tokens && hi - lo <= a.max_new && seq >= 0 &&
           seq <= static_cast<int64_t>(a.max_pages) * a.page_size && (r > 0 || lo == 0);
  }
  __device__ __forceinline__ int tiles() const { return n == 0 ? 0 : max(1, (seq + kCacheTile - 1) / kCacheTile); }
  __device__ __forceinline__ int blocks(const AttnDev& a, int rows) const {
    return static_cast<int>((static_cast<int64_t>(n) * a.G + rows - 1) / rows);
  }
};

// ---------------------------------------------------------------- validation
// The first kernel of a call: the status word, the counters, and what the lengths have wrong. The
// attention runs beside it and waits for it before its first use of either.
__global__ void __launch_bounds__(kPrepThreads) k_cache_prep(AttnDev a, int counters) {
  __shared__ int s_bad;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) s_bad = 0x7fffffff;
  __syncthreads();
  for (int i = threadIdx.x; i < counters; i += kPrepThreads) a.count[i] = 0;
  for (int r = threadIdx.x; r < a.R; r += kPrepThreads) {
    Request q;
    if (!q.load(a, r)) atomicMin(&s_bad, r);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool ok = s_bad == 0x7fffffff;
    *a.st = DevStatus{ok ? 0 : static_cast<int32_t>(AVTP_ERR_DEVICE_INPUT), ok ? 1 : 0, ok ? 0 : s_bad, 0u};
  }
}

// ---------------------------------------------------------------- building blocks
__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::
          "r"(tc::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(tc::smem_u32(bar))
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
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
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
__device__ __forceinline__ void store_row(const AttnDev& a, const Segment& g, int row, int col, float4 v, float m, float l) {
  const int tok = row / a.G, head = g.head * a.G + (row - tok * a.G);
  const int64_t t = static_cast<int64_t>(g.row0) + tok;
  const float inv = l == 0.f ? 0.f : 1.f / l;  // no key visible: zeros
  uint2 w;
  w.x = pack(v.x * inv, v.y * inv);
  w.y = pack(v.z * inv, v.w * inv);
  *reinterpret_cast<uint2*>(a.o + t * a.o_stride + static_cast<int64_t>(head) * D + col) = w;
  if (col == 0 && a.lse != nullptr) a.lse[head * a.lse_stride + t] = (m + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- attention
// mapK, mapV: the cache as {d, head, row of the page, page} (or {d, row, head, page}), box of 64
// elements, one head, `box` rows, one page. kWM warps share the keys of a slice of the tile, 16
// rows each.
template <int D, int kWM>
__global__ void __launch_bounds__(kThreads, 1)
k_cache_attn(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, AttnDev a) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ Shared<D> sh;
  constexpr int kStages = stages(D);
  constexpr int kRows = 16 * kWM;
  constexpr int kSlices = 4 / kWM;            // slices of a tile's keys
  constexpr int kKeys = kCacheTile / kSlices; // keys of a slice
  constexpr uint32_t kPanel = kCacheTile * 128;
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* s_out = reinterpret_cast<float*>(smem + kStages * stage_bytes(D));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&sh.kv_full[s], 1);
      tc::mbar_init(&sh.kv_empty[s], 4);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&sh.seg_full[s], 1);
      tc::mbar_init(&sh.seg_empty[s], 4);
    }
    sh.abort = 0;
    sh.bad_page = -1;
    sh.most = 1;
    tc::fence_mbar_init();
    tc::tma_prefetch_map(&mapK);
    tc::tma_prefetch_map(&mapV);
  }
  pdl_trigger();
  __syncthreads();

  // ---- the plan, by every CTA for itself: tiles before each thread's share of the requests
  const int share = (a.R + kThreads - 1) / kThreads;
  bool ok = true;
  {
    int64_t sum = 0;
    int most = 1;
    for (int r = tid * share; r < min(a.R, (tid + 1) * share); ++r) {
      Request q;
      ok = q.load(a, r) && ok;
      sum += static_cast<int64_t>(q.tiles()) * q.blocks(a, kRows) * a.Hkv;
      most = max(most, q.tiles());
    }
    atomicMax(&sh.most, most);
    sh.pre[tid + 1] = sum;
    if (tid == 0) sh.pre[0] = 0;
    ok = __syncthreads_and(ok);
    if (warp == 0) {
      int64_t carry = 0;
      for (int b = 0; b < kThreads; b += 32) {
        int64_t x = sh.pre[b + lane + 1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        x += carry;
        sh.pre[b + lane + 1] = x;
        carry = __shfl_sync(0xffffffffu, x, 31);
      }
    }
    __syncthreads();
  }
  const int64_t total = ok ? sh.pre[kThreads] : 0;  // lengths that validation refuses: nothing
  // CTAs at work: runs long enough that no row block has more than kCacheMaxPieces pieces
  const int64_t least = (sh.most + kCacheMaxPieces - 3) / (kCacheMaxPieces - 2);
  const int64_t N = max(int64_t(1), min(static_cast<int64_t>(gridDim.x), total / least));
  const int64_t t0 = blockIdx.x < N ? blockIdx.x * total / N : 0, t1 = blockIdx.x < N ? (blockIdx.x + 1) * total / N : 0;
  volatile int* abort_flag = &sh.abort;

  if (warp == kLoadWarp) {
    // ------------------------------------------------------------ segments and loads
    int r = 0;
    int64_t pre = 0;  // tiles before request r
    if (t0 < t1) {
      int lo = 0, hi = kThreads;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sh.pre[mid] <= t0) lo = mid; else hi = mid;
      }
      r = lo * share;
      pre = sh.pre[lo];
    }
    int n = 0, sc = 0;
    bool fine = true;
    for (int64_t t = t0; fine; ++sc) {
      Segment g{};
      g.head = -1;
      int64_t end = t;
      if (t < t1) {
        Request q;
        int64_t len;
        for (;; ++r) {
          q.load(a, r);
          len = static_cast<int64_t>(q.tiles()) * q.blocks(a, kRows) * a.Hkv;
          if (t < pre + len) break;
          pre += len;
        }
        const int tiles = q.tiles(), nb = q.blocks(a, kRows);
        const int64_t b = (t - pre) / tiles, s = pre + b * tiles;
        end = min(t1, s + tiles);
        g.row0 = q.row0;
        g.n = q.n;
        g.seq = q.seq;
        g.head = static_cast<int>(b / nb);
        g.block = static_cast<int>(b - static_cast<int64_t>(g.head) * nb);
        g.tile0 = static_cast<int>(t - s);
        g.tile1 = static_cast<int>(end - s);
        g.tiles = tiles;
        g.c0 = static_cast<int>(((s + 1) * N - 1) / total);
        g.c1 = static_cast<int>(((s + tiles) * N - 1) / total);
        // a CTA's first segment goes to its even slot, its last (the only other that can be a piece) to its odd one
        g.slot = 2 * blockIdx.x + (t == t0 ? 0 : 1);
        g.slot0 = 2 * g.c0 + (g.c0 * total / N == s ? 0 : 1);
        g.req = r;
      }
      if (sc >= 2) fine = tc::mbar_wait_warp(&sh.seg_empty[sc & 1], ((sc >> 1) - 1) & 1);
      if (!fine) break;
      if (lane == 0) {
        sh.seg[sc & 1] = g;
        tc::mbar_arrive(&sh.seg_full[sc & 1]);
      }
      __syncwarp();
      if (g.head < 0) break;
      const int32_t* row = a.table + g.req * a.table_stride;
      auto page_of = [&](int tile) {
        const int64_t key = static_cast<int64_t>(tile) * kCacheTile + lane * a.box;
        return (lane * a.box < kCacheTile && key < g.seq) ? row[key / a.page_size] : 0;
      };
      int page = page_of(g.tile0);
      for (int tile = g.tile0; tile < g.tile1; ++tile, ++n) {
        const int next = tile + 1 < g.tile1 ? page_of(tile + 1) : 0;
        const int sb = n % kStages;
        if (n >= kStages) fine = tc::mbar_wait_warp(&sh.kv_empty[sb], (n / kStages - 1) & 1);
        if (!fine || *abort_flag) break;
        const int keys = min(kCacheTile, g.seq - tile * kCacheTile);  // none: an empty cache
        const int boxes = keys <= 0 ? 0 : (keys + a.box - 1) / a.box;
        if (lane == 0) tc::mbar_arrive_expect_tx(&sh.kv_full[sb], boxes * a.box * D * 4);
        __syncwarp();
        if (lane < boxes) {
          if (page < 0 || page >= a.n_pages) {  // outside the pool: recorded, and another read in its place
            sh.bad_page = g.req;
            page = 0;
          }
          unsigned char* dst = smem + sb * stage_bytes(D) + lane * a.box * 128;
          const int in_page = (tile * kCacheTile + lane * a.box) % a.page_size;
#pragma unroll
          for (int p = 0; p < D / 64; ++p)
            tma_load_4d(dst + p * kPanel, &mapK, p * 64, a.k_tok ? in_page : g.head, a.k_tok ? g.head : in_page, page,
                        &sh.kv_full[sb]);
#pragma unroll
          for (int p = 0; p < D / 64; ++p)
            tma_load_4d(dst + (D / 64 + p) * kPanel, &mapV, p * 64, a.v_tok ? in_page : g.head,
                        a.v_tok ? g.head : in_page, page, &sh.kv_full[sb]);
        }
        __syncwarp();
        page = next;
      }
      if (!fine || *abort_flag) {
        fine = false;
        break;
      }
      t = end;
    }
    if (!fine && lane == 0) *abort_flag = 1;
    // let the copies in flight land before the CTA may exit
    for (int k = (n >= kStages ? n - kStages : 0); k < n; ++k)
      tc::mbar_wait_warp(&sh.kv_full[k % kStages], (k / kStages) & 1);
  } else {
    // ------------------------------------------------------------ products, softmax, output
    const int wm = warp % kWM, slice = warp / kWM;
    const int gr = lane >> 2, tq = lane & 3;  // this lane's row pair and column pair of an MMA
    const uint32_t base = tc::smem_u32(smem);
    const float c2 = a.c2;
    bool waited = false;
    int n = 0;
    for (int sc = 0;; ++sc) {
      if (!tc::mbar_wait_warp(&sh.seg_full[sc & 1], (sc >> 1) & 1)) *abort_flag = 1;
      bar_consumers();
      if (*abort_flag) break;
      const Segment g = sh.seg[sc & 1];
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sh.seg_empty[sc & 1]);
      if (g.head < 0) break;
      const int rows = min(kRows, g.n * a.G - g.block * kRows);  // of the block
      const int first = g.block * kRows;
      // Q as the A operand; keys visible to this lane's two rows
      uint32_t qa[D / 16][4];
      int limit[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = wm * 16 + gr + 8 * i;
        const int at = first + min(row, rows - 1);
        const int tok = at / a.G, head = g.head * a.G + (at - tok * a.G);
        limit[i] = min(g.seq, g.seq - g.n + tok + 1);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (static_cast<int64_t>(g.row0) + tok) * a.q_stride +
                                                                static_cast<int64_t>(head) * D);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          qa[ks][i] = row < rows ? src[ks * 8 + tq] : 0u;
          qa[ks][i + 2] = row < rows ? src[ks * 8 + tq + 4] : 0u;
        }
        if (row >= rows) limit[i] = 0;
      }
      const int all_see = g.seq - g.n + first / a.G + 1;  // keys that every row of the block sees

      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      float o[D / 8][4];
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

      for (int tile = g.tile0; tile < g.tile1; ++tile, ++n) {
        const int sb = n % kStages;
        if (!tc::mbar_wait_warp(&sh.kv_full[sb], (n / kStages) & 1)) {
          *abort_flag = 1;
          break;
        }
        const int key0 = tile * kCacheTile + slice * kKeys;
        if (key0 < g.seq) {
          const uint32_t kb = base + sb * stage_bytes(D), vb = kb + (D / 64) * kPanel;
          float s[kKeys / 8][4];
#pragma unroll
          for (int i = 0; i < kKeys / 8; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
            for (int kk = 0; kk < kKeys / 16; ++kk) {
              const int key = slice * kKeys + kk * 16 + ((lane >> 4) << 3) + (lane & 7);
              const int chunk = ks * 2 + ((lane >> 3) & 1);
              uint32_t b[4];
              ldsm4(kb + (chunk >> 3) * kPanel + key * 128 + (((chunk & 7) ^ (key & 7)) << 4), b);
              mma_16816(s[2 * kk], qa[ks], b[0], b[1]);
              mma_16816(s[2 * kk + 1], qa[ks], b[2], b[3]);
            }
          }
          if (key0 + kKeys > all_see) {
#pragma unroll
            for (int i = 0; i < kKeys / 8; ++i) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (key0 + i * 8 + 2 * tq + (e & 1) >= limit[e >> 1]) s[i][e] = -INFINITY;
            }
          }
          // the running maximum; O and l follow it
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < kKeys / 8; ++i) {
            mx[0] = fmaxf(mx[0], fmaxf(s[i][0], s[i][1]));
            mx[1] = fmaxf(mx[1], fmaxf(s[i][2], s[i][3]));
          }
          float f[2];
          bool moved = false;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float mn = fmaxf(m[i], quad_max(mx[i]) * c2);
            f[i] = mn == m[i] ? 1.f : (m[i] == -INFINITY ? 0.f : tc::ex2(m[i] - mn));
            moved = moved || mn != m[i];
            m[i] = mn;
            l[i] *= f[i];
          }
          if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
              o[i][0] *= f[0];
              o[i][1] *= f[0];
              o[i][2] *= f[1];
              o[i][3] *= f[1];
            }
          }
          const float m0 = m[0] == -INFINITY ? 0.f : m[0], m1 = m[1] == -INFINITY ? 0.f : m[1];
          uint32_t p[kKeys / 16][4];
#pragma unroll
          for (int i = 0; i < kKeys / 8; ++i) {
            const float p0 = tc::ex2(fmaf(s[i][0], c2, -m0)), p1 = tc::ex2(fmaf(s[i][1], c2, -m0));
            const float p2 = tc::ex2(fmaf(s[i][2], c2, -m1)), p3 = tc::ex2(fmaf(s[i][3], c2, -m1));
            l[0] += p0 + p1;
            l[1] += p2 + p3;
            p[i >> 1][(i & 1) * 2] = pack(p0, p1);
            p[i >> 1][(i & 1) * 2 + 1] = pack(p2, p3);
          }
          const bool tail = key0 + kKeys > g.seq;
#pragma unroll
          for (int kk = 0; kk < kKeys / 16; ++kk) {
            // values behind the request's last key: cleared, so that P = 0 meets no infinity
            const int left = g.seq - (key0 + kk * 16 + 2 * tq);
            const uint32_t k0 = left > 1 ? 0xffffffffu : (left == 1 ? 0xffffu : 0u);
            const uint32_t k1 = left > 9 ? 0xffffffffu : (left == 9 ? 0xffffu : 0u);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
              const int key = slice * kKeys + kk * 16 + (lane & 15);
              const int chunk = c * 2 + (lane >> 4);
              uint32_t b[4];
              ldsm4_t(vb + (chunk >> 3) * kPanel + key * 128 + (((chunk & 7) ^ (key & 7)) << 4), b);
              if (tail) {
                b[0] &= k0;
                b[1] &= k1;
                b[2] &= k0;
                b[3] &= k1;
              }
              mma_16816(o[2 * c], p[kk], b[0], b[1]);
              mma_16816(o[2 * c + 1], p[kk], b[2], b[3]);
            }
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
        }
      }
      bar_consumers();
      if (*abort_flag) break;
      const int pieces = g.c1 - g.c0 + 1;
      constexpr int kLanes = D / 4;               // lanes of a row, four columns each
      constexpr int kAtOnce = kConsumers / kLanes;  // rows at once
      const int sub = tid % kLanes, col = sub * 4;
      for (int row = tid / kLanes; row < rows; row += kAtOnce) {
        const int w = row / 16, rr = row % 16;
        float M = -INFINITY;
#pragma unroll
        for (int s = 0; s < kSlices; ++s) M = fmaxf(M, sh.m[s * kWM + w][rr]);
        float L = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int s = 0; s < kSlices; ++s) {
          const float ms = sh.m[s * kWM + w][rr];
          const float f = ms == -INFINITY ? 0.f : tc::ex2(ms - M);
          const float4 x = *reinterpret_cast<const float4*>(s_out + ((s * kWM + w) * 16 + rr) * out_row(D) + col);
          L += f * sh.l[s * kWM + w][rr];
          v.x = fmaf(f, x.x, v.x);
          v.y = fmaf(f, x.y, v.y);
          v.z = fmaf(f, x.z, v.z);
          v.w = fmaf(f, x.w, v.w);
        }
        if (pieces == 1) {
          store_row<D>(a, g, first + row, col, v, M, L);
        } else {
          __stcg(reinterpret_cast<float4*>(a.part_o + (static_cast<int64_t>(g.slot) * kRows + row) * D + col), v);
          if (sub == 0) __stcg(a.part_ml + static_cast<int64_t>(g.slot) * kRows + row, make_float2(M, L));
        }
      }
      if (pieces == 1) continue;

      // ---- a piece: the last of the block's to arrive joins them
      if (!waited) {
        pdl_wait();  // the counters are cleared by the kernel ahead
        waited = true;
      }
      __threadfence();
      bar_consumers();
      if (tid == 0) sh.last = atomicAdd(a.count + g.c0, 1) == pieces - 1;
      bar_consumers();
      if (!sh.last) continue;
      __threadfence();
      for (int row = tid / kLanes; row < rows; row += kAtOnce) {
        auto slot = [&](int k) { return (k == 0 ? g.slot0 : 2 * (g.c0 + k)) * static_cast<int64_t>(kRows) + row; };
        float M = -INFINITY;
#pragma unroll 8
        for (int k = 0; k < pieces; ++k) M = fmaxf(M, __ldcg(a.part_ml + slot(k)).x);
        float L = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = 0; k < pieces; ++k) {
          const float2 ml = __ldcg(a.part_ml + slot(k));
          const float4 x = __ldcg(reinterpret_cast<const float4*>(a.part_o + slot(k) * D + col));
          const float f = ml.x == -INFINITY ? 0.f : tc::ex2(ml.x - M);
          L = fmaf(f, ml.y, L);
          v.x = fmaf(f, x.x, v.x);
          v.y = fmaf(f, x.y, v.y);
          v.z = fmaf(f, x.z, v.z);
          v.w = fmaf(f, x.w, v.w);
        }
        store_row<D>(a, g, first + row, col, v, M, L);
      }
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

// The pool of one tensor, 64 elements x 1 head x `box` rows of a page in the 128-byte swizzle. A
// map's strides ascend, so head and row come in the order of theirs.
bool cache_map(CUtensorMap* m, const void* base, const avtp_cache_t& c, int64_t page, int64_t token, int64_t head,
               int box, bool tok_inner) {
  auto fn = encode_fn();
  if (fn == nullptr) return false;
  const cuuint64_t H = static_cast<cuuint64_t>(c.n_kv_heads), P = static_cast<cuuint64_t>(c.page_size);
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c.head_dim), tok_inner ? P : H, tok_inner ? H : P,
                              static_cast<cuuint64_t>(c.n_pages)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(tok_inner ? token : head) * 2,
                                 static_cast<cuuint64_t>(tok_inner ? head : token) * 2, static_cast<cuuint64_t>(page) * 2};
  const cuuint32_t b = static_cast<cuuint32_t>(box);
  const cuuint32_t boxes[4] = {64, tok_inner ? b : 1, tok_inner ? 1 : b, 1};
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, boxes, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int kWM>
cudaError_t launch_attn(int grid, const CUtensorMap& mk, const CUtensorMap& mv, const AttnDev& a, cudaStream_t s) {
  static PerDevice attrs;
  const cudaError_t e = once_per_device(attrs, [](int, int*) {
    return cudaFuncSetAttribute(k_cache_attn<D, kWM>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(smem_bytes(D)));
  });
  if (e != cudaSuccess) return e;
  return launch_kernel(k_cache_attn<D, kWM>, dim3(grid), dim3(kThreads), smem_bytes(D), s, /*pdl=*/true, mk, mv, a);
}

// Warps that share a slice of keys: 16 rows each, as many as a request can have, at most four.
int row_warps(const avtp_cache_t& c, const avtp_cache_attn_args_t& a) {
  const int64_t rows = static_cast<int64_t>(a.max_new) * (a.n_q_heads / c.n_kv_heads);
  return rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
}

}  // namespace

CacheAttnWs plan_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a) {
  CacheAttnWs p{};
  const size_t grid = static_cast<size_t>(device_sm_count()), rows = 16 * static_cast<size_t>(row_warps(c, a));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~static_cast<size_t>(255);
    return at;
  };
  p.status = take(sizeof(DevStatus));
  p.count = take(grid * 4);
  p.part_o = take(2 * grid * rows * static_cast<size_t>(c.head_dim) * 4);
  p.part_ml = take(2 * grid * rows * 8);
  p.total = off;
  return p;
}

cudaError_t launch_cache_attention(const avtp_cache_t& c, const avtp_cache_attn_args_t& a, void* ws,
                                   const CacheAttnWs& p, cudaStream_t s) {
  AttnDev d{};
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
  d.Hq = a.n_q_heads;
  d.Hkv = c.n_kv_heads;
  d.G = a.n_q_heads / c.n_kv_heads;
  d.page_size = c.page_size;
  d.box = 16;
  while (d.box < kCacheTile && c.page_size % (2 * d.box) == 0) d.box *= 2;
  d.k_tok = c.k_token_stride < c.k_head_stride ? 1 : 0;
  d.v_tok = c.v_token_stride < c.v_head_stride ? 1 : 0;
  d.c2 = a.softmax_scale * kLog2e;
  d.o = static_cast<__nv_bfloat16*>(a.o);
  d.o_stride = a.o_stride;
  d.lse = a.lse;
  d.lse_stride = a.lse_stride;
  d.st = ws_at<DevStatus>(ws, p.status);
  d.count = ws_at<int32_t>(ws, p.count);
  d.part_o = ws_at<float>(ws, p.part_o);
  d.part_ml = ws_at<float2>(ws, p.part_ml);
  const int grid = device_sm_count();
  cudaError_t e = launch_kernel(k_cache_prep, dim3(1), dim3(kPrepThreads), 0, s, /*pdl=*/true, d, grid);
  if (e != cudaSuccess || a.n_tokens == 0) return e;
  CUtensorMap mk, mv;
  if (!cache_map(&mk, c.k, c, c.k_page_stride, c.k_token_stride, c.k_head_stride, d.box, d.k_tok != 0) ||
      !cache_map(&mv, c.v, c, c.v_page_stride, c.v_token_stride, c.v_head_stride, d.box, d.v_tok != 0))
    return cudaErrorInvalidValue;
  const int wm = row_warps(c, a);
  auto launch = c.head_dim == 128 ? (wm == 1 ? launch_attn<128, 1> : wm == 2 ? launch_attn<128, 2> : launch_attn<128, 4>)
                                  : (wm == 1 ? launch_attn<64, 1> : wm == 2 ? launch_attn<64, 2> : launch_attn<64, 4>);
  return launch(grid, mk, mv, d, s);
}

}  // namespace avtp
