// Causal attention over the paged cache for requests that bring many rows a KV head (new tokens x
// heads of the group): chunks of a prompt, and what k_cache_attn.cu's rows are too few for. The
// quantity is that file's; the products run on tcgen05.
//
// Rows are packed token by token: a tile of 128 MMA rows is floor(128 / G) tokens x the G heads of
// a KV head, brought by one TMA box a panel, so that a group's heads share every key and value
// that the SM fetches and a short chunk still fills its tile. A unit is two neighbouring tiles (slots)
// of one KV head on one stream of key blocks of 128:
//   S_j = Q K_j^T           tcgen05, M = 128 rows, N = 128 keys, operands in shared memory
//   P_j = exp2(c2 S_j - m)  a thread per row; bf16, over S_j's first 64 TMEM columns
//   O  += P_j V_j           tcgen05, A (P) from TMEM, V the MN-major operand as the pages hold it
// with the softmax, the order of MMAs and the ring of k_attn_fwd.cu (which see for what they
// measured): while one slot's softmax runs, the tensor core has the other slot's products.
// Keys come as TMA boxes of a page's rows, a lane a box, each after a look at the block table a block
// ahead.
//
// Units are few (a chunk of 512 tokens, G = 4: eight a KV head) and of unequal length, so
// their key blocks, taken as one line (request, unit, head, block), are cut into equal runs, a
// CTA each. A unit that a cut falls into leaves pieces (O, reference and sum of each row) in the
// workspace, and k_cache_join puts them together in their order: results do not depend on which
// came first.
//
// What bounds it: the tensor core (2048 cycles a block and unit at d = 128, the exponentials half
// of that), and for short calls the pieces' way through L2.
//
// Warps 0-3: softmax and output of slot 0, 4-7 of slot 1 (warp w owns rows 32 (w % 4) ..). Warp 8:
// segments, table, TMA. Warp 9: TMEM and the MMAs. Every wait is bounded; a CTA whose wait gives up
// records AVTP_ERR_TIMEOUT and leaves.
#include <type_traits>

#include "avtp_cache_attn.cuh"

namespace avtp {
namespace {

constexpr int kQT = 128;  // rows of a slot (MMA M, TMEM lanes)
constexpr int kKB = 128;  // keys of a block (MMA N of Q K^T, K of P V)
constexpr int kThreads = 320;
constexpr int kSlotWarps = 4;
constexpr int kTmaWarp = 8;
constexpr int kMmaWarp = 9;
constexpr int kStages = 4;      // key or value blocks in shared memory
constexpr int kLeastBlocks = 4; // key blocks of a run, at least
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kSCol = 0;    // S (and P) of slot s at kSCol + 128 s
constexpr uint32_t kOCol = 256;  // O of slot s at kOCol + 128 s
// A half's sum of P above kRescaleSum moves the row's reference, if its maximum exceeds the
// reference by more than kRescaleTau (log2 units).
constexpr float kRescaleSum = 16384.f;
constexpr float kRescaleTau = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
static_assert(kChunkRows == 2 * kQT, "two slots a unit");

__host__ __device__ constexpr uint32_t tile_bytes(int d) { return static_cast<uint32_t>(kQT) * d * 2; }
constexpr uint32_t kPanel = kQT * 128;
constexpr uint32_t kOutStage = 32 * 64;  // a warp's 32 rows x 32 columns of O on their way out
__host__ __device__ constexpr size_t chunk_smem_bytes(int d) {
  const size_t need = 1024 + static_cast<size_t>(2 + kStages) * tile_bytes(d) + 2 * kSlotWarps * kOutStage;
  // more than half the SM's shared memory, so that no second CTA (and its 512 TMEM columns)
  // shares an SM
  return need > 116 * 1024 ? need : 116 * 1024;
}
static_assert(chunk_smem_bytes(128) + sizeof(int64_t) * (kThreads + 1) <= 224 * 1024, "shared memory of one CTA");

// A run's part of one unit: key blocks j0 .. j1 - 1.
struct Segment {
  int32_t row0, n, seq;  // the request's first packed row, new and cached tokens
  int32_t head, unit;    // KV head (-1: no more), unit of the request
  int32_t j0, j1;
  int32_t place;         // where the piece goes; -1: the unit is whole
  int32_t req;
  int32_t nt;            // tokens of a slot

  // the slot's first token, and behind its last
  __device__ __forceinline__ int tok0(int s) const { return (2 * unit + s) * nt; }
  __device__ __forceinline__ int tok1(int s) const { return min(tok0(s) + nt, n); }
  __device__ __forceinline__ bool live(int s) const { return tok0(s) < n; }
  // keys that the slot's last token sees, and the slot's key blocks in this segment
  __device__ __forceinline__ int blocks(int s) const {
    if (!live(s)) return 0;
    const int all = max(1, (seq - n + tok1(s) + kKB - 1) / kKB);
    return max(0, min(j1, all) - j0);
  }
};

struct ChunkSync {
  uint64_t seg_full[2], seg_empty[2];
  uint64_t q_full, q_empty;
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint64_t s_full[2];      // S of a slot written by the MMA
  uint64_t p_full[2][2];   // half of a slot's P written by the softmax (and S read out)
  uint64_t pv_done[2][2];  // P V complete up to that half of a block
  uint64_t drain;
  Segment seg[2];
  CachePlan<kThreads> plan;
  uint32_t tmem;
  int abort, bad_page;
};

// Key blocks of a request's unit: those of its last token, one for a token that sees nothing.
__device__ __forceinline__ int unit_blocks(const CacheRequest& q, int nt, int u) {
  return max(1, (q.seq - q.n + static_cast<int>(min((u + 1) * static_cast<int64_t>(2 * nt), static_cast<int64_t>(q.n))) +
                 kKB - 1) / kKB);
}
__device__ __forceinline__ int units_of(const CacheAttnDev& a, const CacheRequest& q, int nt) {
  return q.rows(a) > a.few_rows ? (q.n + 2 * nt - 1) / (2 * nt) : 0;
}

// ---------------------------------------------------------------- attention
// mapQ: q {d, Hq, T}, box 64 x G x floor(128 / G); mapK, mapV: the cache as
// {d, row of the page, head, page}, box of 64 elements and `box` rows.
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
k_cache_chunk(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
              const __grid_constant__ CUtensorMap mapV, CacheAttnDev a) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ ChunkSync sy;
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  constexpr uint32_t kTile = tile_bytes(D);
  unsigned char* sQ = smem;                   // slot s at sQ + s * kTile
  unsigned char* sKV = smem + 2 * kTile;      // stage b at sKV + b * kTile
  unsigned char* sO = sKV + kStages * kTile;  // warp w at sO + w * kOutStage
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nt = kQT / a.G;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&sy.kv_full[s], 1);
      tc::mbar_init(&sy.kv_empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&sy.seg_full[s], 1);
      tc::mbar_init(&sy.seg_empty[s], 2 * kSlotWarps + 1);
      tc::mbar_init(&sy.s_full[s], 1);
      for (int h = 0; h < 2; ++h) {
        tc::mbar_init(&sy.p_full[s][h], kSlotWarps);
        tc::mbar_init(&sy.pv_done[s][h], 1);
      }
    }
    tc::mbar_init(&sy.q_full, 1);
    tc::mbar_init(&sy.q_empty, 1);
    tc::mbar_init(&sy.drain, 1);
    sy.abort = 0;
    sy.bad_page = -1;
    tc::fence_mbar_init();
    tc::tma_prefetch_map(&mapQ);
    tc::tma_prefetch_map(&mapK);
    tc::tma_prefetch_map(&mapV);
  }
  if (warp == kMmaWarp) {
    tc::tmem_alloc(&sy.tmem, kTmemCols);
    tc::tmem_relinquish();
  }
  // the rows behind a slot's nt * G, which no box writes: zeros
  for (uint32_t i = threadIdx.x; i < 2 * kTile / 16; i += kThreads) reinterpret_cast<uint4*>(sQ)[i] = make_uint4(0u, 0u, 0u, 0u);
  tc::fence_proxy_async();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  pdl_trigger();
  const uint32_t tmem = sy.tmem;
  volatile int* abort_flag = &sy.abort;

  sy.plan.form(a, [&](const CacheRequest& q, int& most) {
    const int U = units_of(a, q, nt);
    int64_t sum = 0;
    for (int u = 0; u < U; ++u) sum += unit_blocks(q, nt, u);
    if (U > 0) most = max(most, unit_blocks(q, nt, U - 1));
    return sum * a.Hkv;
  });
  const CacheRuns runs(sy.plan.pre[kThreads], sy.plan.most, kLeastBlocks);
  const int64_t t0 = runs.begin(blockIdx.x), t1 = runs.begin(blockIdx.x + 1);

  if (warp == kTmaWarp) {
    // ------------------------------------------------------------ segments and TMA loads
    int64_t pre = 0;  // steps before unit u of request r
    int r = t0 < t1 ? sy.plan.find(a, t0, &pre) : 0, u = 0;
    CacheChunkSplit split{};
    split.c1 = -1;
    int sc = 0, n = 0;  // segments published, ring places used (K, V, K, V, ...)
    bool ok = true;
    for (int64_t t = t0;; ++sc) {
      Segment g{};
      g.head = -1;
      int64_t end = t;
      if (t < t1) {
        CacheRequest q;
        int nb;
        for (;; ++r, u = 0) {
          q.load(a, r);
          const int U = units_of(a, q, nt);
          for (; u < U; ++u) {
            nb = unit_blocks(q, nt, u);
            if (t < pre + static_cast<int64_t>(nb) * a.Hkv) break;
            pre += static_cast<int64_t>(nb) * a.Hkv;
          }
          if (u < U) break;
        }
        g.row0 = q.row0;
        g.n = q.n;
        g.seq = q.seq;
        g.nt = nt;
        g.unit = u;
        g.req = r;
        g.head = static_cast<int>((t - pre) / nb);
        const int64_t s = pre + static_cast<int64_t>(g.head) * nb;  // the unit's first step
        end = min(t1, s + nb);
        g.j0 = static_cast<int>(t - s);
        g.j1 = static_cast<int>(end - s);
        const int c0 = runs.cta(s), c1 = runs.cta(s + nb - 1);
        // a CTA's first segment goes to its even place, its last (the only other that can be a piece) to its odd one
        g.place = c0 == c1 ? -1 : 2 * static_cast<int>(blockIdx.x) + (t == t0 ? 0 : 1);
        if (c0 < c1 && c0 == static_cast<int>(blockIdx.x))
          split = CacheChunkSplit{g.row0, g.n, g.head, g.unit, c0, c1, g.place, 0};
      }
      if (sc >= 2) ok = tc::mbar_wait_warp(&sy.seg_empty[sc & 1], ((sc >> 1) - 1) & 1);
      if (!ok) break;
      if (lane == 0) {
        sy.seg[sc & 1] = g;
        tc::mbar_arrive(&sy.seg_full[sc & 1]);
      }
      __syncwarp();
      if (g.head < 0) break;
      if (sc >= 1) ok = tc::mbar_wait_warp(&sy.q_empty, (sc - 1) & 1);
      if (!ok) break;
      const int nq = g.live(1) ? 2 : 1;
      if (lane == 0) {
        tc::mbar_arrive_expect_tx(&sy.q_full, nq * (D / 64) * nt * a.G * 128);
        for (int s = 0; s < nq; ++s)
          for (int ac = 0; ac < D / 64; ++ac)
            tc::tma_load_3d(sQ + s * kTile + ac * kPanel, &mapQ, ac * 64, g.head * a.G, g.row0 + g.tok0(s), &sy.q_full);
      }
      __syncwarp();
      const int32_t* row = a.table + g.req * a.table_stride;
      auto page_of = [&](int j) {
        const int64_t key = static_cast<int64_t>(j) * kKB + lane * a.box;
        return (lane * a.box < kKB && key < g.seq) ? row[key / a.page_size] : 0;
      };
      int page = page_of(g.j0);
      for (int j = g.j0; j < g.j1 && ok; ++j) {
        const int next = j + 1 < g.j1 ? page_of(j + 1) : 0;
        const int keys = min(kKB, g.seq - j * kKB);  // none: an empty cache
        const int boxes = keys <= 0 ? 0 : (keys + a.box - 1) / a.box;
        if (lane < boxes && (page < 0 || page >= a.n_pages)) {  // outside the pool: recorded, another read in its place
          sy.bad_page = g.req;
          page = 0;
        }
        const int in_page = (j * kKB + lane * a.box) % a.page_size;
        for (int kv = 0; kv < 2; ++kv, ++n) {
          const int sb = n % kStages;
          ok = n < kStages || tc::mbar_wait_warp(&sy.kv_empty[sb], (n / kStages - 1) & 1);
          if (!ok || *abort_flag) {
            ok = false;
            break;
          }
          if (lane == 0) tc::mbar_arrive_expect_tx(&sy.kv_full[sb], boxes * a.box * D * 2);
          __syncwarp();
          if (lane < boxes) {
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
              tma_load_4d(sKV + sb * kTile + p * kPanel + lane * a.box * 128, kv ? &mapV : &mapK, p * 64,
                          in_page, g.head, page, &sy.kv_full[sb]);
          }
          __syncwarp();
        }
        page = next;
      }
      // the ring's places are constants of a step: an odd pair is passed on empty
      for (; ok && n % kStages != 0; ++n) {
        const int sb = n % kStages;
        ok = n < kStages || tc::mbar_wait_warp(&sy.kv_empty[sb], (n / kStages - 1) & 1);
        if (ok && lane == 0) tc::mbar_arrive(&sy.kv_full[sb]);
        __syncwarp();
      }
      if (!ok) {
        ++sc;
        break;
      }
      t = end;
    }
    if (lane == 0) {
      if (!ok) *abort_flag = 1;
      a.split[blockIdx.x] = split;
    }
    // let the copies in flight land before the CTA may exit
    if (sc >= 1) tc::mbar_wait_warp(&sy.q_full, (sc - 1) & 1);
    for (int k = (n >= kStages ? n - kStages : 0); k < n; ++k)
      tc::mbar_wait_warp(&sy.kv_full[k % kStages], (k / kStages) & 1);
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------ MMA issuer
    // One elected lane issues (see elect_one), serving both slots in turn, which keeps their
    // softmaxes half a period apart. Every barrier is looked at before the commit ahead of it, and
    // waited for only if it was not complete then.
    if (tc::elect_one()) {
      constexpr uint32_t idS = tc::idesc_bf16(kQT, kKB);
      constexpr uint32_t idO = tc::idesc_bf16(kQT, D) | (1u << 16);  // B (V) MN-major
      const uint32_t q_base = tc::smem_u32(sQ), kv_base = tc::smem_u32(sKV);
      bool bad = false;
      auto wait = [&](uint64_t* bar, uint32_t parity, bool seen) {
        if (!seen && !bad) bad = !tc::mbar_wait(bar, parity);
      };
      auto s_mmas = [&](int s, int stage) {
        const uint64_t dq = tc::desc_k_sw128(q_base + s * kTile), dk = tc::desc_k_sw128(kv_base + stage * kTile);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint32_t off = static_cast<uint32_t>((ks >> 2) * kPanel + (ks & 3) * 32) / 16;  // in 16-byte units
          tc::mma_bf16(tmem + kSCol + s * 128, dq + off, dk + off, idS, ks > 0 ? 1u : 0u);
        }
      };
      // half of O of slot s += P_j V_j, 16 keys an MMA; only the first `steps` of the block's eight
      // where the request's keys end in it
      auto pv_mmas = [&](int s, int j, int stage, int steps, int half) {
        const uint64_t dv = tc::desc_mn_sw128(kv_base + stage * kTile, kPanel);
        const uint32_t tP = tmem + kSCol + s * 128, tO = tmem + kOCol + s * 128;
        if (steps == kKB / 16) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int ks = half * 4 + k;
            tc::mma_bf16_ts(tO, tP + ks * 8, dv + ks * (2048 / 16), idO, (j > 0 || ks > 0) ? 1u : 0u);
          }
        } else {
#pragma unroll 1
          for (int ks = half * 4; ks < min(half * 4 + 4, steps); ++ks)
            tc::mma_bf16_ts(tO, tP + ks * 8, dv + ks * (2048 / 16), idO, (j > 0 || ks > 0) ? 1u : 0u);
        }
      };
      using std::integral_constant;
      // Step j, odd or even: V_j sits in stage 1 or 3, K_{j + 1} in stage 2 or 0, and the next
      // step's blocks in the other two (kStages is 4); ph: the ring phase of V_j; pb[s]: the
      // phase of slot s's barriers at the segment's block 0. p0, kv, kk: whether the first half
      // of the next P and the next V and K were seen complete.
      static_assert(kStages == 4, "stages of a step are compile-time constants");
      bool p0 = false, kv = false, kk = false;
      uint32_t pb[2] = {0, 0};
      int n0 = 0, n1 = 0, nm = 0, last_steps = 0;
      auto slot_group = [&](auto odd, auto slot, int j, uint32_t ph, bool more) {
        constexpr int kOdd = decltype(odd)::value, s = decltype(slot)::value;
        constexpr int sv = kOdd ? 3 : 1, sk = kOdd ? 0 : 2, sv1 = kOdd ? 1 : 3, sk1 = kOdd ? 2 : 0;
        const int steps = j == nm - 1 ? last_steps : kKB / 16;
        const uint32_t pp = kOdd ^ pb[s];
        if (s == 0 || n0 <= j) {  // the first group of the step: V_j and K_{j + 1}
          wait(&sy.kv_full[sv], ph, kv);
          if (j + 1 < nm) wait(&sy.kv_full[sk], kOdd ? ph ^ 1 : ph, kk);
        }
        wait(&sy.p_full[s][0], pp, p0);
        tc::fence_after_sync();
        pv_mmas(s, j, sv, steps, 0);
        const bool p1 = tc::mbar_test_wait(&sy.p_full[s][1], pp);
        tc::mma_commit(&sy.pv_done[s][0]);
        wait(&sy.p_full[s][1], pp, p1);
        tc::fence_after_sync();
        pv_mmas(s, j, sv, steps, 1);
        tc::mma_commit(&sy.pv_done[s][1]);
        const bool last = s == 1 || n1 <= j;
        if (last) tc::mma_commit(&sy.kv_empty[sv]);
        if (more) s_mmas(s, sk);
        // the next group's barriers
        const int s1 = (s == 0 && j < n1) ? 1 : (n0 > j + 1 ? 0 : 1);
        p0 = tc::mbar_test_wait(&sy.p_full[s1][0], (last ? !kOdd : kOdd) ^ (s1 ? pb[1] : pb[0]));
        if (last) {
          kv = tc::mbar_test_wait(&sy.kv_full[sv1], kOdd ? ph ^ 1 : ph);
          kk = tc::mbar_test_wait(&sy.kv_full[sk1], ph ^ 1);
        }
        if (more) tc::mma_commit(&sy.s_full[s]);
        if (last && j + 1 < nm) {  // the step's last group: K_{j + 1} has been read, by whom it had to be
          tc::mma_commit(&sy.kv_empty[sk]);
          if (j + 2 == nm) tc::mma_commit(&sy.q_empty);  // the segment's last S
        }
      };
      auto step = [&](auto odd, int j, uint32_t ph) {
        if (j < n0) slot_group(odd, integral_constant<int, 0>{}, j, ph, j + 1 < n0);
        if (j < n1) slot_group(odd, integral_constant<int, 1>{}, j, ph, j + 1 < n1);
      };
      uint32_t ph = 0;
#pragma unroll 1
      for (int sc = 0; !bad; ++sc) {
        wait(&sy.seg_full[sc & 1], (sc >> 1) & 1, false);
        if (bad) break;
        const Segment g = sy.seg[sc & 1];
        tc::mbar_arrive(&sy.seg_empty[sc & 1]);
        if (g.head < 0) break;
        n0 = g.blocks(0);
        n1 = g.blocks(1);
        nm = max(n0, n1);
        last_steps = max(0, (min(kKB, g.seq - (g.j1 - 1) * kKB) + 15) >> 4);
        p0 = kv = kk = false;
        wait(&sy.q_full, sc & 1, false);
        wait(&sy.kv_full[0], ph, false);
        tc::fence_after_sync();
        if (n0 > 0) {
          s_mmas(0, 0);
          tc::mma_commit(&sy.s_full[0]);
        }
        if (n1 > 0) {
          s_mmas(1, 0);
          tc::mma_commit(&sy.s_full[1]);
        }
        tc::mma_commit(&sy.kv_empty[0]);
        if (nm == 1) tc::mma_commit(&sy.q_empty);
#pragma unroll 1
        for (int j = 0; j < nm; j += 2, ph ^= 1) {
          step(integral_constant<int, 0>{}, j, ph);
          if (j + 1 < nm) {
            step(integral_constant<int, 1>{}, j + 1, ph);
          } else {  // the odd pair of stages, passed on
            wait(&sy.kv_full[2], ph, false);
            tc::mbar_arrive(&sy.kv_empty[2]);
            wait(&sy.kv_full[3], ph, false);
            tc::mbar_arrive(&sy.kv_empty[3]);
          }
        }
        pb[0] ^= n0 & 1;
        pb[1] ^= n1 & 1;
      }
      if (bad) *abort_flag = 1;
      // every MMA issued has completed once this arrives
      tc::mma_commit(&sy.drain);
      tc::mbar_wait(&sy.drain, 0);
    }
  } else {
    // ------------------------------------------------------------ softmax and output (warps 0-7)
    const int slot = warp >> 2, quad = warp & 3;
    const int row = quad * 32 + lane;
    const uint32_t tl = tmem + (static_cast<uint32_t>(quad * 32) << 16);  // this warp's TMEM lanes
    const uint32_t tS = tl + kSCol + slot * 128, tO = tl + kOCol + slot * 128;
    const float c2 = a.c2;
    const float2 cc = make_float2(c2, c2);
    unsigned char* stage = sO + warp * kOutStage;
    const int tok_of_row = row / a.G, head_of_row = row - tok_of_row * a.G;
    bool ok = true;
    int done = 0, turns = 0;  // blocks of this slot and turns of the ring in earlier segments
#pragma unroll 1
    for (int sc = 0;; ++sc) {
      ok = tc::mbar_wait_warp(&sy.seg_full[sc & 1], (sc >> 1) & 1);
      if (!ok) break;
      const Segment g = sy.seg[sc & 1];
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sy.seg_empty[sc & 1]);
      if (g.head < 0) break;
      const int nblk = g.blocks(slot);
      const int tok = g.tok0(slot) + tok_of_row;
      const bool live = tok_of_row < nt && tok < g.n;
      // keys this row sees (all of them for a row that is not stored), and every row of the warp
      const int limit = live ? max(0, g.seq - g.n + tok + 1) : 0x7fffffff;
      const int all_see = __reduce_min_sync(0xffffffffu, limit);
      float m = -INFINITY, l = 0.f;  // row reference (log2 units); sum of exp2(c2 s - m)
      for (int j = 0; j < nblk; ++j) {
        ok = tc::mbar_wait_warp(&sy.s_full[slot], (done + j) & 1);
        if (!ok) break;
        tc::fence_after_sync();
        const int key0 = (g.j0 + j) * kKB;
        const bool masked = key0 + kKB > all_see;
        const int seen = limit - key0;  // of the block's keys
        const int valid = g.seq - key0;
        if (quad == 0 && valid < kKB && valid > 0) {
          // the request's keys end in this block: the values behind them that share the last
          // 16-key step are whatever the page held and are multiplied by P = 0; they are
          // cleared, so that nothing there (an infinity or a NaN) reaches a row
          const int n = 2 * j + 1;
          ok = tc::mbar_wait_warp(&sy.kv_full[n % kStages], (turns + n / kStages) & 1);
          if (!ok) break;
          unsigned char* v = sKV + (n % kStages) * kTile;
          const int dead = ((valid + 15) & ~15) - valid;
          for (int e = lane; e < dead * 8 * (D / 64); e += 32) {
            const int ac = e / (dead * 8), w = e - ac * dead * 8;
            *reinterpret_cast<uint4*>(v + ac * kPanel + valid * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          tc::fence_proxy_async();
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t su[64];  // the row's logits of this half
          uint32_t pk[32];
          auto load = [&](int half) {
            tc::tmem_ld64_async(tS + half * 64, su);
            tc::tmem_wait64(su);
            if (masked) {
#pragma unroll
              for (int c = 0; c < 64; ++c) su[c] = (half * 64 + c < seen) ? su[c] : 0xff800000u;
            }
          };
          // P of the half against the reference m, and its sum
          auto exps = [&]() {
            const float nm = (m == -INFINITY) ? 0.f : -m;
            const float2 nn = make_float2(nm, nm);
            float2 acc0 = make_float2(0.f, 0.f), acc1 = acc0;
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
              const float2 z01 = tc::ffma2(make_float2(__uint_as_float(su[c]), __uint_as_float(su[c + 1])), cc, nn);
              const float2 z23 = tc::ffma2(make_float2(__uint_as_float(su[c + 2]), __uint_as_float(su[c + 3])), cc, nn);
              const float p0 = tc::ex2(z01.x), p1 = tc::ex2(z01.y), p2 = tc::ex2(z23.x), p3 = tc::ex2(z23.y);
              acc0 = tc::add2(acc0, make_float2(p0, p1));
              acc1 = tc::add2(acc1, make_float2(p2, p3));
              pk[c / 2] = tc::pack_bf16x2(p0, p1);
              pk[c / 2 + 1] = tc::pack_bf16x2(p2, p3);
            }
            return (acc0.x + acc0.y) + (acc1.x + acc1.y);
          };
          load(hf);
          float sum = exps();
          // no reference yet, a value far above it, or a NaN: take the maximum of what is left
          // of the block as the reference and start the half again (its logits are in TMEM)
          if (__any_sync(0xffffffffu, live && (m == -INFINITY || !(sum <= kRescaleSum)))) {
            float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
            for (int half = 1; half >= hf; --half) {
              load(half);
#pragma unroll
              for (int c = 0; c < 64; c += 8) {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                  t[w] = tc::max3(t[w], __uint_as_float(su[c + 2 * w]), __uint_as_float(su[c + 2 * w + 1]));
              }
            }
            const float mb = fmaxf(tc::max3(t[0], t[1], t[2]), t[3]) * c2;  // -inf when nothing is visible
            float factor = 1.f;
            if (mb > m + kRescaleTau) {
              if (m != -INFINITY) factor = tc::ex2(m - mb);
              l *= factor;
              m = mb;
            }
            if (__any_sync(0xffffffffu, factor != 1.f)) {
              // O is final up to the previous half once its P V is done
              ok = tc::mbar_wait_warp(&sy.pv_done[slot][hf ^ 1], (done + j + hf + 1) & 1);
              if (!ok) break;
              tc::fence_after_sync();
#pragma unroll 1
              for (int oc = 0; oc < D; oc += 32) {
                uint32_t ov[32];
                tc::tmem_ld32_async(tO + oc, ov);
                tc::tmem_wait(ov);
#pragma unroll
                for (int i = 0; i < 32; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * factor);
                tc::tmem_st32(tO + oc, ov);
              }
              tc::tmem_wait_st();
            }
            sum = exps();
          }
          l += sum;
          tc::tmem_st32(tS + hf * 32, pk);
          tc::tmem_wait_st();
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&sy.p_full[slot][hf]);
        }
        if (!ok) break;
      }
      if (ok && nblk > 0) ok = tc::mbar_wait_warp(&sy.pv_done[slot][1], (done + nblk - 1) & 1);
      if (!ok) break;
      done += nblk;
      turns += (2 * max(g.blocks(0), g.blocks(1)) + kStages - 1) / kStages;
      if (!g.live(slot)) continue;
      tc::fence_after_sync();
      // ---- the segment's rows out. The next segment's S may run meanwhile; its P V, which
      // overwrites O, waits for this warp's next P.
      if (g.place >= 0) {
        // a piece: columns in fours, a row a lane, so that a store takes whole lines
        const int64_t at = static_cast<int64_t>(g.place) * 2 + slot;
        __stcg(a.chunk_ml + at * kQT + row, make_float2(m, l));
        if (nblk == 0) continue;
        float4* out = reinterpret_cast<float4*>(a.chunk_o) + at * (D / 4) * kQT + row;
#pragma unroll 1
        for (int oc = 0; oc < D; oc += 32) {
          float v[32];
          tc::tmem_ld32(tO + oc, v);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            __stcg(out + (oc / 4 + i) * kQT, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
        }
        continue;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t t = static_cast<int64_t>(g.row0) + tok;
      const int head = g.head * a.G + head_of_row;
      const int64_t at = live ? t * a.o_stride + static_cast<int64_t>(head) * D : -1;
      if (live && a.lse != nullptr) a.lse[head * a.lse_stride + t] = (m + log2f(l)) * kLn2;
      // 32 columns at a time through this warp's stage, 16-byte pieces in the 64-byte swizzle; four
      // lanes then store a row's 64 bytes
#pragma unroll 1
      for (int oc = 0; oc < D; oc += 32) {
        float v[32];
        tc::tmem_ld32(tO + oc, v);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint4 w;
          // a row that sees nothing is zero whatever its accumulator holds
          auto two = [&](int c) { return l == 0.f ? 0u : tc::pack_bf16x2(v[c] * inv, v[c + 1] * inv); };
          w.x = two(8 * i);
          w.y = two(8 * i + 2);
          w.z = two(8 * i + 4);
          w.w = two(8 * i + 6);
          *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = w;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int rr = 8 * i + (lane >> 2), piece = lane & 3;
          const int64_t to = __shfl_sync(0xffffffffu, at, rr);
          const uint4 w = *reinterpret_cast<const uint4*>(stage + rr * 64 + ((piece ^ ((rr >> 1) & 3)) << 4));
          if (to >= 0) *reinterpret_cast<uint4*>(a.o + to + oc + piece * 8) = w;
        }
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, kTmemCols);
  }
  pdl_wait();  // this grid's end implies the validation kernel's, which resets the status word
  if (threadIdx.x == 0) {
    if (sy.abort) record_error(a.st, AVTP_ERR_TIMEOUT, static_cast<int32_t>(blockIdx.x));
    if (sy.bad_page >= 0) record_error(a.st, AVTP_ERR_DEVICE_INPUT, sy.bad_page);
  }
}

// ---------------------------------------------------------------- the units in pieces
// CTA (c, y): the unit whose first piece is CTA c's last, eight columns of its 256 rows, a
// row a thread. O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i with M the largest reference.
__global__ void __launch_bounds__(kChunkRows) k_cache_join(CacheAttnDev a, int d) {
  pdl_wait();
  pdl_trigger();
  const CacheChunkSplit u = a.split[blockIdx.x];
  if (u.c1 <= u.c0) return;
  const int slot = threadIdx.x / kQT, row = threadIdx.x % kQT, nt = kQT / a.G;
  const int in_tile = row / a.G, tok = (2 * u.unit + slot) * nt + in_tile;
  if (in_tile >= nt || tok >= u.n) return;
  const int pieces = u.c1 - u.c0 + 1, col4 = 2 * blockIdx.y;
  auto piece = [&](int k) { return static_cast<int64_t>(k == 0 ? u.slot0 : 2 * (u.c0 + k)) * 2 + slot; };
  float M = -INFINITY;
#pragma unroll 4
  for (int k = 0; k < pieces; ++k) M = fmaxf(M, __ldcg(a.chunk_ml + piece(k) * kQT + row).x);
  float L = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
  const float4* part = reinterpret_cast<const float4*>(a.chunk_o);
#pragma unroll 4
  for (int k = 0; k < pieces; ++k) {
    const float2 ml = __ldcg(a.chunk_ml + piece(k) * kQT + row);
    if (ml.x == -INFINITY && ml.y == 0.f) continue;  // saw nothing, or holds no block of this slot
    const float f = tc::ex2(ml.x - M);
    const float4* src = part + (piece(k) * (d / 4) + col4) * kQT + row;
    const float4 p = __ldcg(src), q = __ldcg(src + kQT);
    L = fmaf(f, ml.y, L);
    x = make_float4(fmaf(f, p.x, x.x), fmaf(f, p.y, x.y), fmaf(f, p.z, x.z), fmaf(f, p.w, x.w));
    y = make_float4(fmaf(f, q.x, y.x), fmaf(f, q.y, y.y), fmaf(f, q.z, y.z), fmaf(f, q.w, y.w));
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t t = static_cast<int64_t>(u.row0) + tok;
  const int head = u.head * a.G + (row - in_tile * a.G);
  uint4 w;
  w.x = tc::pack_bf16x2(x.x * inv, x.y * inv);
  w.y = tc::pack_bf16x2(x.z * inv, x.w * inv);
  w.z = tc::pack_bf16x2(y.x * inv, y.y * inv);
  w.w = tc::pack_bf16x2(y.z * inv, y.w * inv);
  *reinterpret_cast<uint4*>(a.o + t * a.o_stride + static_cast<int64_t>(head) * d + col4 * 4) = w;
  if (blockIdx.y == 0 && a.lse != nullptr) a.lse[head * a.lse_stride + t] = (M + log2f(L)) * kLn2;
}

template <int D>
cudaError_t launch(int grid, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttnDev& a,
                   cudaStream_t s) {
  static PerDevice attrs;
  cudaError_t e = once_per_device(attrs, [](int, int*) {
    return cudaFuncSetAttribute(k_cache_chunk<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(chunk_smem_bytes(D)));
  });
  if (e != cudaSuccess) return e;
  e = launch_kernel(k_cache_chunk<D>, dim3(grid), dim3(kThreads), chunk_smem_bytes(D), s, /*pdl=*/true, mq, mk, mv, a);
  if (e != cudaSuccess) return e;
  return launch_kernel(k_cache_join, dim3(grid, D / 8), dim3(kChunkRows), 0, s, /*pdl=*/true, a, D);
}

}  // namespace

cudaError_t launch_cache_chunk(int head_dim, int grid, const CUtensorMap& mq, const CUtensorMap& mk,
                               const CUtensorMap& mv, const CacheAttnDev& a, cudaStream_t s) {
  return head_dim == 128 ? launch<128>(grid, mq, mk, mv, a, s) : launch<64>(grid, mq, mk, mv, a, s);
}

}  // namespace avtp
