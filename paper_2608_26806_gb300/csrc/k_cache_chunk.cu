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
// with the softmax, the order of MMAs and the ring of k_attn_fwd.cu: while one slot's softmax runs, the
// tensor core has the other slot's products.
// Keys and values come as TMA boxes of a page's rows, 32 boxes' places looked up in the block table
// at a time, by a warp each (one warp for both, looking up every block's, took 3000 cycles a block).
//
// Units are few (a chunk of 512 tokens, G = 4: eight a KV head) and of unequal length, so
// their key blocks, taken as one line (request, unit, head, block), are cut into equal runs, a
// CTA each. A unit that a cut falls into leaves pieces (O, reference and sum of each row) in the
// workspace, and k_cache_join puts them together in their order: results do not depend on which
// came first.
//
// What bounds it: the tensor core, 2048 cycles a block and unit at d = 128 of the 2550 that one takes (a
// slot's softmax, its last P V, its next S and the hand-overs between are one chain of that length; the
// exponentials alone would take half of it), at full load the power limit, and a unit's ends: 9000 cycles
// from its last S to the next unit's first, of which its masked block's softmax 2600 and its rows' way out.
// Short calls are launches and the way to the first S (10000 cycles), and the pieces' way through L2.
//
// Instructions are what this kernel is short of: eleven warps in four roles go through more of them than
// the SM's nearest instruction cache holds, and a first pass over code waits for it line by line. So the
// softmax has its usual path in one piece and everything else once behind it, waits and sums are calls,
// one-time code is rolled; a second copy of the loads, or waits compiled into the issuing loop, cost 10 to
// 60 %. The issuing loop is the exception: a copy a slot, whose descriptors are constants, is faster than
// one for both (32 query heads, 8 KV heads, 8192 tokens behind 2176, one call at full clock: 507 us against 533; a
// copy a slot and parity 500, but eight requests of 700 tokens behind 300 take 90 us instead of 84 then).
//
// P is rounded to bf16 for its product and O divided by the sum l of the weights before that rounding: an
// error of O of 2.3e-3 (2-norm, with some sharp queries; 1.6e-3 is O's own rounding). The sum of the
// rounded ones, which k_cache_attn divides by and which would make it about 1.9e-3, takes the softmax 9 to 20 %
// of the kernel's time here (504 -> 549 us, 491 -> 566), having no column of the accumulators left to come
// from the tensor core.
//
// Measured, calls one behind the other (32 query heads, 8 KV heads, d = 128, pages of 64 tokens): 9856 tokens 500-530
// us, 1500-1590 TFLOP/s; 8192 behind 2176 529-552 us, 1525-1590 TFLOP/s; 512 behind 9300 65-67 us, 1205-1230
// TFLOP/s. (With 30 ms between the calls, at full clock, 497 and 511 us.) At d = 64 8192 behind 2176 takes 443 us:
// 2510 cycles a block, since that chain does not depend on d, with the tensor pipe 41 % active.
//
// Warps 0-3: softmax and output of slot 0, 4-7 of slot 1 (warp w owns rows 32 (w % 4) ..). Warp 8:
// segments, queries and keys; warp 10: values. Warp 9: TMEM and the MMAs. Every wait is bounded; a
// CTA whose wait gives up records AVTP_ERR_TIMEOUT and leaves.
#include <type_traits>

#include "avtp_cache_attn.cuh"

namespace avtp {
namespace {

constexpr int kQT = 128;  // rows of a slot (MMA M, TMEM lanes)
constexpr int kKB = kChunkKeys;  // MMA N of Q K^T, K of P V
constexpr int kSlotWarps = 4;
constexpr int kKeyWarp = 2 * kSlotWarps;
constexpr int kMmaWarp = kKeyWarp + 1;
constexpr int kValueWarp = kMmaWarp + 1;
constexpr int kThreads = 32 * (kValueWarp + 1);
static_assert(kSlotWarps * 32 == kQT, "a thread a row of a slot");
constexpr int kStages = 4;      // key or value blocks in shared memory
// A unit's beginning costs about as much as this many key blocks (its queries' arrival, the first
// softmax with nothing to overlap, its rows' way out): its steps on the line are its blocks and these.
// (With three, 9856 tokens 488 us instead of 494, 512 behind 9300 63.6 instead of 62.8.)
constexpr int kUnitSteps = 2;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kSCol = 0;    // S (and P) of slot s at kSCol + 128 s
constexpr uint32_t kOCol = 256;  // O of slot s at kOCol + 128 s
// A half's sum of P above kRescaleSum moves the row's reference, if its maximum exceeds the
// reference by more than kRescaleTau (log2 units).
constexpr float kRescaleSum = 16384.f;
constexpr float kRescaleTau = 8.f;
// A row whose sum is below this has no reference yet, or one too far above its logits.
constexpr float kLeastSum = 1.f / 1024.f;
constexpr float kLn2 = 0.6931471805599453f;
static_assert(kChunkRows == 2 * kQT, "two slots a unit");

__host__ __device__ constexpr uint32_t tile_bytes(int d) { return static_cast<uint32_t>(kQT) * d * 2; }
constexpr uint32_t kPanel = kQT * 128;
constexpr uint32_t kOutStage = 2048;  // a warp's 32 rows x 32 columns of O on their way out
__host__ __device__ constexpr size_t chunk_smem_bytes(int d) {
  const size_t need = 1024 + static_cast<size_t>(2 + kStages) * tile_bytes(d) + 2 * kSlotWarps * kOutStage;
  // more than half the SM's shared memory, so that no second CTA (and its 512 TMEM columns)
  // shares an SM
  return need > 116 * 1024 ? need : 116 * 1024;
}

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
  uint64_t kv_full[kStages];
  uint64_t kv_empty[2];    // V_j and K_{j + 1} read, j even, odd (or -1: K_0)
  uint64_t s_full[2];      // S of a slot written by the MMA, and P V of the block before complete
  uint64_t p_full[2][2];   // half of a slot's P written by the softmax (and S read out)
  uint64_t half_done[2];   // P V of a block's first half complete (when someone may wait for that)
  uint64_t o_done[2];      // P V of a slot's last block in the segment complete
  uint64_t drain;
  Segment seg[2];
  CachePlan<kThreads> plan;
  CacheWindow window[2];  // of the keys' warp, of the values'
  uint32_t tmem;
  int abort, bad_page;
};
static_assert(chunk_smem_bytes(128) + sizeof(ChunkSync) <= 227 * 1024, "shared memory of one CTA");

// sum_{i < n} floor((a i + b) / m), by Euclid's steps on (a, m); a n + b is below 2^32, the sum below 2^31.
__host__ __device__ inline uint32_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  uint32_t sum = 0;
  while (true) {
    sum += static_cast<uint32_t>(static_cast<uint64_t>(n) * (n - 1) / 2 * (a / m)) + n * (b / m);
    a %= m;
    b %= m;
    const uint32_t top = a * n + b;
    if (top < m) return sum;
    n = top / m;
    b = top % m;
    const uint32_t t = m;
    m = a;
    a = t;
  }
}

// Key blocks of a request's unit: those of its last token, one for a token that sees nothing.
__device__ __forceinline__ int unit_blocks(const CacheRequest& q, int nt, int u) {
  return max(1, (q.seq - q.n + static_cast<int>(min((u + 1) * static_cast<int64_t>(2 * nt), static_cast<int64_t>(q.n))) +
                 kKB - 1) / kKB);
}
__device__ __forceinline__ int units_of(const CacheAttnDev& a, const CacheRequest& q, int nt) {
  return q.rows(a) > a.few_rows ? (q.n + 2 * nt - 1) / (2 * nt) : 0;
}

// Behind the queries before (qn of them), a segment's, by one thread of the calling warp; false if the
// wait gave up.
template <int D>
__device__ __noinline__ bool load_queries(const CUtensorMap* map, unsigned char* sQ, const Segment& g, int G, ChunkSync& sy,
                                          int qn) {
  bool ok = true;
  if (tc::elect_one()) {
    ok = qn == 0 || cache_wait(&sy.q_empty, (qn - 1) & 1);
    if (ok) {
      const int nq = g.live(1) ? 2 : 1;
      tc::mbar_arrive_expect_tx(&sy.q_full, nq * (D / 64) * g.nt * G * 128);
#pragma unroll 1
      for (int i = 0; i < nq * (D / 64); ++i)
        tc::tma_load_3d(sQ + i * kPanel, map, i % (D / 64) * 64, g.head * G, g.row0 + g.tok0(i / (D / 64)), &sy.q_full);
    }
  }
  return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ int steps_of(const CacheAttnDev& a, int blocks) {
  return kUnitSteps + ((blocks + (1 << a.step_shift) - 1) >> a.step_shift);
}

// Steps of the first u units of a request's head, the last of all not among them, in closed form: unit i's
// last token sees x = past + rows (i + 1) keys, for which it has kUnitSteps + max(1, ceil(x / (128 * 2^step_shift))) of them. For
// requests of more than kNearUnits units: 128 of them, added up one by one and passed one by one, took up to
// 24000 cycles before a CTA's first product and take 9000 so; eight of them 2500 and 5300.
constexpr int kNearUnits = 32;
static __device__ __noinline__ int steps_before(int past, int rows, int step_shift, int u) {
  const int blind = past >= 0 ? 0 : min(u, -past / rows);  // units that see nothing
  const uint32_t keys = static_cast<uint32_t>(kKB) << step_shift;
  int sum = kUnitSteps * u + blind;
  if (u > blind) sum += floor_sum(u - blind, keys, rows, past + (blind + 1) * rows + keys - 1);
  return sum;
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
    for (int s = 0; s < kStages; ++s) tc::mbar_init(&sy.kv_full[s], 1);
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&sy.kv_empty[s], 1);
      tc::mbar_init(&sy.half_done[s], 1);
      tc::mbar_init(&sy.o_done[s], 1);
      tc::mbar_init(&sy.seg_full[s], 1);
      tc::mbar_init(&sy.seg_empty[s], 2 * kSlotWarps + 2);
      tc::mbar_init(&sy.s_full[s], 1);
      for (int h = 0; h < 2; ++h) tc::mbar_init(&sy.p_full[s][h], kSlotWarps);
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
  CacheRequest mine{};  // a lane's request of a call of few: on its way while the barriers are made
  bool mine_ok = true;
  if (warp == kKeyWarp && lane < a.R) mine_ok = mine.load(a, lane);
  // the rows behind a slot's nt * G, which no box writes: zeros
  const int spare = kQT - nt * a.G;
  for (int i = threadIdx.x; i < 2 * (D / 64) * spare * 8; i += kThreads) {
    const int panel = i / (spare * 8), e = i - panel * spare * 8;
    *reinterpret_cast<uint4*>(sQ + panel * kPanel + nt * a.G * 128 + e * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
  tc::fence_proxy_async();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = sy.tmem;
  volatile int* abort_flag = &sy.abort;

  auto steps = [&](const CacheRequest& q, int& most) {
    const int U = units_of(a, q, nt);
    if (U == 0) return 0;
    int sum = steps_of(a, unit_blocks(q, nt, U - 1));  // the last unit may be short
    most = max(most, sum);
    if (U > kNearUnits) {
      sum += steps_before(q.seq - q.n, 2 * nt, a.step_shift, U - 1);
    } else {
#pragma unroll 1
      for (int u = 0; u < U - 1; ++u) sum += steps_of(a, unit_blocks(q, nt, u));
    }
    return sum * a.Hkv;
  };
  if (a.R > kNearRequests) sy.plan.form(a, steps);

  // The ring. K_j and V_j of a segment lie in stages 2 (j % 2) and 2 (j % 2) + 1. The MMA thread
  // releases V_j and K_{j + 1} together, behind the last product with either: kv_empty[j % 2], once
  // a step but the last, and kv_empty[1] once before, for K_0. The last values are released with the
  // segment's O.
  if (warp == kKeyWarp || warp == kValueWarp) {
    // ------------------------------------------------------------ segments, queries, keys; values
    const int kv = warp == kKeyWarp ? 0 : 1;
    const CUtensorMap* map = kv ? &mapV : &mapK;
    const int per_block = kKB / a.box;
    int fired0 = 0, fired1 = 0;  // completions of kv_empty[0] and [1] in the segments before
    int outs0 = 0, outs1 = 0;    // of o_done[0] and [1]
    int loads0 = 0, loads1 = 0;  // into the even and the odd blocks' stage
    int qn = 0;                  // queries loaded
    bool ok = true;
    int t = 0, t1 = 0, pre = 0;  // steps: next, the run's end, before unit u of request r
    int r = 0, u = 0;
    CacheRuns runs;
    CacheLine line;
    CacheChunkSplit split{};
    split.c1 = -1;
    if (kv == 0) {
      line = CacheLine(a, sy.plan, mine, mine_ok, steps);
      runs = CacheRuns(line.total, line.most, kUnitSteps + 1, cache_ctas(a, line.weights, false));
      t = runs.begin(blockIdx.x);
      t1 = runs.begin(blockIdx.x + 1);
      if (t < t1) {
        r = line.find(a, sy.plan, t, &pre);
        // a request of many units: its last one that begins at or before step t, 32 tries at a time (the
        // units of few, and the requests behind r, are passed one by one below)
        const CacheRequest q = line.request(a, mine, r);
        const int past = q.seq - q.n, U = units_of(a, q, nt);
        if (U > kNearUnits) {
#pragma unroll 1
          for (int n = U; n > 1;) {  // it is among units u .. u + n - 1
            const int each = (n + 31) / 32, at = lane * each;
            const bool before = at < n && pre + steps_before(past, 2 * nt, a.step_shift, u + at) * a.Hkv <= t;
            const int on = (__popc(__ballot_sync(0xffffffffu, before)) - 1) * each;
            u += on;
            n = min(each, n - on);
          }
          pre += steps_before(past, 2 * nt, a.step_shift, u) * a.Hkv;
        }
      }
    }
#pragma unroll 1
    for (int sc = 0;; ++sc) {
      Segment g{};
      if (kv == 0) {
        g.head = -1;
        int end = t;
        if (t < t1) {
          CacheRequest q;
          int nb = 0, len = 0;  // key blocks and steps of the unit
#pragma unroll 1
          for (;; ++r, u = 0) {
            q = line.request(a, mine, r);
            const int U = units_of(a, q, nt);
#pragma unroll 1
            for (; u < U; ++u) {
              nb = unit_blocks(q, nt, u);
              len = steps_of(a, nb);
              if (t < pre + len * a.Hkv) break;
              pre += len * a.Hkv;
            }
            if (u < U) break;
          }
          const int head = static_cast<int>(static_cast<uint32_t>(t - pre) / static_cast<uint32_t>(len));
          const int s = pre + head * len;  // the unit's first step
          end = min(t1, s + len);
          // a run that ends in a unit's first steps leaves its blocks to the next
          g.head = end > s + kUnitSteps ? head : -1;
          g.row0 = q.row0;
          g.n = q.n;
          g.seq = q.seq;
          g.nt = nt;
          g.unit = u;
          g.req = r;
          g.j0 = max(0, t - s - kUnitSteps) << a.step_shift;
          g.j1 = min(nb, (end - s - kUnitSteps) << a.step_shift);
          const int me = static_cast<int>(blockIdx.x);
          const int c0 = g.j0 == 0 ? me : runs.run(s + kUnitSteps);
          const int c1 = end == s + len ? me : runs.run(s + len - 1);
          g.place = c0 == c1 ? -1 : piece_place(me, g.j0 == 0);
          if (g.head >= 0 && c0 < c1 && c0 == me) split = CacheChunkSplit{g.row0, g.n, g.head, g.unit, c0, c1};
        }
        t = end;
        if (sc >= 2) ok = cache_wait_warp(&sy.seg_empty[sc & 1], ((sc >> 1) - 1) & 1);
        if (!ok) break;
        if (lane == 0) {
          sy.seg[sc & 1] = g;
          tc::mbar_arrive(&sy.seg_full[sc & 1]);
        }
        __syncwarp();
      } else {
        ok = cache_wait_warp(&sy.seg_full[sc & 1], (sc >> 1) & 1);
        if (!ok) break;
        g = sy.seg[sc & 1];
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sy.seg_empty[sc & 1]);
      }
      if (g.head < 0) break;
      const int32_t* row = a.table + g.req * a.table_stride;
      const int blocks = g.j1 - g.j0;
      // the first queries wait for nothing; later ones come behind the segment's first keys, which
      // need not wait for the last product with the queries before
      if (kv == 0 && sc == 0) {
        ok = load_queries<D>(&mapQ, sQ, sy.seg[sc & 1], a.G, sy, sc);
        qn = ok ? 1 : 0;
      }
#pragma unroll 1
      for (int j = 0; j < blocks && !cache_raised(abort_flag); ++j) {
        const int i0 = (g.j0 + j) * per_block, sb = 2 * (j & 1) + kv;
        if (j == 0 || (i0 & 31) == 0)
          if (sy.window[kv].load(a, row, g.seq, i0 & ~31)) sy.bad_page = g.req;
        const int keys = min(kKB, g.seq - (g.j0 + j) * kKB);  // none: an empty cache
        const int boxes = keys <= 0 ? 0 : (keys + a.box - 1) / a.box;
        // the stage's last occupant, block j - 2: V_{j - 2} is released in step j - 2, K_{j - 2} in
        // step j - 3; before the first two keys, the last release of the segment before, before the
        // first two values, its O
        const int bar = (j & 1) ^ (kv ^ 1);
        const int which = (bar ? fired1 : fired0) + (j < 2 ? -1 : (j >> 1) - 1 + (kv & bar));
        if (tc::elect_one()) {
          bool fine = true;
          if (kv == 0 || j >= 2) {
            fine = which < 0 || cache_wait(&sy.kv_empty[bar], which & 1);
          } else if (j == 0) {
            fine = (outs0 == 0 || cache_wait(&sy.o_done[0], (outs0 - 1) & 1)) &&
                   (outs1 == 0 || cache_wait(&sy.o_done[1], (outs1 - 1) & 1));
          }
          if (!fine) {
            *abort_flag = 1;
          } else {
            tc::mbar_arrive_expect_tx(&sy.kv_full[sb], boxes * a.box * D * 2);
            unsigned char* dst = sKV + sb * kTile;
#pragma unroll 1
            for (int b = 0; b < boxes; ++b, dst += a.box * 128) {
              const int2 at = sy.window[kv].at[(i0 + b) & 31];
#pragma unroll
              for (int p = 0; p < D / 64; ++p)
                tma_load_4d(dst + p * kPanel, map, p * 64, at.y, g.head, at.x, &sy.kv_full[sb]);
            }
          }
        }
        __syncwarp();
        if (j & 1) ++loads1; else ++loads0;
        if (kv == 0 && j == 0 && sc > 0) {
          ok = load_queries<D>(&mapQ, sQ, sy.seg[sc & 1], a.G, sy, sc);
          if (ok) qn = sc + 1;
        }
      }
      ok = ok && !cache_raised(abort_flag);
      if (!ok) break;
      fired0 += blocks >> 1;
      fired1 += 1 + ((blocks - 1) >> 1);
      outs0 += g.blocks(0) > 0 ? 1 : 0;
      outs1 += g.blocks(1) > 0 ? 1 : 0;
    }
    if (lane == 0) {
      if (!ok) *abort_flag = 1;
      if (kv == 0) a.split[blockIdx.x] = split;
    }
    // let the copies in flight land before the CTA may exit
    if (kv == 0 && qn > 0) cache_wait_warp(&sy.q_full, (qn - 1) & 1);
    if (loads0 > 0) cache_wait_warp(&sy.kv_full[kv], (loads0 - 1) & 1);
    if (loads1 > 0) cache_wait_warp(&sy.kv_full[2 + kv], (loads1 - 1) & 1);
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
        if (!seen && !bad) bad = !cache_wait(bar, parity);
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
        const uint64_t dv = tc::desc_mn_sw128(kv_base + stage * kTile, kPanel) + half * (4 * 2048 / 16);
        const uint32_t tP = tmem + kSCol + s * 128 + half * 32, tO = tmem + kOCol + s * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (half * 4 + k < steps)
            tc::mma_bf16_ts(tO, tP + k * 8, dv + k * (2048 / 16), idO, (j > 0 || half > 0 || k > 0) ? 1u : 0u);
      };
      uint32_t ph0 = 0, ph1 = 0;  // phases of stages 0 and 1, and of 2 and 3, at the segment's block 0
      uint32_t pb0 = 0, pb1 = 0;  // phase of each slot's barriers at the segment's block 0
#pragma unroll 1
      for (int sc = 0; !bad; ++sc) {
        wait(&sy.seg_full[sc & 1], (sc >> 1) & 1, false);
        if (bad) break;
        const Segment g = sy.seg[sc & 1];
        tc::mbar_arrive(&sy.seg_empty[sc & 1]);
        if (g.head < 0) break;
        const int n0 = g.blocks(0), n1 = g.blocks(1), nm = max(n0, n1);
        const int last_steps = max(0, (min(kKB, g.seq - (g.j1 - 1) * kKB) + 15) >> 4);
        wait(&sy.q_full, sc & 1, false);
        wait(&sy.kv_full[0], ph0, false);
        tc::fence_after_sync();
        bool p0 = false, kv = false, kk = false;
        // S_0 of both slots. Few commits, here and below: the thread stands still for most of one, longer
        // than the two MMAs that the tensor core queues. p0, kv, kk: whether the first half of the next P and
        // the next V and K were seen complete.
#pragma unroll 1
        for (int s = n0 > 0 ? 0 : 1; s < (n1 > 0 ? 2 : 1); ++s) {
          s_mmas(s, 0);
          tc::mma_commit(&sy.s_full[s]);
        }
        tc::mma_commit(&sy.kv_empty[1]);
        if (nm == 1) tc::mma_commit(&sy.q_empty);
        auto group = [&](auto odd_, auto slot_, int j) {
          const int odd = odd_, s = slot_;
          const uint32_t turn = static_cast<uint32_t>(j) >> 1;  // of V_j's stage in this segment
          const uint32_t pv = (odd ? ph1 : ph0) ^ (turn & 1), pk = (odd ? ph0 : ph1) ^ ((turn + odd) & 1);
          const int steps = j == nm - 1 ? last_steps : kKB / 16;
          const bool keys = j + 1 < nm;
          const bool more = j + 1 < (s ? n1 : n0), last = s == 1 || n1 <= j;
          const uint32_t pp = odd ^ (s ? pb1 : pb0);
          if (s == 0 || n0 <= j) {  // the first group of the step: V_j and K_{j + 1}
            wait(&sy.kv_full[2 * odd + 1], pv, kv);
            if (keys) wait(&sy.kv_full[2 - 2 * odd], pk, kk);
          }
          wait(&sy.p_full[s][0], pp, p0);
          tc::fence_after_sync();
          pv_mmas(s, j, 2 * odd + 1, steps, 0);
          // a softmax that is still at the second half may have to wait for the first half's P V;
          // where it is through, a plain arrival keeps the barrier's phase
          if (tc::mbar_test_wait(&sy.p_full[s][1], pp)) {
            tc::mbar_arrive(&sy.half_done[s]);
          } else {
            tc::mma_commit(&sy.half_done[s]);
            wait(&sy.p_full[s][1], pp, false);
          }
          tc::fence_after_sync();
          pv_mmas(s, j, 2 * odd + 1, steps, 1);
          if (more) s_mmas(s, 2 - 2 * odd);
          // the next group's barriers
          const int s1 = (s == 0 && j < n1) ? 1 : (n0 > j + 1 ? 0 : 1);
          p0 = tc::mbar_test_wait(&sy.p_full[s1][0], (last ? odd ^ 1 : odd) ^ (s1 ? pb1 : pb0));
          if (last) {  // V_{j + 1} and K_{j + 2}, in the other two stages
            kv = tc::mbar_test_wait(&sy.kv_full[3 - 2 * odd], pk);
            kk = tc::mbar_test_wait(&sy.kv_full[2 * odd], pv ^ 1);
          }
          if (more) tc::mma_commit(&sy.s_full[s]);
          else tc::mma_commit(&sy.o_done[s]);
          if (last && keys) {
            tc::mma_commit(&sy.kv_empty[odd]);
            if (j + 2 == nm) tc::mma_commit(&sy.q_empty);  // the segment's last S
          }
        };
#pragma unroll 1
        for (int j = 0; j < nm; ++j) {
          if (j < n0) group(j & 1, std::integral_constant<int, 0>{}, j);
          if (j < n1) group(j & 1, std::integral_constant<int, 1>{}, j);
        }
        ph0 ^= ((nm + 1) >> 1) & 1;
        ph1 ^= (nm >> 1) & 1;
        pb0 ^= n0 & 1;
        pb1 ^= n1 & 1;
      }
      if (bad) *abort_flag = 1;
      // every MMA issued has completed once this arrives
      tc::mma_commit(&sy.drain);
      cache_wait(&sy.drain, 0);
    }
  } else {
    // ------------------------------------------------------------ softmax and output (warps 0-7)
    const int slot = warp >> 2, quad = warp & 3;
    const int row = quad * 32 + lane;
    const uint32_t tl = tmem + (static_cast<uint32_t>(quad * 32) << 16);  // this warp's TMEM lanes
    const uint32_t tS = tl + kSCol + slot * 128, tO = tl + kOCol + slot * 128;
    const float c2 = a.c2;
    const float2 cc = make_float2(c2, c2);
    const int tok_of_row = row / a.G, head_of_row = row - tok_of_row * a.G;
    bool ok = true;
    int done = 0, outs = 0;         // blocks of this slot, and segments that held some, so far
    int loads0 = 0, loads1 = 0;     // blocks in the even and the odd stages in earlier segments
#pragma unroll 1
    for (int sc = 0;; ++sc) {
      ok = cache_wait_warp(&sy.seg_full[sc & 1], (sc >> 1) & 1);
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
      // row reference (log2 units), sum of exp2(c2 s - m). The reference begins as the maximum of the
      // first half, which is in registers anyway (the whole block's, with the half's exponentials
      // taken twice, cost 1400 cycles a segment; beginning at 0, sharp queries moved it too often).
      float m = 0.f, l = 0.f;
      for (int j = 0; j < nblk; ++j) {
        ok = cache_wait_warp(&sy.s_full[slot], (done + j) & 1);
        if (!ok) break;
        tc::fence_after_sync();
        const int key0 = (g.j0 + j) * kKB;
        const bool masked = key0 + kKB > all_see;
        const int seen = limit - key0;  // of the block's keys
        const int valid = g.seq - key0;
        if (masked && quad == 0 && valid < kKB && valid > 0) {
          // the request's keys end in this block: the values behind them that share the last
          // 16-key step are whatever the page held and are multiplied by P = 0; they are
          // cleared, so that nothing there (an infinity or a NaN) reaches a row. (The stage's values
          // before these have been multiplied, or S_j would not be here: the phase waited for is the next.)
          const int sb = 2 * (j & 1) + 1;
          ok = cache_wait_warp(&sy.kv_full[sb], ((j & 1 ? loads1 : loads0) + (j >> 1)) & 1);
          if (!ok) break;
          unsigned char* v = sKV + sb * kTile;
          const int dead = ((valid + 15) & ~15) - valid;
          for (int e = lane; e < dead * 8 * (D / 64); e += 32) {
            const int ac = e / (dead * 8), w = e - ac * dead * 8;
            *reinterpret_cast<uint4*>(v + ac * kPanel + valid * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          tc::fence_proxy_async();
        }
        uint32_t su[64];  // the row's logits of a half
        uint32_t pk[32];  // its P
        // P of the half in su against the reference m; its sum
        auto exps = [&]() {
          const float2 nn = make_float2(-m, -m);
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
        // values far above the reference or, as yet, all far below it, or a NaN
        auto off = [&](float sum) { return __any_sync(0xffffffffu, live && (!(sum <= kRescaleSum) || l + sum < kLeastSum)); };
        auto hand_over = [&](int hf, float sum) {
          l += sum;
          tc::tmem_st32(tS + hf * 32, pk);
          tc::tmem_wait_st();
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&sy.p_full[slot][hf]);
        };
        // Nearly every block: no mask, and a reference that stays. Its instructions lie one behind the
        // other; what the others need comes behind, once.
        int hf = 0;
        if (!masked && j > 0) {
          tc::tmem_ld64_async(tS, su);
          tc::tmem_wait64(su);
          float sum = exps();
          if (!off(sum)) {
            hand_over(0, sum);
            hf = 1;
            tc::tmem_ld64_async(tS + 64, su);
            tc::tmem_wait64(su);
            sum = exps();
            if (!off(sum)) {
              hand_over(1, sum);
              hf = 2;
            }
          }
        }
#pragma unroll 1
        for (; hf < 2; ++hf) {
          float sum, mb = -INFINITY;
          // Once through the loop but for a reference to be found: the half's maximum as a segment's
          // first one (kFirst), the maximum of what is left of the block where a sum asks for it (kMove).
          enum { kPlain, kFirst, kMove };
          int mode = hf == 0 && j == 0 ? kFirst : kPlain;
          int at = hf;  // the half in su
#pragma unroll 1
          for (;;) {
            tc::tmem_ld64_async(tS + at * 64, su);
            tc::tmem_wait64(su);
            if (masked) {
              const int left = seen - at * 64;
#pragma unroll
              for (int c = 0; c < 64; ++c) su[c] = c < left ? su[c] : 0xff800000u;
            }
            if (mode != kPlain) {
              float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
              for (int c = 0; c < 64; c += 8) {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                  t[w] = tc::max3(t[w], __uint_as_float(su[c + 2 * w]), __uint_as_float(su[c + 2 * w + 1]));
              }
              mb = fmaxf(mb, fmaxf(tc::max3(t[0], t[1], t[2]), t[3]) * c2);  // stays -inf when nothing is visible
              if (mode == kFirst) {
                m = mb == -INFINITY ? 0.f : mb;
              } else if (at > hf) {
                at = hf;
                continue;
              } else {
                float factor = 1.f;
                // A reference moves down before a row's first term alone, so nothing was lost to underflow
                // (l = 0, and O is zero or not yet written); behind that l stays above kLeastSum, but for
                // a half whose block's maximum, then the reference, is in the other half.
                if (mb > m + kRescaleTau || (l < kLeastSum && mb != -INFINITY)) {
                  factor = l > 0.f ? tc::ex2(m - mb) : 1.f;
                  l *= factor;
                  m = mb;
                }
                if (__any_sync(0xffffffffu, factor != 1.f)) {
                  if (hf == 1) ok = cache_wait_warp(&sy.half_done[slot], (done + j) & 1);
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
              }
            }
            sum = exps();
            if (mode == kMove || !off(sum)) break;
            mode = kMove;
            mb = -INFINITY;
            at = 1;
          }
          if (!ok) break;
          hand_over(hf, sum);
        }
        if (!ok) break;
      }
      if (ok && nblk > 0) ok = cache_wait_warp(&sy.o_done[slot], outs & 1);
      if (!ok) break;
      done += nblk;
      outs += nblk > 0 ? 1 : 0;
      loads0 += (g.j1 - g.j0 + 1) >> 1;
      loads1 += (g.j1 - g.j0) >> 1;
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
      const float inv = 1.f / l;
      const uint32_t sees = l == 0.f ? 0u : 0xffffffffu;  // a row that sees nothing is zero whatever its accumulator holds
      const int64_t t = static_cast<int64_t>(g.row0) + tok;
      const int head = g.head * a.G + head_of_row;
      if (live && a.lse != nullptr) a.lse[head * a.lse_stride + t] = (m + log2f(l)) * kLn2;
      // 32 columns at a time through shared memory (16-byte pieces, swizzled), so that four lanes store 64
      // bytes of a row: a lane a row, 16 bytes at a time, each store takes 32 turns of the memory pipe
      unsigned char* stage = sO + warp * kOutStage;
      const int piece = lane & 3;
      const unsigned long long dst =
          live ? reinterpret_cast<unsigned long long>(a.o + t * a.o_stride + static_cast<int64_t>(head) * D) : 0ull;
      unsigned long long to[4];  // rows lane / 4, + 8, ...
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        to[i] = __shfl_sync(0xffffffffu, dst, i * 8 + (lane >> 2));
        if (to[i] != 0) to[i] += piece * 16;
      }
#pragma unroll 1
      for (int oc = 0; oc < D; oc += 32) {
        float v[32];
        tc::tmem_ld32(tO + oc, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          auto two = [&](int c) { return tc::pack_bf16x2(v[8 * i + c] * inv, v[8 * i + c + 1] * inv) & sees; };
          *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) =
              make_uint4(two(0), two(2), two(4), two(6));
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = i * 8 + (lane >> 2);
          const uint4 x = *reinterpret_cast<const uint4*>(stage + r * 64 + ((piece ^ ((r >> 1) & 3)) << 4));
          if (to[i] != 0) *reinterpret_cast<uint4*>(to[i] + oc * 2) = x;
        }
        __syncwarp();
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
  // only now: a grid waiting to start beside this one costs it 3 %
  pdl_trigger();
  pdl_wait();  // this grid's end implies the validation kernel's, which resets the status word
  if (threadIdx.x == 0) {
    if (sy.abort) record_error(a.st, AVTP_ERR_TIMEOUT, static_cast<int32_t>(blockIdx.x));
    if (sy.bad_page >= 0) record_error(a.st, AVTP_ERR_DEVICE_INPUT, sy.bad_page);
  }
}

// ---------------------------------------------------------------- the units in pieces
// CTA (c, y): the unit that goes on behind run c and began in it, 16 columns of its 256 rows, a row a
// thread. O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i with M the largest reference of the
// pieces that saw a key. The weights are formed first, all their loads at once, so that four
// pieces' columns are under way together.
__global__ void __launch_bounds__(kChunkRows) k_cache_join(CacheAttnDev a, int d) {
  __shared__ float s_weight[kCacheMaxPieces][kChunkRows];
  pdl_wait();
  pdl_trigger();
  const CacheChunkSplit u = a.split[blockIdx.x];
  if (u.c1 <= u.c0) return;
  const int slot = threadIdx.x / kQT, row = threadIdx.x % kQT, nt = kQT / a.G;
  const int in_tile = row / a.G, tok = (2 * u.unit + slot) * nt + in_tile;
  if (in_tile >= nt || tok >= u.n) return;
  const int pieces = min(u.c1 - u.c0 + 1, kCacheMaxPieces), col4 = 4 * blockIdx.y;
  auto piece = [&](int k) { return static_cast<int64_t>(piece_place(u.c0 + k, k == 0)) * 2 + slot; };
  float M = -INFINITY, L = 0.f;
  for (int k0 = 0; k0 < pieces; k0 += 8) {
    float2 ml[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      ml[k] = k0 + k < pieces ? __ldcg(a.chunk_ml + piece(k0 + k) * kQT + row) : make_float2(0.f, 0.f);
    float mn = M;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (ml[k].y != 0.f) mn = fmaxf(mn, ml[k].x);  // a sum of zero: it saw no key, or holds no block of this slot
    const float old = M == -INFINITY ? 0.f : tc::ex2(M - mn);
    if (old != 1.f)
      for (int k = 0; k < k0; ++k) s_weight[k][threadIdx.x] *= old;
    L *= old;
    M = mn;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float f = ml[k].y == 0.f ? 0.f : tc::ex2(ml[k].x - M);
      if (k0 + k < pieces) s_weight[k0 + k][threadIdx.x] = f;
      L = fmaf(f, ml[k].y, L);
    }
  }
  float4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < pieces; k0 += 4) {
    float4 p[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4* src =
          reinterpret_cast<const float4*>(a.chunk_o) + (piece(min(k0 + k, pieces - 1)) * (d / 4) + col4) * kQT + row;
#pragma unroll
      for (int i = 0; i < 4; ++i) p[k][i] = __ldcg(src + i * kQT);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float f = k0 + k < pieces ? s_weight[k0 + k][threadIdx.x] : 0.f;
      if (f == 0.f) continue;  // its O may never have been written
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = make_float4(fmaf(f, p[k][i].x, v[i].x), fmaf(f, p[k][i].y, v[i].y), fmaf(f, p[k][i].z, v[i].z),
                           fmaf(f, p[k][i].w, v[i].w));
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t t = static_cast<int64_t>(u.row0) + tok;
  const int head = u.head * a.G + (row - in_tile * a.G);
  uint4* out = reinterpret_cast<uint4*>(a.o + t * a.o_stride + static_cast<int64_t>(head) * d + col4 * 4);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint4 w;
    w.x = tc::pack_bf16x2(v[2 * i].x * inv, v[2 * i].y * inv);
    w.y = tc::pack_bf16x2(v[2 * i].z * inv, v[2 * i].w * inv);
    w.z = tc::pack_bf16x2(v[2 * i + 1].x * inv, v[2 * i + 1].y * inv);
    w.w = tc::pack_bf16x2(v[2 * i + 1].z * inv, v[2 * i + 1].w * inv);
    out[i] = w;
  }
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
  return launch_kernel(k_cache_join, dim3(grid, D / 16), dim3(kChunkRows), 0, s, /*pdl=*/true, a, D);
}

}  // namespace

cudaError_t launch_cache_chunk(int head_dim, int grid, const CUtensorMap& mq, const CUtensorMap& mk,
                               const CUtensorMap& mv, const CacheAttnDev& a, cudaStream_t s) {
  return head_dim == 128 ? launch<128>(grid, mq, mk, mv, a, s) : launch<64>(grid, mq, mk, mv, a, s);
}

}  // namespace avtp
