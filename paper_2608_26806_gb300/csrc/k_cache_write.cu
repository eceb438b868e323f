// Keys and values of new tokens to their slots of the paged cache:
//   cache_k[slot_map[j]] = k[kept_idx[j]],  cache_v likewise,  slot s = row s % P of page s / P.
// With avtp_prune's kept_idx this is the compaction's gather, its output going to pages.
//
// A copy: 4 * Hkv * d bytes read and written a token, which bounds it for thousands of tokens; a
// step's few rows are latency. A row's 16-byte pieces are dealt to a warp, or to as many of
// its lanes as a short row has pieces (several rows a warp then), K and V alike, so that eight
// loads a lane are under way before its first store.
//
// The status word has to be cleared before anyone records in it. Up to kClusterCtas CTAs are one
// cluster, whose first CTA clears it and whose barrier, passed behind the rows, orders that: one
// launch. More run beside a kernel that clears it, and wait for that one at their end. Calls one behind
// the other, rows of 2 KiB: 64 rows 3.3 us in a cluster and 5.0 beside (the host's two launches), 128
// 3.5 and 5.0, 256 5.5 and 5.0; in a captured graph 2.3, 3.4, 5.5 against 2.7.
#include "avtp_cache.cuh"

namespace avtp {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // pieces of K and of V that a lane has under way
constexpr int kClusterCtas = 8;
constexpr int64_t kClusterRows = 2;  // rows of a group of lanes, at most, in a cluster's CTAs

struct WriteDev {
  avtp_cache_t c;
  avtp_cache_write_args_t a;
  int lanes;    // lanes of a row: a power of two, at most 32
  int pieces;   // 16-byte pieces of a row
  int head_sh;  // log2 of a head's pieces
  DevStatus* st;
};

__global__ void k_cache_write_reset(DevStatus* st) {
  pdl_wait();
  pdl_trigger();
  *st = DevStatus{0, 0, 0, 0u};
}

template <bool kCluster>
__global__ void __launch_bounds__(kThreads) k_cache_write(WriteDev w) {
  if (kCluster) pdl_wait();
  pdl_trigger();
  if (kCluster) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.st = DevStatus{0, 0, 0, 0u};
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  }
  int64_t bad = -1;
  const int sub = threadIdx.x & (w.lanes - 1);
  const int64_t groups = static_cast<int64_t>(gridDim.x) * (kThreads / w.lanes);
  const int64_t slots = w.c.n_pages * w.c.page_size;
  for (int64_t j = static_cast<int64_t>(blockIdx.x) * (kThreads / w.lanes) + threadIdx.x / w.lanes; j < w.a.n; j += groups) {
    const int64_t slot = w.a.slot_map[j];
    const int64_t row = w.a.kept_idx != nullptr ? w.a.kept_idx[j] : j;
    if (slot == -1) continue;
    if (slot < 0 || slot >= slots || row < 0 || row >= w.a.n_rows) {
      bad = j;
      continue;
    }
    const int64_t page = static_cast<uint32_t>(slot) / static_cast<uint32_t>(w.c.page_size);
    const int64_t in_page = slot - page * w.c.page_size;
    const uint4* ks = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w.a.k) + row * w.a.k_stride);
    const uint4* vs = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w.a.v) + row * w.a.v_stride);
    __nv_bfloat16* kd = static_cast<__nv_bfloat16*>(w.c.k) + page * w.c.k_page_stride + in_page * w.c.k_token_stride;
    __nv_bfloat16* vd = static_cast<__nv_bfloat16*>(w.c.v) + page * w.c.v_page_stride + in_page * w.c.v_token_stride;
    for (int c0 = sub; c0 < w.pieces; c0 += w.lanes * kUnroll) {
      uint4 kx[kUnroll], vx[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int c = c0 + u * w.lanes;
        if (c < w.pieces) {
          kx[u] = __ldcs(ks + c);
          vx[u] = __ldcs(vs + c);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int c = c0 + u * w.lanes;
        if (c < w.pieces) {
          const int64_t h = c >> w.head_sh;
          const int off = (c & ((1 << w.head_sh) - 1)) * 8;
          *reinterpret_cast<uint4*>(kd + h * w.c.k_head_stride + off) = kx[u];
          *reinterpret_cast<uint4*>(vd + h * w.c.v_head_stride + off) = vx[u];
        }
      }
    }
  }
  if (kCluster) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  else pdl_wait();
  if (bad >= 0) record_error(w.st, AVTP_ERR_DEVICE_INPUT, static_cast<int32_t>(bad));
}

}  // namespace

cudaError_t launch_cache_status(DevStatus* st, cudaStream_t s) {
  return launch_kernel(k_cache_write_reset, dim3(1), dim3(1), 0, s, /*pdl=*/true, st);
}

cudaError_t launch_cache_write(const avtp_cache_t& c, const avtp_cache_write_args_t& a, void* ws, cudaStream_t s) {
  WriteDev w{};
  w.c = c;
  w.a = a;
  w.pieces = c.n_kv_heads * c.head_dim / 8;
  w.head_sh = c.head_dim == 128 ? 4 : 3;
  w.lanes = 8;
  while (w.lanes < 32 && w.lanes < w.pieces) w.lanes *= 2;
  w.st = static_cast<DevStatus*>(ws);
  const int64_t rows = kThreads / w.lanes;
  const int64_t want = (a.n + rows - 1) / rows, most = 8 * static_cast<int64_t>(device_sm_count());
  if (want <= kClusterRows * kClusterCtas) {
    const unsigned grid = static_cast<unsigned>(want < 1 ? 1 : (want < kClusterCtas ? want : kClusterCtas));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = grid;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_cache_write<true>, w);
  }
  const cudaError_t e = launch_cache_status(w.st, s);
  if (e != cudaSuccess) return e;
  return launch_kernel(k_cache_write<false>, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(kThreads), 0, s,
                       /*pdl=*/true, w);
}

}  // namespace avtp
