// y = a b^T with both matrices in MX4, on the block-scaled 4-bit tensor cores.
//
// The tensor core multiplies E2M1 codes and applies the two blocks' power-of-two scales itself, so the
// kernel only moves codes and scale bytes: TMA brings 128-byte (256-value) pieces of rows into
// swizzled shared memory, bulk copies bring the scale bytes, tcgen05.cp places those in tensor memory
// next to the accumulators.  Rows of b (a layer's outputs) are the 128 lanes of an accumulator and rows
// of a (tokens) its columns, so one shape serves a single token (16 columns) as well as large
// batches (256), and neighbouring lanes write neighbouring outputs.
//
// Few tiles: the reduction is split over the blocks of a cluster, which add their parts in rank order
// through distributed shared memory; the sum does not depend on the run.
#include <algorithm>

#include "blocks.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

constexpr int kThreads = 192;        // warp 0 loads, warp 1 issues, warps 2-5 take the results
constexpr uint32_t kStageBytes = 128;   // of a row per stage: 256 values

template <int COLS> struct Shape {
  static constexpr uint32_t kRowAtoms = COLS > 128 ? COLS / 128 : 1;     // 512-byte scale atoms per 128 values
  static constexpr uint32_t kLanes = 128 * kStageBytes;
  static constexpr uint32_t kColumns = COLS * kStageBytes;
  static constexpr uint32_t kScales = 1024 * (1 + kRowAtoms);
  static constexpr uint32_t kStage = kLanes + kColumns + kScales;
  static constexpr uint32_t kStages = COLS == 256 ? 4 : COLS == 128 ? 5 : 8;
  static constexpr uint32_t kScaleColumns = 8 * (1 + kRowAtoms);         // tensor memory per stage
  static constexpr uint32_t kUsed = COLS + kStages * kScaleColumns;
  static constexpr uint32_t kTmem = kUsed > 256 ? 512 : 256;
  static constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
  static_assert(kUsed <= 512 && kSmem <= 227 * 1024, "does not fit an SM");
  static_assert(kStages * kStage >= COLS * 512, "the parts of a split sum are kept where the stages were");
};

struct Params {
  const uint8_t* lane_scales;     // of b
  const uint8_t* column_scales;   // of a
  void* y;
  uint64_t ldy;
  uint32_t m, n;                  // rows of a, rows of b
  uint32_t kt;                    // 128-value scale atoms along a row
  uint32_t lane_tiles;
  uint32_t split;                 // blocks of a cluster that share a tile
};

__device__ uint32_t g_wait_failed;

// Instruction descriptor of kind::mxf4: E2M1 x E2M1, E8M0 scales, M = 128.
template <int COLS> __device__ constexpr uint32_t instruction() {
  return 1u << 7 | 1u << 10 | (COLS / 8) << 17 | 1u << 23 | 1u << 27;
}

__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t sa, uint32_t sb, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(what), "r"(sa), "r"(sb), "r"(add) : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float peer_float(uint32_t at, uint32_t rank) {
  uint32_t remote;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
  return v;
}

template <typename G> __device__ __forceinline__ void put(const Params& p, uint32_t m, uint32_t n, float v) {
  G* y = static_cast<G*>(p.y) + (uint64_t)m * p.ldy + n;
  if constexpr (sizeof(G) == 2) *y = __float2bfloat16_rn(v);
  else *y = v;
}

template <typename G, int COLS>
__global__ void __launch_bounds__(kThreads) matmul_kernel(const __grid_constant__ CUtensorMap lane_map,
                                                          const __grid_constant__ CUtensorMap column_map,
                                                          const __grid_constant__ Params p) {
  using S = Shape<COLS>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_address(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  const uint32_t full = smem_address(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 2 * S::kStages + 1);

  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = p.split > 1 ? cluster_rank() : 0;
  const uint32_t tile = blockIdx.x / p.split;
  const uint32_t n0 = (tile % p.lane_tiles) * 128, m0 = (tile / p.lane_tiles) * COLS;
  const uint32_t stages = (p.kt + 1) / 2;
  const uint32_t first = (uint32_t)((uint64_t)stages * rank / p.split), last = (uint32_t)((uint64_t)stages * (rank + 1) / p.split);

  if (threadIdx.x == 0) {
    prefetch_map(&lane_map);
    prefetch_map(&column_map);
    for (uint32_t s = 0; s < S::kStages; ++s) {
      barrier_init(full + 8 * s, 1);
      barrier_init(empty + 8 * s, 1);
    }
    barrier_init(done, 1);
    barrier_init_fence();
  }
  if (warp == 1) tmem_alloc(smem_address(slot), S::kTmem);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *slot;
  bool ok = true;

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t atoms_of_columns = min(S::kRowAtoms, (p.m - m0 + 127) / 128);
      uint32_t issued = 0;
      for (uint32_t i = first; i < last; ++i, ++issued) {
        const uint32_t s = issued % S::kStages, round = issued / S::kStages;
        if (!(ok = barrier_wait(empty + 8 * s, (round & 1) ^ 1))) break;
        const uint32_t at = stage0 + s * S::kStage, bar = full + 8 * s;
        const uint32_t atoms = min(2u, p.kt - 2 * i);
        barrier_expect(bar, S::kLanes + S::kColumns + atoms * 512 * (1 + atoms_of_columns));
        copy_box(at, &lane_map, (int)(i * kStageBytes), (int)n0, bar);
        copy_box(at + S::kLanes, &column_map, (int)(i * kStageBytes), (int)m0, bar);
        const uint32_t scales = at + S::kLanes + S::kColumns;
        copy_bulk(scales, p.lane_scales + ((uint64_t)(n0 / 128) * p.kt + 2 * i) * 512, atoms * 512, bar);
        for (uint32_t r = 0; r < atoms_of_columns; ++r)
          copy_bulk(scales + 1024 * (1 + r), p.column_scales + ((uint64_t)(m0 / 128 + r) * p.kt + 2 * i) * 512, atoms * 512, bar);
      }
      // given up: what is on its way lands before the block may end
      if (!ok)
        for (uint32_t k = issued > S::kStages ? issued - S::kStages : 0; k < issued; ++k)
          barrier_wait(full + 8 * (k % S::kStages), (k / S::kStages) & 1);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      for (uint32_t i = first; i < last; ++i) {
        const uint32_t c = i - first, s = c % S::kStages;
        if (!(ok = barrier_wait(full + 8 * s, (c / S::kStages) & 1))) break;
        tmem_fence_after();
        const uint32_t at = stage0 + s * S::kStage, scales = at + S::kLanes + S::kColumns;
        const uint32_t ts = tmem + COLS + s * S::kScaleColumns;
        const uint32_t atoms = min(2u, p.kt - 2 * i);
        for (uint32_t k = 0; k < atoms; ++k) {
          const uint32_t tl = ts + k * 4 * (1 + S::kRowAtoms), tc = tl + 4;
          scales_to_tmem(tl, scale_rows(scales + 512 * k));
#pragma unroll
          for (uint32_t r = 0; r < S::kRowAtoms; ++r) scales_to_tmem(tc + 4 * r, scale_rows(scales + 1024 * (1 + r) + 512 * k));
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) {   // 64 values: two scale bytes of the four
            const uint32_t off = (2 * k + h) * 32;
            multiply(tmem, swizzled_rows(at + off), swizzled_rows(at + S::kLanes + off), instruction<COLS>() | (2 * h) << 29 | (2 * h) << 4,
                     tl, tc, c || k || h);
          }
        }
        tensor_commit(empty + 8 * s);
      }
      if (ok) tensor_commit(done);
    }
  }
  __syncwarp();

  const uint32_t group = warp % 4;                       // the lanes of tensor memory a warp may read
  const uint32_t n = n0 + group * 32 + lane;
  float* part = reinterpret_cast<float*>(smem);          // [column][lane]
  if (warp >= 2) {
    ok = barrier_wait(done, 0);
    tmem_fence_after();
#pragma unroll 1
    for (uint32_t c = 0; c < COLS; c += 16) {
      uint32_t r[16];
      tmem_load16(tmem + (group * 32 << 16) + c, r);
      tmem_load_wait();
#pragma unroll
      for (uint32_t j = 0; j < 16; ++j) {
        const float v = __uint_as_float(r[j]);
        if (p.split > 1) part[(c + j) * 128 + group * 32 + lane] = v;
        else if (n < p.n && m0 + c + j < p.m) put<G>(p, m0 + c + j, n, v);
      }
    }
  }
  if (!ok) g_wait_failed = 1;
  __syncwarp();
  if (p.split > 1) {
    cluster_sync();
    const uint32_t have = min((uint32_t)COLS, p.m - m0);
    for (uint32_t e = rank * kThreads + threadIdx.x; e < have * 128; e += p.split * kThreads) {
      float v = 0.f;
      for (uint32_t r = 0; r < p.split; ++r) v += peer_float(stage0 + e * 4, r);
      if (n0 + e % 128 < p.n) put<G>(p, m0 + e / 128, n0 + e % 128, v);
    }
    cluster_sync();
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 1) {
    tmem_fence_after();
    tmem_free(tmem, S::kTmem);
  }
}

template <typename G, int COLS>
cudaError_t launch(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  using S = Shape<COLS>;
  static Device device;
  int sms;
  cudaError_t e = device.prepare(reinterpret_cast<const void*>(matmul_kernel<G, COLS>), S::kSmem, &sms);
  if (e != cudaSuccess) return e;
  Params p = {};
  const uint64_t nb = (a.cols + 31) / 32;
  p.lane_scales = static_cast<const uint8_t*>(b.scales);
  p.column_scales = static_cast<const uint8_t*>(a.scales);
  p.y = y.p;
  p.ldy = y.ld;
  p.m = (uint32_t)y.rows;
  p.n = (uint32_t)y.cols;
  p.kt = (uint32_t)((nb + 3) / 4);
  p.lane_tiles = (p.n + 127) / 128;
  const uint64_t tiles = (uint64_t)p.lane_tiles * ((p.m + COLS - 1) / COLS);
  if (tiles > 0x0FFFFFFFull) return cudaErrorInvalidConfiguration;
  const uint32_t stages = (p.kt + 1) / 2;
  p.split = 1;
  while (p.split < 8 && tiles * p.split * 2 <= (uint64_t)sms && stages >= p.split * 2) p.split *= 2;
  CUtensorMap lane_map, column_map;
  e = encode_rows(&lane_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, nb * 16, b.rows, nb * 16, 128);
  if (e == cudaSuccess) e = encode_rows(&column_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, nb * 16, a.rows, nb * 16, COLS);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute cluster;
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = p.split;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cfg.attrs = &cluster;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, matmul_kernel<G, COLS>, lane_map, column_map, p);
}

template <typename G> cudaError_t by_rows(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  if (y.rows <= 16) return launch<G, 16>(a, b, y, stream);
  if (y.rows <= 32) return launch<G, 32>(a, b, y, stream);
  if (y.rows <= 64) return launch<G, 64>(a, b, y, stream);
  if (y.rows <= 128) return launch<G, 128>(a, b, y, stream);
  return launch<G, 256>(a, b, y, stream);
}

}  // namespace

cudaError_t launch_mx4_matmul(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  if (a.cols == 0)   // a sum over nothing
    return cudaMemset2DAsync(y.p, y.ld * (y.type == kBF16 ? 2 : 4), 0, y.cols * (y.type == kBF16 ? 2 : 4), y.rows, stream);
  return y.type == kBF16 ? by_rows<__nv_bfloat16>(a, b, y, stream) : by_rows<float>(a, b, y, stream);
}

}  // namespace rudra
