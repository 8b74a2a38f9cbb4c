// y = a b^T with both matrices in MX4, for products of many tiles: two SMs to a tile of 256 x 256.
//
// What bounds a large product here is not the tensor core but the way to it: a 128 x 256 tile on one SM
// brings 51 KB of codes and scales into shared memory for 512 cycles of multiplication, a pair
// (cta_group::2) 35 KB to each SM, because each holds half of the rows of a and the tensor cores share
// them.  Each block loads 128 rows of b (its lanes), 128 rows of a and all of a's scale bytes; the
// first of the two issues for both.
//
// One pair per two SMs walks over its tiles.  Tensor memory holds one accumulator (256 columns; the
// scale bytes of six stages take another 144), so results are first taken into registers, which frees
// it for the next tile, and written out while that one is computed.
//
// Measured at 8192 x 4096 x 9216: 93 to 96 us = 6.5 PFLOP/s, four times the measured bf16 rate (246 us with one SM to a
// tile of 128 x 256); the copies alone, with no multiplication, 89 us.  Repeated for long it runs into the power cap and
// takes 116 us = 5.3 PFLOP/s.
#include <algorithm>

#include "blocks.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

constexpr uint32_t kThreads = 384;        // warp 0 loads, warp 1 issues, warp 2 allocates; warps 4-11 take results out
constexpr uint32_t kRows = 128, kTile = 256, kStageBytes = 128;      // rows of either matrix in a block; a tile's; of a row per stage
constexpr uint32_t kMatrix = kRows * kStageBytes, kScales = 1024, kStage = 2 * kMatrix + 3 * kScales, kStages = 6;
constexpr uint32_t kScaleColumns = 24;    // tensor memory per stage: two scale atoms of the lanes and of each half of the columns
constexpr uint32_t kTmem = 512;
constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
static_assert(kTile + kStages * kScaleColumns <= kTmem && kSmem <= 227 * 1024, "does not fit an SM");

struct Params {
  void* y;
  uint64_t ldy;
  uint32_t m, n;
  uint32_t kt;                   // 128-value scale atoms along a row
  uint32_t lane_tiles, tiles;
};

__device__ uint32_t g_gave_up;   // counts up

// kind::mxf4: E2M1 x E2M1, E8M0 scales, 256 x 256.
constexpr uint32_t kInstruction = 1u << 7 | 1u << 10 | (kTile / 8) << 17 | 1u << 23 | (kTile / 128) << 27;

__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t sa, uint32_t sb, uint32_t add, uint32_t elected) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %6, 0;\n\tsetp.ne.u32 q, %7, 0;\n\t"
               "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(what), "r"(sa), "r"(sb), "r"(add), "r"(elected) : "memory");
}

template <typename G>
__global__ void __launch_bounds__(kThreads, 1)
matmul_pair_kernel(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap column_map,
                   const __grid_constant__ CUtensorMap lane_scales, const __grid_constant__ CUtensorMap column_scales,
                   const __grid_constant__ Params p) {
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_address(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * kStage);
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages, drained = ready + 8;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 2);

  const uint32_t warp = warp_index(), lane = threadIdx.x % 32, rank = cluster_rank();
  const uint32_t tile0 = blockIdx.x / 2, tile_step = gridDim.x / 2, stages = (p.kt + 1) / 2;

  if (threadIdx.x == 0) {
    prefetch_map(&lane_map);
    prefetch_map(&column_map);
    prefetch_map(&lane_scales);
    prefetch_map(&column_scales);
    for (uint32_t s = 0; s < kStages; ++s) {
      barrier_init(full + 8 * s, 1);       // the first block's counts both blocks' copies
      barrier_init(empty + 8 * s, 1);
    }
    barrier_init(ready, 1);
    barrier_init(drained, 16);             // the first block's: eight warps of each block
    barrier_init_fence();
  }
  if (warp == 2) tmem_alloc_pair(smem_address(slot), kTmem);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  cluster_arrive();
  cluster_wait();
  const uint32_t tmem = *slot;
  bool ok = true;
  admit_next_kernel();
  await_previous_kernel();

  if (warp == 0) {
    const uint32_t elected = elect(), first_full = peer_address(full, 0);
    uint32_t s = 0, parity = 1, issued = 0;
    for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
      const uint32_t n0 = tile % p.lane_tiles * kTile + rank * kRows, m0 = tile / p.lane_tiles * kTile;
      const uint32_t lane_atom = n0 / 128 * p.kt, column_atom = m0 / 128 * p.kt;
      for (uint32_t i = 0; i < stages; ++i) {
        const uint32_t at = stage0 + s * kStage, bar = first_full + 8 * s;
        if (!(ok = barrier_wait(empty + 8 * s, parity))) break;
        if (rank == 0) barrier_expect(full + 8 * s, 2 * kStage, elected);
        copy_box_pair(at, &lane_map, (int)(i * kStageBytes), (int)n0, bar, elected);
        copy_box_pair(at + kMatrix, &column_map, (int)(i * kStageBytes), (int)(m0 + rank * kRows), bar, elected);
        // atoms past a row's last one are read from elsewhere, or as zero, and not used
        copy_box_pair(at + 2 * kMatrix, &lane_scales, 0, (int)(lane_atom + 2 * i), bar, elected);
        copy_box_pair(at + 2 * kMatrix + kScales, &column_scales, 0, (int)(column_atom + 2 * i), bar, elected);
        copy_box_pair(at + 2 * kMatrix + 2 * kScales, &column_scales, 0, (int)(column_atom + p.kt + 2 * i), bar, elected);
        ++issued;
        if (++s == kStages) s = 0, parity ^= 1;
      }
    }
    if (rank == 0) await_copies(full, issued, kStages);      // for both blocks, which end together
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t elected = elect();
      uint32_t q = 0, s = 0, parity = 0;
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step, ++q) {
        if (!(ok = barrier_wait(drained, (q & 1) ^ 1))) break;
        tmem_fence_after();
        for (uint32_t i = 0; i < stages; ++i) {
          if (!(ok = barrier_wait(full + 8 * s, parity))) break;
          tmem_fence_after();
          const uint32_t at = stage0 + s * kStage, ts = tmem + kTile + s * kScaleColumns;
          const uint64_t lanes = swizzled_rows(at), columns = swizzled_rows(at + kMatrix), scales = scale_rows(at + 2 * kMatrix);
          const uint32_t atoms = min(2u, p.kt - 2 * i);
          // descriptors count in units of 16 bytes
#pragma unroll
          for (uint32_t k = 0; k < 2; ++k) {
            if (k == atoms) break;
            const uint32_t tl = ts + k * 12, tc = tl + 4;
            scales_to_tmem_pair(tl, scales + 32 * k, elected);
            scales_to_tmem_pair(tc, scales + (kScales / 16 + 32 * k), elected);
            scales_to_tmem_pair(tc + 4, scales + (2 * kScales / 16 + 32 * k), elected);
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h)   // 64 values: two scale bytes of the four
              multiply(tmem, lanes + (2 * k + h) * 2, columns + (2 * k + h) * 2, kInstruction | (2 * h) << 29 | (2 * h) << 4, tl, tc, i || k || h,
                       elected);
          }
          tensor_commit_pair(empty + 8 * s, elected);
          if (++s == kStages) s = 0, parity ^= 1;
        }
        if (ok) tensor_commit_pair(ready, elected);
      }
    }
  } else if (warp >= 4) {
    const uint32_t group = warp % 4, half = (warp - 4) / 4 * 128;   // the lanes a warp may read; its columns
    const uint32_t first_drained = peer_address(drained, 0);
    uint32_t q = 0;
    for (uint32_t tile = tile0; tile < p.tiles; tile += tile_step, ++q) {
      const uint32_t n = tile % p.lane_tiles * kTile + rank * kRows + group * 32 + lane, m = tile / p.lane_tiles * kTile + half;
      const uint32_t have = m < p.m ? min(128u, p.m - m) : 0;
      if (!(ok = barrier_wait(ready, q & 1))) break;
      tmem_fence_after();
      uint32_t r[8][16];
#pragma unroll
      for (uint32_t c = 0; c < 8; ++c) tmem_load16(tmem + (group * 32 << 16) + half + 16 * c, r[c]);
      tmem_load_wait();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive_cluster(first_drained);
      if (n < p.n) {
        G* y = static_cast<G*>(p.y) + (uint64_t)m * p.ldy + n;
        if (have == 128) {
#pragma unroll
          for (uint32_t c = 0; c < 128; ++c, y += p.ldy) put(y, __uint_as_float(r[c / 16][c % 16]));
        } else {
#pragma unroll
          for (uint32_t c = 0; c < 128; ++c, y += p.ldy)
            if (c < have) put(y, __uint_as_float(r[c / 16][c % 16]));
        }
      }
    }
  }
  if (!ok) atomicAdd(&g_gave_up, 1u);
  __syncwarp();
  tmem_fence_before();
  __syncthreads();
  cluster_arrive();      // neither block ends while the other may still use its memory
  cluster_wait();
  if (warp == 2) {
    tmem_fence_after();
    tmem_free_pair(tmem, kTmem);
  }
}

template <typename G> cudaError_t launch(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  static Device device;
  const Device::Facts* facts;
  cudaError_t e = device.prepare(matmul_pair_kernel<G>, kThreads, kSmem, 0, &facts);
  if (e != cudaSuccess) return e;
  const uint64_t nb = (a.cols + 31) / 32, kt = (nb + 3) / 4, lane_tiles = (b.rows + kTile - 1) / kTile;
  const uint64_t tiles = lane_tiles * ((a.rows + kTile - 1) / kTile);
  const uint64_t a_atoms = (a.rows + 127) / 128 * kt, b_atoms = (b.rows + 127) / 128 * kt;
  if (tiles > 0x7FFFFFFFull || a_atoms > 0x7FFFFF00ull - kt || b_atoms > 0x7FFFFF00ull - kt) return cudaErrorInvalidConfiguration;
  CUtensorMap lane_map, column_map, lane_scales, column_scales;
  e = encode_rows(&lane_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, nb * 16, b.rows, nb * 16, kRows);
  if (e == cudaSuccess) e = encode_rows(&column_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, nb * 16, a.rows, nb * 16, kRows);
  // scale bytes by whole atoms of 512, two at a time
  if (e == cudaSuccess) e = encode_plain(&lane_scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, b.scales, 128, b_atoms, 512, 128, 2);
  if (e == cudaSuccess) e = encode_plain(&column_scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, a.scales, 128, a_atoms, 512, 128, 2);
  if (e != cudaSuccess) return e;
  const Params p = {y.p, y.ld, (uint32_t)y.rows, (uint32_t)y.cols, (uint32_t)kt, (uint32_t)lane_tiles, (uint32_t)tiles};
  const unsigned pairs = (unsigned)std::min<uint64_t>(tiles, (uint64_t)facts->sms / 2);
  return launch_after(matmul_pair_kernel<G>, 2 * pairs, kThreads, kSmem, 2, stream, lane_map, column_map, lane_scales, column_scales, p);
}

}  // namespace

cudaError_t launch_mx4_matmul_pair(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  return y.type == kBF16 ? launch<__nv_bfloat16>(a, b, y, stream) : launch<float>(a, b, y, stream);
}

cudaError_t mx4_matmul_pair_gave_up(uint32_t* count, cudaStream_t stream) { return read_count(g_gave_up, count, stream); }
cudaError_t mx4_matmul_pair_count(const uint32_t** at) { return count_address(g_gave_up, at); }

}  // namespace rudra
