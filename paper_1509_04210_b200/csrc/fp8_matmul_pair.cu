// y = a b^T with both matrices in FP8 (E4M3, a scale for each 128 values of a row), for products of many tiles: two SMs
// to a tile of 256 x 256.
//
// The tensor core takes a scale byte for each 32 values of a row; four instructions along a row are given the same one, so
// that a block of 128 needs one byte in memory and the sum never leaves the accumulator for its scales.
//
// A pair (cta_group::2) brings 34 KB to each SM for 512 cycles of multiplication, because each holds half of the rows of a
// and the tensor cores share them.  Each block loads 128 rows of b (its lanes), 128 rows of a and all of a's scale bytes; the
// first of the two issues for both.
//
// One pair per two SMs walks over its tiles.  Tensor memory holds one accumulator (256 columns; the
// scale bytes another 36), so results are first taken into registers, which frees
// it for the next tile, and written out while that one is computed.
//
// Measured at 8192 x 4096 x 9216: 201 us = 3.07 PFLOP/s, 1.84 times the measured bf16 rate; repeated for long it runs into the power
// cap and takes 231 us = 2.67 PFLOP/s, 1.90 times the sustained bf16 rate.  A stage takes 0.30 us on a few SMs (0.27 of it
// multiplication) and 0.36 on all.  4096 x 4096 x 9216: 109 us, with 3.5 rounds of tiles taking four.  Sums that are gathered in
// registers cost 2048 x 4096 x 131072 3 %: 797 us, and 773 in one sum.
#include <algorithm>

#include "fp8.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

constexpr uint32_t kThreads = 384;        // warp 0 loads, warp 1 issues, warp 2 allocates; warps 4-11 take results out
constexpr uint32_t kRows = 128, kTile = 256, kStageBytes = 128;      // rows of either matrix in a block; a tile's; of a row per stage
constexpr uint32_t kMatrix = kRows * kStageBytes, kScales = 512, kBytes = 2 * kMatrix + 3 * kScales, kStages = 6;
constexpr uint32_t kStage = (kBytes + 1023) / 1024 * 1024;   // the swizzle repeats every 1024 bytes
// An atom of scale bytes serves four stages, and is copied to tensor memory with the first of them: next to every stage the copies,
// which the tensor core makes itself, took a fifth of its time.  A third set of atoms is begun with when the stage six before it,
// and so the last that read the first set, is done.
constexpr uint32_t kScaleColumns = 12, kScaleSets = 3;    // tensor memory of a set: an atom of the lanes and of each half of the columns
constexpr uint32_t kTmem = 512;
constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
static_assert(4 * kScaleSets - 4 >= kStages + 2 && kTile + kScaleSets * kScaleColumns <= kTmem && kSmem <= 227 * 1024, "does not fit an SM");

struct Params {
  void* y;
  uint64_t ldy;
  uint32_t m, n;
  uint32_t begin, stages;        // 128-value blocks along a row: the first, a multiple of four, and how many
  uint32_t kt;                   // scale atoms, of four of them
  uint32_t lane_tiles, tiles;
  uint32_t each;                 // GATHER: blocks that a sum in the accumulator has, a multiple of four
};

__device__ uint32_t g_gave_up;   // counts up

// kind::mxf8f6f4: E4M3 x E4M3, E8M0 scales, 256 x 256.
constexpr uint32_t kInstruction = (kTile / 8) << 17 | 1u << 23 | (kTile / 128) << 27;

__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t sa, uint32_t sb, uint32_t add, uint32_t elected) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %6, 0;\n\tsetp.ne.u32 q, %7, 0;\n\t"
               "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(what), "r"(sa), "r"(sb), "r"(add), "r"(elected) : "memory");
}

// ADD: to what y holds.  GATHER: a long sum's parts of p.each blocks leave the accumulator one after another and are added in
// registers.
template <typename G, bool ADD, bool GATHER>
__global__ void __launch_bounds__(kThreads, 1)
fp8_pair_kernel(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap column_map,
                const __grid_constant__ CUtensorMap lane_scales, const __grid_constant__ CUtensorMap column_scales,
                const __grid_constant__ Params p) {
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_address(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * kStage);
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages, drained = ready + 8;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 2);

  const uint32_t warp = warp_index(), lane = threadIdx.x % 32, rank = cluster_rank();
  const uint32_t tile0 = blockIdx.x / 2, tile_step = gridDim.x / 2, stages = p.stages;

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
      const uint32_t lane_atom = n0 / 128 * p.kt + p.begin / 4, column_atom = m0 / 128 * p.kt + p.begin / 4;
      for (uint32_t i = 0; i < stages; ++i) {
        const uint32_t at = stage0 + s * kStage, bar = first_full + 8 * s;
        if (!(ok = barrier_wait(empty + 8 * s, parity))) break;
        if (rank == 0) barrier_expect(full + 8 * s, 2 * (i % 4 ? 2 * kMatrix : kBytes), elected);
        copy_box_pair(at, &lane_map, (int)((p.begin + i) * kStageBytes), (int)n0, bar, elected);
        copy_box_pair(at + kMatrix, &column_map, (int)((p.begin + i) * kStageBytes), (int)(m0 + rank * kRows), bar, elected);
        if (i % 4 == 0) {
          copy_box_pair(at + 2 * kMatrix, &lane_scales, 0, (int)(lane_atom + i / 4), bar, elected);
          copy_box_pair(at + 2 * kMatrix + kScales, &column_scales, 0, (int)(column_atom + i / 4), bar, elected);
          copy_box_pair(at + 2 * kMatrix + 2 * kScales, &column_scales, 0, (int)(column_atom + p.kt + i / 4), bar, elected);   // past the last: zero
        }
        ++issued;
        if (++s == kStages) s = 0, parity ^= 1;
      }
    }
    if (rank == 0) await_copies(full, issued, kStages);      // for both blocks, which end together
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t elected = elect();
      uint32_t q = 0, s = 0, parity = 0, set = 0;
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step, ++q) {
        if (!(ok = barrier_wait(drained, (q & 1) ^ 1))) break;
        tmem_fence_after();
        uint32_t part_end = p.each;
        for (uint32_t i = 0; i < stages; ++i) {
          bool begin = i == 0;
          if (GATHER && i == part_end) {
            tensor_commit_pair(ready, elected);
            ++q;
            if (!(ok = barrier_wait(drained, (q & 1) ^ 1))) break;
            part_end += p.each;
            begin = true;
          }
          if (!(ok = barrier_wait(full + 8 * s, parity))) break;
          tmem_fence_after();
          const uint32_t at = stage0 + s * kStage, ts = tmem + kTile + set * kScaleColumns;
          const uint64_t lanes = swizzled_rows(at), columns = swizzled_rows(at + kMatrix), scales = scale_rows(at + 2 * kMatrix);
          const uint32_t tl = ts, tc = ts + 4, what = kInstruction | (i % 4) << 29 | (i % 4) << 4;   // the block's byte of the four
          if (i % 4 == 0) {
            scales_to_tmem_pair(tl, scales, elected);
            scales_to_tmem_pair(tc, scales + kScales / 16, elected);
            scales_to_tmem_pair(tc + 4, scales + 2 * kScales / 16, elected);
          }
          // descriptors count in units of 16 bytes
#pragma unroll
          for (uint32_t h = 0; h < 4; ++h)   // 32 values
            multiply(tmem, lanes + h * 2, columns + h * 2, what, tl, tc, !begin || h, elected);
          if (i % 4 == 3 || i + 1 == stages) set = set + 1 == kScaleSets ? 0 : set + 1;
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
      uint32_t r[8][16];
      if constexpr (GATHER) {
        float sum[8][16] = {};
        const uint32_t parts = (stages + p.each - 1) / p.each;
        for (uint32_t part = 0; part < parts; ++part) {
          if (part) ++q;
          if (!(ok = barrier_wait(ready, q & 1))) break;
          tmem_fence_after();
#pragma unroll
          for (uint32_t c = 0; c < 8; ++c) {
            uint32_t more[16];
            tmem_load16(tmem + (group * 32 << 16) + half + 16 * c, more);
            tmem_load_wait();
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) sum[c][j] += __uint_as_float(more[j]);
          }
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) barrier_arrive_cluster(first_drained);
        }
        if (!ok) break;
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c)
#pragma unroll
          for (uint32_t j = 0; j < 16; ++j) r[c][j] = __float_as_uint(sum[c][j]);
      } else {
        if (!(ok = barrier_wait(ready, q & 1))) break;
        tmem_fence_after();
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) tmem_load16(tmem + (group * 32 << 16) + half + 16 * c, r[c]);
        tmem_load_wait();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) barrier_arrive_cluster(first_drained);
      }
      if (n < p.n) {
        G* y = static_cast<G*>(p.y) + (uint64_t)m * p.ldy + n;
        const auto value = [](uint32_t bits, const G* to) { return ADD ? __uint_as_float(bits) + (float)*to : __uint_as_float(bits); };
        if (have == 128) {
#pragma unroll
          for (uint32_t c = 0; c < 128; ++c, y += p.ldy) put(y, value(r[c / 16][c % 16], y));
        } else {
#pragma unroll
          for (uint32_t c = 0; c < 128; ++c, y += p.ldy)
            if (c < have) put(y, value(r[c / 16][c % 16], y));
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

template <typename G, bool ADD, bool GATHER>
cudaError_t launch(const Fp8& a, const Fp8& b, const MatrixOut& y, uint32_t begin, uint32_t count, uint32_t each, cudaStream_t stream) {
  static Device device;
  const Device::Facts* facts;
  cudaError_t e = device.prepare(fp8_pair_kernel<G, ADD, GATHER>, kThreads, kSmem, 0, &facts);
  if (e != cudaSuccess) return e;
  const uint64_t nb = (a.cols + kFp8Block - 1) / kFp8Block, kt = (nb + 3) / 4, lane_tiles = (b.rows + kTile - 1) / kTile;
  const uint64_t tiles = lane_tiles * ((a.rows + kTile - 1) / kTile);
  const uint64_t a_atoms = (a.rows + 127) / 128 * kt, b_atoms = (b.rows + 127) / 128 * kt;
  if (tiles > 0x7FFFFFFFull || a_atoms > 0x7FFFFF00ull - kt || b_atoms > 0x7FFFFF00ull - kt) return cudaErrorInvalidConfiguration;
  CUtensorMap lane_map, column_map, lane_scales, column_scales;
  e = encode_rows(&lane_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, nb * kFp8Block, b.rows, nb * kFp8Block, kRows);
  if (e == cudaSuccess) e = encode_rows(&column_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, nb * kFp8Block, a.rows, nb * kFp8Block, kRows);
  // scale bytes by whole atoms of 512
  if (e == cudaSuccess) e = encode_plain(&lane_scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, b.scales, 128, b_atoms, 512, 128, 1);
  if (e == cudaSuccess) e = encode_plain(&column_scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, a.scales, 128, a_atoms, 512, 128, 1);
  if (e != cudaSuccess) return e;
  const Params p = {y.p, y.ld, (uint32_t)y.rows, (uint32_t)y.cols, begin, count, (uint32_t)kt, (uint32_t)lane_tiles, (uint32_t)tiles, each};
  const unsigned pairs = (unsigned)std::min<uint64_t>(tiles, (uint64_t)facts->sms / 2);
  return launch_overlapped(fp8_pair_kernel<G, ADD, GATHER>, 2 * pairs, kThreads, kSmem, 2, stream, lane_map, column_map, lane_scales, column_scales, p);
}

}  // namespace

cudaError_t launch_fp8_matmul_pair(const Fp8& a, const Fp8& b, const MatrixOut& y, uint32_t begin, uint32_t count, uint32_t one_sum, cudaStream_t stream) {
  if (y.type == kBF16) {
    if (begin) return cudaErrorInvalidValue;
    return count > one_sum ? launch<__nv_bfloat16, false, true>(a, b, y, 0, count, one_sum, stream) : launch<__nv_bfloat16, false, false>(a, b, y, 0, count, 0, stream);
  }
  return begin ? launch<float, true, false>(a, b, y, begin, count, 0, stream) : launch<float, false, false>(a, b, y, 0, count, 0, stream);
}

cudaError_t fp8_matmul_pair_gave_up(uint32_t* count, cudaStream_t stream) { return read_count(g_gave_up, count, stream); }
cudaError_t fp8_matmul_pair_count(const uint32_t** at) { return count_address(g_gave_up, at); }

}  // namespace rudra
