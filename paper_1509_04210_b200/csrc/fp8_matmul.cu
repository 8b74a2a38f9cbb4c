// y = a b^T with both matrices in FP8 (E4M3, a scale for each 128 values of a row), on the block-scaled tensor cores.
//
// The tensor core multiplies the codes and applies power-of-two scales itself, a byte for each 32 values of a row; four
// instructions along a row are given the same byte, so that a block of 128 needs one in memory and a sum never leaves its
// accumulator for its scales.  The kernel only moves codes and scale bytes: TMA brings 128-byte pieces of rows, one
// block each, into swizzled shared memory, bulk copies bring the scale bytes, tcgen05.cp places those in tensor
// memory next to the accumulator.  Rows of b (a layer's outputs) are the 128 lanes of an accumulator and rows
// of a (tokens) its columns, so one shape serves a single token (16 columns) as well as a batch, and
// neighbouring lanes write neighbouring outputs.
//
// Few tiles: the reduction is split over the blocks of a cluster.  Their parts are added in rank order
// through distributed shared memory, so the sum does not depend on the run.
//
// Up to 16 tokens the kernel takes x itself: every block brings its slice of the few rows to FP8 on
// the way into shared memory.
//
// Measured: one token through 4096 x 9216 9.1 us (37.7 MB of weights at 4.1 TB/s; 2 us of it before the first and 1 joining; a kernel that
// multiplies on the ordinary cores as the weights pass took 13), 256 x 4096 x 4096 8.1 us, 128 x 1000 x 4096 5.3 us, 512 x 512 x 512
// 2.9 us.  A stage of 64 columns brings 24 KB to an SM in 0.16 us, 83 bytes a cycle, which is what an SM takes in.
#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

// Warp 0 loads, warp 1 issues, warps 2-5 take the results; where x is brought to FP8 here, warps 2-9 do that.
template <int COLS, bool QUANTIZE> struct Shape {
  static constexpr uint32_t kQuantizers = QUANTIZE ? 8 : 0;
  static constexpr uint32_t kThreads = QUANTIZE ? 320 : 192;
  static constexpr uint32_t kLanes = 128 * kFp8Block;
  static constexpr uint32_t kColumns = COLS * kFp8Block;
  static constexpr uint32_t kScales = 512 * 2;                           // a scale atom of each operand
  static constexpr uint32_t kStage = kLanes + kColumns + kScales;
  static constexpr uint32_t kStages = COLS == 128 ? 6 : COLS == 64 ? 8 : COLS == 32 ? 9 : 10;
  // Tensor memory of a set of scale atoms.  An atom serves four stages and comes with the first of them; x brought to FP8 here has
  // one in every stage.  A set is written again once the last stage that read it is done, as the stage whose place it takes is.
  static constexpr uint32_t kScaleColumns = 8, kSets = QUANTIZE ? kStages : (kStages + 2 + 3) / 4 + 1;
  static constexpr uint32_t kTmem = 256;
  static constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
  static_assert(kStage % 1024 == 0 && COLS + kSets * kScaleColumns <= kTmem && kSmem <= 227 * 1024, "does not fit an SM");
};

struct Params {
  const uint8_t* lane_scales;     // of b
  const uint8_t* column_scales;   // of a
  void* y;
  uint64_t ldy;
  uint32_t m, n, k;               // rows of a, rows of b, their length
  uint32_t begin, stages;         // 128-value blocks along a row: the first, and how many
  uint32_t kt;                    // scale atoms, of four of them
  uint32_t lane_tiles;
  uint32_t split;                 // blocks of a cluster that share a tile
  uint32_t add;                   // to what y holds
  uint32_t each;                  // GATHER: blocks that a sum in the accumulator has
};

__device__ uint32_t g_gave_up;   // counts up

// Instruction descriptor of kind::mxf8f6f4: E4M3 x E4M3, E8M0 scales, M = 128.
template <int COLS> __device__ constexpr uint32_t instruction() { return (COLS / 8) << 17 | 1u << 23 | 1u << 27; }

__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t sa, uint32_t sb, uint32_t add, uint32_t elected) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %6, 0;\n\tsetp.ne.u32 q, %7, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(what), "r"(sa), "r"(sb), "r"(add), "r"(elected) : "memory");
}

// X: type of x where it is brought to FP8 here, else void.  GATHER: a long sum's parts of p.each blocks leave the accumulator one after
// another and are added in registers.
template <typename G, int COLS, typename X, bool GATHER>
__global__ void __launch_bounds__(Shape<COLS, !std::is_void<X>::value>::kThreads)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap column_map, const __grid_constant__ Params p,
                  const __grid_constant__ Rows<typename std::conditional<std::is_void<X>::value, float, X>::type> x) {
  constexpr bool kQuantize = !std::is_void<X>::value;
  using S = Shape<COLS, kQuantize>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_address(smem);
  float* part = reinterpret_cast<float*>(smem);      // [column][lane], once the stages are done with
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  const uint32_t full = smem_address(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages, drained = done + 8;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 2 * S::kStages + 2);

  const uint32_t warp = warp_index(), lane = threadIdx.x % 32;
  const uint32_t rank = p.split > 1 ? cluster_rank() : 0;
  const uint32_t tile = blockIdx.x / p.split;
  const uint32_t n0 = (tile % p.lane_tiles) * 128, m0 = (tile / p.lane_tiles) * COLS;
  const uint32_t first = p.begin + (uint32_t)((uint64_t)p.stages * rank / p.split), last = p.begin + (uint32_t)((uint64_t)p.stages * (rank + 1) / p.split);

  if (threadIdx.x == 0) {
    prefetch_map(&lane_map);
    if (!kQuantize) prefetch_map(&column_map);
    for (uint32_t s = 0; s < S::kStages; ++s) {
      barrier_init(full + 8 * s, kQuantize ? 2 : 1);
      barrier_init(empty + 8 * s, 1);
    }
    barrier_init(done, 1);
    if (GATHER) barrier_init(drained, 4);      // the warps that take results
    barrier_init_fence();
  }
  if (warp == 1) tmem_alloc(smem_address(slot), S::kTmem);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *slot;
  bool ok = true;
  admit_next_kernel();
  await_previous_kernel();

  const uint32_t group = warp % 4;                       // the lanes of tensor memory a warp may read
  const bool takes = warp >= 2 && warp < 6;
  float sum[GATHER ? COLS : 1] = {};
  uint32_t taken = 0;                                    // parts of the sum
  // The next part of the sum, as soon as it is there; the accumulator is then free for the one after it.
  const auto take = [&]() -> bool {
    if (!barrier_wait(done, taken & 1)) return false;
    tmem_fence_after();
#pragma unroll
    for (int c = 0; c < (GATHER ? COLS : 0); c += 16) {
      if (m0 + c >= p.m) continue;
      uint32_t r[16];
      tmem_load16(tmem + (group * 32 << 16) + c, r);
      tmem_load_wait();
#pragma unroll
      for (int j = 0; j < 16; ++j) sum[c + j] += __uint_as_float(r[j]);
    }
    ++taken;
    tmem_fence_before();
    __syncwarp();
    if (lane == 0) barrier_arrive(drained);
    return true;
  };

  if (warp == 0) {
    const uint32_t elected = elect();
    uint32_t s = 0, parity = 1, issued = 0;
    for (uint32_t i = first; i < last; ++i, ++issued) {
      if (!(ok = barrier_wait(empty + 8 * s, parity))) break;
      const uint32_t at = stage0 + s * S::kStage, bar = full + 8 * s, scales = at + S::kLanes + S::kColumns;
      const bool fresh = kQuantize || i == first || i % 4 == 0;
      barrier_expect(bar, S::kLanes + (fresh ? 512 : 0) + (kQuantize ? 0 : S::kColumns + (fresh ? 512 : 0)), elected);
      copy_box(at, &lane_map, (int)(i * kFp8Block), (int)n0, bar, elected);
      if (fresh) copy_bulk(scales, p.lane_scales + ((uint64_t)(n0 / 128) * p.kt + i / 4) * 512, 512, bar, elected);
      if (!kQuantize) {
        copy_box(at + S::kLanes, &column_map, (int)(i * kFp8Block), (int)m0, bar, elected);
        if (fresh) copy_bulk(scales + 512, p.column_scales + ((uint64_t)(m0 / 128) * p.kt + i / 4) * 512, 512, bar, elected);
      }
      if (++s == S::kStages) s = 0, parity ^= 1;
    }
    await_copies(full, issued, S::kStages);
  } else if (warp == 1) {
    const uint32_t elected = elect();
    uint32_t s = 0, parity = 0, set = 0, part_end = first + p.each, parts = 0;
    for (uint32_t i = first; i < last; ++i) {
      bool begin = i == first;
      if (GATHER && i == part_end) {
        tensor_commit(done, elected);
        if (!(ok = barrier_wait(drained, parts++ & 1))) break;
        part_end += p.each;
        begin = true;
      }
      if (!(ok = barrier_wait(full + 8 * s, parity))) break;
      tmem_fence_after();
      const uint32_t at = stage0 + s * S::kStage, ts = tmem + COLS + set * S::kScaleColumns;
      const uint64_t lanes = swizzled_rows(at), columns = swizzled_rows(at + S::kLanes), scales = scale_rows(at + S::kLanes + S::kColumns);
      const uint32_t tl = ts, tc = ts + 4, what = instruction<COLS>() | (i % 4) << 29 | (i % 4) << 4;   // the block's byte of the four
      const uint32_t mine = tc + m0 % 128 / 32;                        // a tile of 64 rows may be the second half of an atom
      // descriptors count in units of 16 bytes
      if (kQuantize || i == first || i % 4 == 0) {
        scales_to_tmem(tl, scales, elected);
        scales_to_tmem(tc, scales + 32, elected);
      }
#pragma unroll
      for (uint32_t h = 0; h < 4; ++h)   // 32 values
        multiply(tmem, lanes + h * 2, columns + h * 2, what, tl, mine, !begin || h, elected);
      if (kQuantize || i % 4 == 3) set = set + 1 == S::kSets ? 0 : set + 1;
      tensor_commit(empty + 8 * s, elected);
      if (++s == S::kStages) s = 0, parity ^= 1;
    }
    if (ok) tensor_commit(done, elected);
  } else if (kQuantize) {
    // a warp brings every eighth stage's values to FP8, where TMA and the bulk copies would have put them
    using T = typename std::conditional<kQuantize, X, float>::type;
    for (uint32_t i = first + (warp - 2); i < last; i += S::kQuantizers) {
      const uint32_t c = i - first, s = c % S::kStages;
      // a part of the sum has all its stages of this warp
      if (GATHER && takes && c / p.each > taken && !(ok = take())) break;
      uint8_t* stage = smem + s * S::kStage + S::kLanes;
      bool free = c < S::kStages;
#pragma unroll 1
      for (uint32_t r0 = 0; r0 < p.m; r0 += 8) {      // eight lanes to a row: eight rows on their way at a time
        Values<T> v[2];
        const uint32_t k0 = i * kFp8Block + lane % 8 * kValues;
        const int have = k0 < p.k ? (int)min((uint32_t)kValues, p.k - k0) : 0;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          const uint32_t r = r0 + 4 * h + lane / 8;
          const int some = r < p.m ? have : 0;
          v[h].template load<true>(x, some ? r * x.ld + k0 : 0, some);
        }
        if (!free && !(ok = free = barrier_wait(empty + 8 * s, (c / S::kStages & 1) ^ 1))) break;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          if (r0 + 4 * h >= p.m) break;
          const uint32_t r = r0 + 4 * h + lane / 8, u = lane % 8;
          const uint32_t e = fp8_scale_byte(fp8_block_max_bits(v[h].max_bits()));
          const uint4 w = e4m3_codes([&](int j) { return v[h].get(j); }, e);
          if (r >= p.m) continue;
          *reinterpret_cast<uint4*>(stage + r * 128 + (u ^ (r % 8)) * 16) = w;
          if (u == 0) stage[S::kColumns + 512 + r * 16 + i % 4] = (uint8_t)e;   // r < 16
        }
      }
      if (!ok) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) barrier_arrive(full + 8 * s);
    }
  }
  __syncwarp();

  const uint32_t n = n0 + group * 32 + lane;
  if (takes) {
    if constexpr (GATHER) {
      const uint32_t parts = (last - first + p.each - 1) / p.each;
      while (ok && taken < parts) ok = take();
#pragma unroll
      for (int c = 0; c < COLS; ++c) {
        if (m0 + c >= p.m) continue;
        if (p.split > 1) part[c * 128 + group * 32 + lane] = sum[c];
        else if (n < p.n) put(static_cast<G*>(p.y) + (uint64_t)(m0 + c) * p.ldy + n, sum[c]);
      }
    } else {
      if (!barrier_wait(done, 0)) ok = false;
      tmem_fence_after();
#pragma unroll 1
      for (uint32_t c = 0; c < COLS && m0 + c < p.m; c += 16) {
        uint32_t r[16];
        tmem_load16(tmem + (group * 32 << 16) + c, r);
        tmem_load_wait();
        if (p.split > 1) {
#pragma unroll
          for (uint32_t j = 0; j < 16; ++j) part[(c + j) * 128 + group * 32 + lane] = __uint_as_float(r[j]);
        } else if (n < p.n) {
          G* y = static_cast<G*>(p.y) + (uint64_t)(m0 + c) * p.ldy + n;
#pragma unroll
          for (uint32_t j = 0; j < 16; ++j, y += p.ldy)
            if (m0 + c + j < p.m) put(y, __uint_as_float(r[j]) + (sizeof(G) == 4 && p.add ? (float)*y : 0.f));
        }
      }
    }
  }
  if (!ok) atomicAdd(&g_gave_up, 1u);
  __syncwarp();
  if (p.split > 1)
    join_parts(stage0, p.split, rank, min((uint32_t)COLS, p.m - m0), min(128u, p.n - n0), static_cast<G*>(p.y) + (uint64_t)m0 * p.ldy + n0, p.ldy, sizeof(G) == 4 && p.add);
  tmem_fence_before();
  __syncthreads();
  if (warp == 1) {
    tmem_fence_after();
    tmem_free(tmem, S::kTmem);
  }
}

// How long a product takes, in ns, by its shape.  Measured (warm, one after another, weights out of HBM): a stage of 16, 32, 64 and
// 128 columns 140, 145, 170 and 210 ns, what comes after a tile's last stage 100 to 1000, joining the parts of a tile 1100 to 4350 by its
// rows, 2000 for setting up, again for every round of blocks; a pair's stage 300 (360 on all SMs), 1000 a tile and 2700 once.  For instance
// 256 x 4096 x 4096: 64 columns 8.1 us, 128 columns 9.7 and split in two 10.5, pairs 13.7; 128 x 4096 x 4096: 64 columns 7.9 us, in two parts
// 9.0, 128 columns in four parts 8.8; 65 x 4096 x 4096: that 7.4; 512 x 300 x 8192: 64 columns 11.7 us and in four parts 7.0, 128 columns in
// eight parts 7.8; 1000 x 4096 x 4096: pairs 14.7 us, 128 columns 19.6; 4096 x 4096 x 9216: pairs 109 us, 128 columns 134, 64 columns 190.
struct Timed {
  uint32_t split;
  uint64_t time;
};
Timed best_split(const Device::Facts& f, int columns, uint64_t m, uint64_t n, uint64_t stages) {
  const int i = columns == 16 ? 0 : columns == 32 ? 1 : columns == 64 ? 2 : 3;
  constexpr uint64_t kStageTime[4] = {140, 145, 170, 210}, kAfter[4] = {100, 200, 500, 1000}, kJoin[4] = {1100, 1400, 1000, 1150}, kJoinRow[4] = {0, 0, 30, 25};
  const uint64_t tiles = ((n + 127) / 128) * ((m + columns - 1) / columns), waves = (tiles + f.sms - 1) / f.sms;
  Timed best = {1, waves * (2000 + stages * kStageTime[i] + kAfter[i])};
  for (uint32_t k = 1; k < 4; ++k) {
    const uint32_t split = 1u << k;
    const uint64_t time = 2000 + (stages + split - 1) / split * kStageTime[i] + kAfter[i] + kJoin[i] + std::min<uint64_t>(m, columns) * kJoinRow[i];
    if (split <= stages && tiles <= (uint64_t)f.clusters[k] && time < best.time) best = {split, time};
  }
  return best;
}
uint64_t pair_time(const Device::Facts& f, uint64_t m, uint64_t n, uint64_t stages) {
  const uint64_t tiles = ((n + 255) / 256) * ((m + 255) / 256), waves = (2 * tiles + f.sms - 1) / f.sms;
  return 2700 + waves * (stages * (waves > 1 ? 360 : 300) + 1000);
}

// Blocks along the rows that one sum takes.
struct Blocks {
  uint32_t begin, count;
};

// Blocks that an accumulator's sum has at most where results are bf16; longer ones are gathered in registers.  The tensor core cuts a sum off
// where it adds to it: of 2^24 positive values in a cluster of eight 6e-3 were lost, in parts of 512 blocks under 2e-4 are, a twentieth
// of what the rounding to bf16 takes off.
constexpr uint32_t kOneSum = 512;
static_assert(kOneSum % 8 == 0, "every quantizing warp has a stage in a whole part");

template <typename G, int COLS, typename X>
cudaError_t launch(const Fp8& a, const MatrixIn* x, const Fp8& b, const MatrixOut& y, Blocks part, cudaStream_t stream) {
  using S = Shape<COLS, !std::is_void<X>::value>;
  using T = typename std::conditional<std::is_void<X>::value, float, X>::type;
  static Device device;
  const Device::Facts* facts;
  cudaError_t e = device.prepare(fp8_matmul_kernel<G, COLS, X, false>, S::kThreads, S::kSmem, 0, &facts);
  if (e != cudaSuccess) return e;
  Params p = {};
  const uint64_t nb = (b.cols + kFp8Block - 1) / kFp8Block;
  p.lane_scales = static_cast<const uint8_t*>(b.scales);
  p.column_scales = static_cast<const uint8_t*>(a.scales);
  p.y = y.p;
  p.ldy = y.ld;
  p.m = (uint32_t)y.rows;
  p.n = (uint32_t)y.cols;
  p.k = (uint32_t)b.cols;
  p.begin = part.begin;
  p.stages = part.count;
  p.add = part.begin != 0;
  p.kt = (uint32_t)((nb + 3) / 4);
  p.lane_tiles = (p.n + 127) / 128;
  const uint64_t tiles = (uint64_t)p.lane_tiles * ((p.m + COLS - 1) / COLS);
  if (tiles > 0x0FFFFFFFull) return cudaErrorInvalidConfiguration;
  p.split = best_split(*facts, COLS, p.m, p.n, p.stages).split;
  CUtensorMap lane_map, column_map = {};
  e = encode_rows(&lane_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, nb * kFp8Block, b.rows, nb * kFp8Block, 128);
  if (e == cudaSuccess && !x) e = encode_rows(&column_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, nb * kFp8Block, a.rows, nb * kFp8Block, COLS);
  if (e != cudaSuccess) return e;
  const auto run = [&](auto* kernel) {
    return launch_overlapped(kernel, (uint32_t)(tiles * p.split), S::kThreads, S::kSmem, p.split, stream, lane_map, column_map, p,
                             x ? Rows<T>::of(x->p, x->rows, x->cols, x->ld, 0) : Rows<T>::of(nullptr, 0, 0, 0, 0));
  };
  if constexpr (sizeof(G) == 2) {
    if ((p.stages + p.split - 1) / p.split > kOneSum) {
      p.each = kOneSum;
      static Device gathering;
      e = gathering.prepare(fp8_matmul_kernel<G, COLS, X, true>, S::kThreads, S::kSmem, 0, &facts);
      return e != cudaSuccess ? e : run(fp8_matmul_kernel<G, COLS, X, true>);
    }
  }
  return run(fp8_matmul_kernel<G, COLS, X, false>);
}

// The shape that is done soonest.  Sixteen or 32 columns only where they take all rows: scale bytes come in atoms of 128 rows, of
// which a tile takes all, the first part or a half.
template <typename G> cudaError_t by_time(const Fp8& a, const Fp8& b, const MatrixOut& y, Blocks part, cudaStream_t stream) {
  const uint64_t m = y.rows, n = y.cols, stages = part.count;
  if (m <= 16) return launch<G, 16, void>(a, nullptr, b, y, part, stream);
  if (m <= 32) return launch<G, 32, void>(a, nullptr, b, y, part, stream);
  static Device device;
  const Device::Facts* facts;
  const cudaError_t e = device.prepare(fp8_matmul_kernel<G, 64, void, false>, Shape<64, false>::kThreads, Shape<64, false>::kSmem, 0, &facts);
  if (e != cudaSuccess) return e;
  const uint64_t narrow = best_split(*facts, 64, m, n, stages).time, wide = best_split(*facts, 128, m, n, stages).time;
  if (pair_time(*facts, m, n, stages) < std::min(narrow, wide)) return launch_fp8_matmul_pair(a, b, y, part.begin, part.count, kOneSum, stream);
  return narrow <= wide ? launch<G, 64, void>(a, nullptr, b, y, part, stream) : launch<G, 128, void>(a, nullptr, b, y, part, stream);
}

// f32 results of long rows are gathered in memory: the tensor core cuts a sum off where it adds to it, every 32 values, by more the more
// there is of it.  (Rows of 2^20 positive values: 1.6e-4 too little in one sum.)  So many blocks to a sum, about; a multiple of the four
// whose scale bytes share an atom.  Every sum is a launch that reads y and writes it again: 2048 x 4096 x 131072 takes 2.04 ms in f32 and 0.80 in
// bf16, whose parts stay in registers; 128 x 4096 x 131072 217 and 93 us.
constexpr uint32_t kGathered = 64;
template <typename G, typename F> cudaError_t in_sums(uint64_t cols, F&& body) {
  const uint32_t blocks = (uint32_t)((cols + kFp8Block - 1) / kFp8Block), sums = sizeof(G) == 4 ? std::max(1u, (blocks + kGathered / 2) / kGathered) : 1;
  const uint32_t each = (blocks + sums - 1) / sums + 3 & ~3u;
  for (uint32_t at = 0; at < blocks; at += each) {
    const cudaError_t e = body(Blocks{at, std::min(each, blocks - at)});
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}
template <typename G> cudaError_t product(const Fp8& a, const Fp8& b, const MatrixOut& y, cudaStream_t stream) {
  return in_sums<G>(b.cols, [&](Blocks part) { return by_time<G>(a, b, y, part, stream); });
}

template <typename G, typename X> cudaError_t quantizing(const MatrixIn& x, const Fp8& b, const MatrixOut& y, cudaStream_t stream) {
  return in_sums<G>(b.cols, [&](Blocks part) { return launch<G, 16, X>({}, &x, b, y, part, stream); });
}

cudaError_t nothing(const MatrixOut& y, cudaStream_t stream) {   // a sum over nothing
  return cudaMemset2DAsync(y.p, y.ld * (y.type == kBF16 ? 2 : 4), 0, y.cols * (y.type == kBF16 ? 2 : 4), y.rows, stream);
}

// Rows of x up to which the product brings them to FP8 itself, and beyond which that is a launch of its own: they fill the
// narrowest tile.
constexpr uint64_t kQuantizedInside = 16;

}  // namespace

cudaError_t launch_fp8_matmul(const Fp8& a, const Fp8& b, const MatrixOut& y, cudaStream_t stream) {
  if (a.cols == 0) return nothing(y, stream);
  return y.type == kBF16 ? product<__nv_bfloat16>(a, b, y, stream) : product<float>(a, b, y, stream);
}

uint64_t fp8_linear_workspace(uint64_t m, uint64_t k) {
  if (m <= kQuantizedInside) return 0;
  const uint64_t nb = (k + kFp8Block - 1) / kFp8Block;
  return m * nb * kFp8Block + (m + 127) / 128 * ((nb + 3) / 4) * 512;
}

cudaError_t launch_fp8_linear(const MatrixIn& x, const Fp8& b, const MatrixOut& y, void* workspace, cudaStream_t stream) {
  if (x.cols == 0) return nothing(y, stream);
  if (x.rows <= kQuantizedInside) {
    if (y.type == kBF16) return x.type == kBF16 ? quantizing<__nv_bfloat16, __nv_bfloat16>(x, b, y, stream) : quantizing<__nv_bfloat16, float>(x, b, y, stream);
    return x.type == kBF16 ? quantizing<float, __nv_bfloat16>(x, b, y, stream) : quantizing<float, float>(x, b, y, stream);
  }
  uint8_t* codes = static_cast<uint8_t*>(workspace);
  uint8_t* scales = codes + x.rows * ((x.cols + kFp8Block - 1) / kFp8Block) * kFp8Block;
  const cudaError_t e = launch_fp8_quantize(x, false, false, codes, scales, stream);
  return e != cudaSuccess ? e : launch_fp8_matmul({codes, scales, x.rows, x.cols}, b, y, stream);
}

cudaError_t fp8_matmul_gave_up(uint32_t* count, cudaStream_t stream) { return read_count(g_gave_up, count, stream); }
cudaError_t fp8_matmul_count(const uint32_t** at) { return count_address(g_gave_up, at); }

}  // namespace rudra
