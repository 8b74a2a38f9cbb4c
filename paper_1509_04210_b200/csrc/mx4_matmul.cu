// y = a b^T with both matrices in MX4, on the block-scaled 4-bit tensor cores.
//
// The tensor core multiplies E2M1 codes and applies the two blocks' power-of-two scales itself, so the
// kernel only moves codes and scale bytes: TMA brings 128-byte (256-value) pieces of rows into
// swizzled shared memory, bulk copies bring the scale bytes, tcgen05.cp places those in tensor memory
// next to the accumulators.  Rows of b (a layer's outputs) are the 128 lanes of an accumulator and rows
// of a (tokens) its columns, so one shape serves a single token (16 columns) as well as a batch, and
// neighbouring lanes write neighbouring outputs.
//
// Few tiles: the reduction is split over the blocks of a cluster.  Their parts are added in rank order
// through distributed shared memory, so the sum does not depend on the run.
//
// Up to 16 tokens the kernel takes x itself: every block brings its slice of the few rows to MX4 on
// the way into shared memory, which costs less than another launch (figures at kQuantizedInside).
//
// Measured: one token through 4096 x 9216 6.2 us (20 MB of weights, of which 1.9 us are spent before the first
// and 1.2 us joining), 100 x 1000 x 4096 6.9 us, 256 x 4096 x 4096 7.6 us: latencies, of the copies and of the
// stages that follow one another (0.2 us each), not a rate.
#include <algorithm>
#include <type_traits>

#include "blocks.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

constexpr uint32_t kStageBytes = 128;   // of a row per stage: 256 values

// Warp 0 loads, warp 1 issues, warps 2-5 take the results; where x is brought to MX4 here, warps 2-9 do that.
template <int COLS, bool QUANTIZE> struct Shape {
  static constexpr uint32_t kQuantizers = QUANTIZE ? 8 : 0;
  static constexpr uint32_t kThreads = QUANTIZE ? 320 : 192;
  static constexpr uint32_t kLanes = 128 * kStageBytes;
  static constexpr uint32_t kColumns = COLS * kStageBytes;
  static constexpr uint32_t kScales = 1024 * 2;                          // two 512-byte scale atoms of each operand
  static constexpr uint32_t kStage = kLanes + kColumns + kScales;
  static constexpr uint32_t kStages = COLS == 128 ? 6 : COLS == 64 ? 8 : COLS == 32 ? 9 : 10;
  static constexpr uint32_t kScaleColumns = 16;                          // tensor memory per stage
  static constexpr uint32_t kTmem = 256;
  static constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
  static_assert(COLS + kStages * kScaleColumns <= kTmem && kSmem <= 227 * 1024, "does not fit an SM");
};

struct Params {
  const uint8_t* lane_scales;     // of b
  const uint8_t* column_scales;   // of a
  void* y;
  uint64_t ldy;
  uint32_t m, n, k;               // rows of a, rows of b, their length
  uint32_t kt;                    // 128-value scale atoms along a row
  uint32_t lane_tiles;
  uint32_t split;                 // blocks of a cluster that share a tile
};

__device__ uint32_t g_gave_up;   // counts up

// Instruction descriptor of kind::mxf4: E2M1 x E2M1, E8M0 scales, M = 128.
template <int COLS> __device__ constexpr uint32_t instruction() {
  return 1u << 7 | 1u << 10 | (COLS / 8) << 17 | 1u << 23 | 1u << 27;
}

__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t sa, uint32_t sb, uint32_t add, uint32_t elected) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %6, 0;\n\tsetp.ne.u32 q, %7, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(what), "r"(sa), "r"(sb), "r"(add), "r"(elected) : "memory");
}

// X: type of x where it is brought to MX4 here, else void.
template <typename G, int COLS, typename X>
__global__ void __launch_bounds__(Shape<COLS, !std::is_void<X>::value>::kThreads)
matmul_kernel(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap column_map, const __grid_constant__ Params p,
              const __grid_constant__ Rows<typename std::conditional<std::is_void<X>::value, float, X>::type> x) {
  constexpr bool kQuantize = !std::is_void<X>::value;
  using S = Shape<COLS, kQuantize>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_address(smem);
  float* part = reinterpret_cast<float*>(smem);      // [column][lane], once the stages are done with
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  const uint32_t full = smem_address(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 2 * S::kStages + 1);

  const uint32_t warp = warp_index(), lane = threadIdx.x % 32;
  const uint32_t rank = p.split > 1 ? cluster_rank() : 0;
  const uint32_t tile = blockIdx.x / p.split;
  const uint32_t n0 = (tile % p.lane_tiles) * 128, m0 = (tile / p.lane_tiles) * COLS;
  const uint32_t stages = (p.kt + 1) / 2;
  const uint32_t first = (uint32_t)((uint64_t)stages * rank / p.split), last = (uint32_t)((uint64_t)stages * (rank + 1) / p.split);

  if (threadIdx.x == 0) {
    prefetch_map(&lane_map);
    if (!kQuantize) prefetch_map(&column_map);
    for (uint32_t s = 0; s < S::kStages; ++s) {
      barrier_init(full + 8 * s, kQuantize ? 2 : 1);
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
  admit_next_kernel();
  await_previous_kernel();

  if (warp == 0) {
    const uint32_t elected = elect();
    uint32_t s = 0, parity = 1, issued = 0;
    for (uint32_t i = first; i < last; ++i, ++issued) {
      if (!(ok = barrier_wait(empty + 8 * s, parity))) break;
      const uint32_t at = stage0 + s * S::kStage, bar = full + 8 * s, scales = at + S::kLanes + S::kColumns;
      const uint32_t atoms = min(2u, p.kt - 2 * i);
      barrier_expect(bar, S::kLanes + atoms * 512 + (kQuantize ? 0 : S::kColumns + atoms * 512), elected);
      copy_box(at, &lane_map, (int)(i * kStageBytes), (int)n0, bar, elected);
      copy_bulk(scales, p.lane_scales + ((uint64_t)(n0 / 128) * p.kt + 2 * i) * 512, atoms * 512, bar, elected);
      if (!kQuantize) {
        copy_box(at + S::kLanes, &column_map, (int)(i * kStageBytes), (int)m0, bar, elected);
        copy_bulk(scales + 1024, p.column_scales + ((uint64_t)(m0 / 128) * p.kt + 2 * i) * 512, atoms * 512, bar, elected);
      }
      if (++s == S::kStages) s = 0, parity ^= 1;
    }
    await_copies(full, issued, S::kStages);
  } else if (warp == 1) {
    const uint32_t elected = elect();
    uint32_t s = 0, parity = 0;
    for (uint32_t i = first; i < last; ++i) {
      if (!(ok = barrier_wait(full + 8 * s, parity))) break;
      tmem_fence_after();
      const uint32_t at = stage0 + s * S::kStage, ts = tmem + COLS + s * S::kScaleColumns;
      const uint64_t lanes = swizzled_rows(at), columns = swizzled_rows(at + S::kLanes), scales = scale_rows(at + S::kLanes + S::kColumns);
      const uint32_t atoms = min(2u, p.kt - 2 * i);
      // descriptors count in units of 16 bytes
#pragma unroll
      for (uint32_t k = 0; k < 2; ++k) {
        if (k == atoms) break;
        const uint32_t tl = ts + k * 8, tc = tl + 4;
        scales_to_tmem(tl, scales + 32 * k, elected);
        scales_to_tmem(tc, scales + (64 + 32 * k), elected);
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h)   // 64 values: two scale bytes of the four
          multiply(tmem, lanes + (2 * k + h) * 2, columns + (2 * k + h) * 2, instruction<COLS>() | (2 * h) << 29 | (2 * h) << 4, tl, tc,
                   i != first || k || h, elected);
      }
      tensor_commit(empty + 8 * s, elected);
      if (++s == S::kStages) s = 0, parity ^= 1;
    }
    if (ok) tensor_commit(done, elected);
  } else if (kQuantize) {
    // a warp brings every eighth stage's values to MX4, where TMA and the bulk copies would have put them
    using T = typename std::conditional<kQuantize, X, float>::type;
    for (uint32_t i = first + (warp - 2); i < last; i += S::kQuantizers) {
      const uint32_t c = i - first, s = c % S::kStages;
      uint8_t* stage = smem + s * S::kStage + S::kLanes;
      bool free = c < S::kStages;
#pragma unroll 1
      for (uint32_t r0 = 0; r0 < p.m; r0 += 8) {      // 16 lanes to a row: eight rows on their way at a time
        Values<T> v[4];
        const uint32_t k0 = i * 256 + lane % 16 * kValues;
        const int have = k0 < p.k ? (int)min((uint32_t)kValues, p.k - k0) : 0;
#pragma unroll
        for (uint32_t h = 0; h < 4; ++h) {
          const uint32_t r = r0 + 2 * h + lane / 16;
          const int some = r < p.m ? have : 0;
          v[h].template load<true>(x, some ? r * x.ld + k0 : 0, some);
        }
        if (!free && !(ok = free = barrier_wait(empty + 8 * s, (c / S::kStages & 1) ^ 1))) break;
#pragma unroll
        for (uint32_t h = 0; h < 4; ++h) {
          if (r0 + 2 * h >= p.m) break;
          const uint32_t r = r0 + 2 * h + lane / 16, u = lane % 16;
          const uint32_t e = scale_byte(block_max_bits(v[h].max_bits()), 2);
          const uint2 w = e2m1_codes(v[h], e);
          if (r >= p.m) continue;
          *reinterpret_cast<uint2*>(stage + r * 128 + ((u / 2) ^ (r % 8)) * 16 + u % 2 * 8) = w;
          if (u % 2 == 0) stage[S::kColumns + 1024 + u / 8 * 512 + r * 16 + u / 2 % 4] = (uint8_t)e;   // r < 16
        }
      }
      if (!ok) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) barrier_arrive(full + 8 * s);
    }
  }
  __syncwarp();

  const uint32_t group = warp % 4;                       // the lanes of tensor memory a warp may read
  const uint32_t n = n0 + group * 32 + lane;
  if (warp >= 2 && warp < 6) {
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
          if (m0 + c + j < p.m) put(y, __uint_as_float(r[j]));
      }
    }
  }
  if (!ok) atomicAdd(&g_gave_up, 1u);
  __syncwarp();
  if (p.split > 1)
    join_parts(stage0, p.split, rank, min((uint32_t)COLS, p.m - m0), min(128u, p.n - n0), static_cast<G*>(p.y) + (uint64_t)m0 * p.ldy + n0, p.ldy);
  tmem_fence_before();
  __syncthreads();
  if (warp == 1) {
    tmem_fence_after();
    tmem_free(tmem, S::kTmem);
  }
}

template <typename G, int COLS, typename X>
cudaError_t launch(const Mx4& a, const MatrixIn* x, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  using S = Shape<COLS, !std::is_void<X>::value>;
  using T = typename std::conditional<std::is_void<X>::value, float, X>::type;
  static Device device;
  const Device::Facts* facts;
  cudaError_t e = device.prepare(matmul_kernel<G, COLS, X>, S::kThreads, S::kSmem, 0, &facts);
  if (e != cudaSuccess) return e;
  Params p = {};
  const uint64_t nb = (b.cols + 31) / 32;
  p.lane_scales = static_cast<const uint8_t*>(b.scales);
  p.column_scales = static_cast<const uint8_t*>(a.scales);
  p.y = y.p;
  p.ldy = y.ld;
  p.m = (uint32_t)y.rows;
  p.n = (uint32_t)y.cols;
  p.k = (uint32_t)b.cols;
  p.kt = (uint32_t)((nb + 3) / 4);
  p.lane_tiles = (p.n + 127) / 128;
  const uint64_t tiles = (uint64_t)p.lane_tiles * ((p.m + COLS - 1) / COLS);
  if (tiles > 0x0FFFFFFFull) return cudaErrorInvalidConfiguration;
  // A stage takes 0.2 us; joining 0.7 us at 16 columns and 2.7 at 128 (one token through 4096 x 4096: 6.6 us by one
  // block a tile, 5.3 by four; 128 tokens: 7.4 and 8.3).
  p.split = pick_split(*facts, tiles, (p.kt + 1) / 2, 2 + COLS / 11);
  CUtensorMap lane_map, column_map = {};
  e = encode_rows(&lane_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, nb * 16, b.rows, nb * 16, 128);
  if (e == cudaSuccess && !x) e = encode_rows(&column_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, nb * 16, a.rows, nb * 16, COLS);
  if (e != cudaSuccess) return e;
  return launch_after(matmul_kernel<G, COLS, X>, (uint32_t)(tiles * p.split), S::kThreads, S::kSmem, p.split, stream, lane_map, column_map, p,
                      x ? Rows<T>::of(x->p, x->rows, x->cols, x->ld, 0) : Rows<T>::of(nullptr, 0, 0, 0, 0));
}

// The narrowest tile that takes all rows, else 128: scale bytes come in atoms of 128 rows, and a tile begins with one.
template <typename G> cudaError_t by_rows(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  if (y.rows <= 16) return launch<G, 16, void>(a, nullptr, b, y, stream);
  if (y.rows <= 32) return launch<G, 32, void>(a, nullptr, b, y, stream);
  if (y.rows <= 64) return launch<G, 64, void>(a, nullptr, b, y, stream);
  return launch<G, 128, void>(a, nullptr, b, y, stream);
}

template <typename G, typename X> cudaError_t quantizing(const MatrixIn& x, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  return launch<G, 16, X>({}, &x, b, y, stream);
}

cudaError_t nothing(const MatrixOut& y, cudaStream_t stream) {   // a sum over nothing
  return cudaMemset2DAsync(y.p, y.ld * (y.type == kBF16 ? 2 : 4), 0, y.cols * (y.type == kBF16 ? 2 : 4), y.rows, stream);
}

// Rows of x up to which the product brings them to MX4 itself, and beyond which that is a launch of its own.  Inside and by
// itself, bf16: 4096 outputs of 9216 inputs, device time of 8, 16 and 32 rows 6.2, 8.8 and 13.8 us and 6.1, 6.4 and 7.3 us, one call
// among others from the host 6.5, 9.2, 14.1 and 7.2, 7.5, 8.3; 4096 of 4096 device 4.9, 6.4, 8.8 and 5.3, 5.5, 6.1, host 5.2, 6.7,
// 9.1 and 7.0, 7.0, 7.2 (two calls into the driver, and a workspace).  Sixteen rows fill the narrowest tile.
constexpr uint64_t kQuantizedInside = 16;

}  // namespace

cudaError_t launch_mx4_matmul(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  if (a.cols == 0) return nothing(y, stream);
  // Pairs once the tiles of single blocks no longer fit the SMs at once (4096 values: 128 tiles of 512 x 4096 8.0 us
  // and 10.2 by pairs, 256 tiles of 1024 x 4096 15.0 and 10.8).
  if (((a.rows + 127) / 128) * ((b.rows + 127) / 128) > kSms) return launch_mx4_matmul_pair(a, b, y, stream);
  return y.type == kBF16 ? by_rows<__nv_bfloat16>(a, b, y, stream) : by_rows<float>(a, b, y, stream);
}

uint64_t mx4_linear_workspace(uint64_t m, uint64_t k) {
  if (m <= kQuantizedInside) return 0;
  return m * ((k + 31) / 32) * 16 + 512 + (m + 127) / 128 * ((k + 127) / 128) * 512;
}

cudaError_t launch_mx4_linear(const MatrixIn& x, const Mx4& b, const MatrixOut& y, void* workspace, cudaStream_t stream) {
  if (x.cols == 0) return nothing(y, stream);
  if (x.rows <= kQuantizedInside) {
    if (y.type == kBF16) return x.type == kBF16 ? quantizing<__nv_bfloat16, __nv_bfloat16>(x, b, y, stream) : quantizing<__nv_bfloat16, float>(x, b, y, stream);
    return x.type == kBF16 ? quantizing<float, __nv_bfloat16>(x, b, y, stream) : quantizing<float, float>(x, b, y, stream);
  }
  uint8_t* codes = static_cast<uint8_t*>(workspace);
  uint8_t* scales = codes + (x.rows * ((x.cols + 31) / 32) * 16 + 511) / 512 * 512;
  const cudaError_t e = launch_mx4_quantize(x, false, codes, scales, stream);
  return e != cudaSuccess ? e : launch_mx4_matmul({codes, scales, x.rows, x.cols}, b, y, stream);
}

cudaError_t mx4_matmul_gave_up(uint32_t* count, cudaStream_t stream) { return read_count(g_gave_up, count, stream); }

}  // namespace rudra
