// 8-bit floating point in blocks of 128: quantization of a matrix or its transpose, by pieces of rows or by squares, and
// expansion.
//
// A block's scale is a power of two read off its largest magnitude, so scaling is exact and the only rounding is the one
// to E4M3, done by the conversion instruction.  One read and 129/128 bytes written per value: bound by HBM for large
// matrices, by launch latency for small ones.  Measured: rows of 8192 x 9216 bf16 35.7 us and of 4096 x 9216 f32 29.6 us = 6.4 TB/s,
// expanded 35.1 and 29.5 us; 8192 x 4096 bf16 transposed 19.6 us = 5.1 TB/s (256-byte pieces of rows), 4096 x 9216 f32 by squares
// 25.5 and transposed 26.6 us (partly out of L2); 4 x 4096 bf16 2.6 us.
#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "pairs.cuh"

namespace rudra {
namespace {

constexpr int kThreads = 256;

// Rows as they stand: eight lanes take a block.  `scales` from the launch's first row on, a multiple of 128.
template <typename G, bool ANY>
__global__ void __launch_bounds__(kThreads) fp8_rows_kernel(Rows<G> src, uint32_t cols, Divisor per_row, uint32_t kt, uint32_t items, uint4* codes,
                                                            uint8_t* scales) {
  constexpr uint32_t U = 2, kItems = kThreads / 8;
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t lane = threadIdx.x % 8, nb = per_row.d;
  Values<G> x[U];
  uint32_t row[U], b[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t item = blockIdx.x * (U * kItems) + u * kItems + threadIdx.x / 8;
    row[u] = per_row.quotient(item);
    b[u] = item - row[u] * nb;
    const uint32_t c = b[u] * kFp8Block + lane * kValues;
    const int have = item < items && c < cols ? (int)min((uint32_t)kValues, cols - c) : 0;
    x[u].template load<ANY, true>(src, have ? row[u] * src.ld + c : 0, have);
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t item = blockIdx.x * (U * kItems) + u * kItems + threadIdx.x / 8;
    const uint32_t s = fp8_scale_byte(fp8_block_max_bits(x[u].max_bits()));
    const uint4 w = e4m3_codes([&](int i) { return x[u].get(i); }, s);
    if (item >= items) continue;
    codes[(uint64_t)item * 8 + lane] = w;
    if (lane == 0) put_fp8_scale(scales, row[u], b[u], nb, kt, s);
  }
}

// A tile of 128 x 128 values of src: as a square with one scale, or with a scale for each of its columns, which are rows
// of the result.  A warp takes 16 whole rows of it, a lane 16 values of each of four columns: neighbouring ones where four values can be
// read at once (QUADS), else every 32nd; maxima and codes meet in shared memory, from which the codes leave as rows of 128 bytes.
template <typename G, bool TRANSPOSE, bool SQUARE, bool QUADS>
__global__ void __launch_bounds__(kThreads, 3) fp8_tile_kernel(const G* src, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t column_tiles, uint8_t* codes,
                                                            uint8_t* scales) {
  static_assert(TRANSPOSE || SQUARE, "pieces of rows have a kernel of their own");
  constexpr uint32_t kPitch = kFp8Block + 16, kRows = 16;
  __shared__ alignas(16) uint8_t tile[kFp8Block * kPitch];
  __shared__ uint32_t top[SQUARE ? 1 : kFp8Block];
  admit_next_kernel();
  const uint32_t lane = threadIdx.x % 32, rl = threadIdx.x / 32 * kRows;
  const uint32_t r0 = blockIdx.x / column_tiles * kFp8Block, c0 = blockIdx.x % column_tiles * kFp8Block;
  const auto column = [&](uint32_t j) { return QUADS ? 4 * lane + j : lane + 32 * j; };
  if (threadIdx.x < (SQUARE ? 1 : kFp8Block)) top[threadIdx.x] = 0;
  await_previous_kernel();
  // all on their way before the first is looked at: a value used in the branch that loads it would hold up the next load
  // (509 x 4096 bf16 19.6 us that way)
  float x[4][kRows];
  if (QUADS && c0 + 4 * lane + 3 < cols) {
    using Word = typename std::conditional<sizeof(G) == 4, uint4, uint2>::type;
    Word raw[kRows];
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) {
      const uint64_t r = (uint64_t)r0 + rl + i;
      raw[i] = r < rows ? read_once(reinterpret_cast<const Word*>(src + r * ld + c0 + 4 * lane)) : Word{};
    }
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) {
      if constexpr (sizeof(G) == 4) {
        x[0][i] = __uint_as_float(raw[i].x);
        x[1][i] = __uint_as_float(raw[i].y);
        x[2][i] = __uint_as_float(raw[i].z);
        x[3][i] = __uint_as_float(raw[i].w);
      } else {
        x[0][i] = __uint_as_float(raw[i].x << 16);
        x[1][i] = __uint_as_float(raw[i].x & 0xFFFF0000u);
        x[2][i] = __uint_as_float(raw[i].y << 16);
        x[3][i] = __uint_as_float(raw[i].y & 0xFFFF0000u);
      }
    }
  } else {
    G raw[4][kRows];
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i)
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const uint64_t r = (uint64_t)r0 + rl + i, c = (uint64_t)c0 + column(j);
        raw[j][i] = r < rows && c < cols ? src[r * ld + c] : G(0.f);
      }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
      for (uint32_t i = 0; i < kRows; ++i) x[j][i] = (float)raw[j][i];
  }
  float m[4];
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    m[j] = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) m[j] = larger(m[j], x[j][i]);
  }
  __syncthreads();
  if (SQUARE) {
    const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(larger(larger(m[0], m[1]), larger(m[2], m[3]))));
    if (lane == 0) atomicMax(top, most);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) atomicMax(top + column(j), __float_as_uint(m[j]));
  }
  __syncthreads();
  uint32_t keep[4];      // no bits of what stands for NaN as a whole
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t s = fp8_scale_byte(top[SQUARE ? 0 : column(j)]);
    const float inv = inverse_scale(s);
    keep[j] = s == 255u ? 0u : 0xFFFFFFFFu;
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) x[j][i] *= inv;
  }
  if (TRANSPOSE) {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      uint32_t w[4];
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) w[q] = e4m3_codes4(x[j][4 * q], x[j][4 * q + 1], x[j][4 * q + 2], x[j][4 * q + 3]) & keep[j];
      *reinterpret_cast<uint4*>(tile + column(j) * kPitch + rl) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {      // one scale for all
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) {
      const uint32_t w = e4m3_codes4(x[0][i], x[1][i], x[2][i], x[3][i]) & keep[0];
      if (QUADS) {
        *reinterpret_cast<uint32_t*>(tile + (rl + i) * kPitch + 4 * lane) = w;
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) tile[(rl + i) * kPitch + column(j)] = (uint8_t)(w >> 8 * j);
      }
    }
  }
  __syncthreads();
  // rows and blocks of the result
  const uint32_t first = TRANSPOSE ? c0 : r0, all = TRANSPOSE ? cols : rows, length = TRANSPOSE ? rows : cols;
  const uint32_t b = (TRANSPOSE ? r0 : c0) / kFp8Block, nb = (length + kFp8Block - 1) / kFp8Block;
#pragma unroll
  for (uint32_t j = 0; j < kFp8Block * 8 / kThreads; ++j) {
    const uint32_t t = threadIdx.x + kThreads * j, row = first + t / 8;
    if (row < all) *reinterpret_cast<uint4*>(codes + ((uint64_t)row * nb + b) * kFp8Block + t % 8 * 16) = *reinterpret_cast<const uint4*>(tile + t / 8 * kPitch + t % 8 * 16);
  }
  const uint32_t row = first + threadIdx.x;
  if (threadIdx.x < kFp8Block && row < all) put_fp8_scale(scales, row, b, nb, (nb + 3) / 4, fp8_scale_byte(top[SQUARE ? 0 : threadIdx.x]));
}

// codes and dst from a launch's first row on, scales of the whole matrix.
template <typename G, bool ANY>
__global__ void __launch_bounds__(kThreads) fp8_values_kernel(const uint4* codes, const uint8_t* scales, uint32_t first_row, uint32_t cols, Divisor per_row,
                                                              uint32_t units, Access access, G* dst, uint64_t ld) {
  constexpr uint32_t U = 2;
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t nb = (cols + kFp8Block - 1) / kFp8Block, kt = (nb + 3) / 4;
  uint4 w[U];
  uint32_t s[U], row[U], c[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t i = (blockIdx.x * U + u) * kThreads + threadIdx.x;
    row[u] = per_row.quotient(i);
    c[u] = (i - row[u] * per_row.d) * kValues;
    if (i < units) {
      w[u] = read_once(codes + (uint64_t)row[u] * nb * 8 + c[u] / kValues);
      s[u] = read_byte(scales + mx4_scale_at((uint64_t)first_row + row[u], c[u] / kFp8Block, kt));
    }
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const bool in = (blockIdx.x * U + u) * kThreads + threadIdx.x < units;
    const int have = in ? (int)min((uint32_t)kValues, cols - c[u]) : 0;
    float x[kValues] = {};
    if (in) e4m3_values(w[u], scale_value(s[u]), x);
    G* const to = dst + (in ? row[u] * ld + c[u] : 0);
    if constexpr (ANY) {
      __shared__ Meeting meeting[kThreads / 32];
      store_values_anyhow(meeting[threadIdx.x / 32], to, have, x);
    } else {
      store_values(to, access, have, x);
    }
  }
}

unsigned grid_of(uint64_t work, uint64_t per_block) { return (unsigned)((work + per_block - 1) / per_block); }

template <typename G> cudaError_t quantize(const MatrixIn& m, bool transpose, bool square, void* codes, void* scales, cudaStream_t stream) {
  if (!transpose && !square) {
    // as many rows to a launch as keep the count of its work below 2^31; scale bytes come by 128 rows
    const uint64_t nb = (m.cols + kFp8Block - 1) / kFp8Block, kt = (nb + 3) / 4, most = std::max<uint64_t>(1, 0x70000000ull / nb / 128) * 128;
    for (uint64_t r = 0; r < m.rows; r += most) {
      const uint64_t rows = std::min(most, m.rows - r);
      if (rows * nb > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
      const cudaError_t e = launch_overlapped(
          access_of<G>(m.p, m.ld) == kByElement ? fp8_rows_kernel<G, true> : fp8_rows_kernel<G, false>, grid_of(rows * nb, 2 * kThreads / 8), kThreads, 0, 1, stream,
          Rows<G>::of(m.p, m.rows, m.cols, m.ld, r), (uint32_t)m.cols, Divisor((uint32_t)nb), (uint32_t)kt, (uint32_t)(rows * nb), static_cast<uint4*>(codes) + r * nb * 8,
          static_cast<uint8_t*>(scales) + mx4_scale_at(r, 0, kt));
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  const uint64_t tiles = (m.cols + kFp8Block - 1) / kFp8Block, blocks = tiles * ((m.rows + kFp8Block - 1) / kFp8Block);
  if (blocks > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  const bool quads = reinterpret_cast<uintptr_t>(m.p) % (4 * sizeof(G)) == 0 && m.ld % 4 == 0;
  const auto kernel = !transpose ? quads ? fp8_tile_kernel<G, false, true, true> : fp8_tile_kernel<G, false, true, false>
                      : square ? quads ? fp8_tile_kernel<G, true, true, true> : fp8_tile_kernel<G, true, true, false>
                               : quads ? fp8_tile_kernel<G, true, false, true> : fp8_tile_kernel<G, true, false, false>;
  return launch_overlapped(kernel, (uint32_t)blocks, kThreads, 0, 1, stream, static_cast<const G*>(m.p), m.ld, (uint32_t)m.rows, (uint32_t)m.cols, (uint32_t)tiles,
                           static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
}

template <typename G> cudaError_t dequantize(const Fp8& m, const MatrixOut& d, cudaStream_t stream) {
  const uint64_t per_row = (m.cols + kValues - 1) / kValues, nb = (m.cols + kFp8Block - 1) / kFp8Block;
  const uint64_t most = 0x70000000ull / per_row;   // rows of a launch, 14 or more: the count of its work stays below 2^31
  for (uint64_t r = 0; r < m.rows; r += most) {
    const uint64_t units = std::min(most, m.rows - r) * per_row;
    const cudaError_t e = launch_overlapped(
        access_of<G>(d.p, d.ld) == kByElement ? fp8_values_kernel<G, true> : fp8_values_kernel<G, false>, grid_of(units, 2 * kThreads), kThreads, 0, 1, stream,
        static_cast<const uint4*>(m.codes) + r * nb * 8, static_cast<const uint8_t*>(m.scales), (uint32_t)r, (uint32_t)m.cols, Divisor((uint32_t)per_row), (uint32_t)units,
        access_of<G>(d.p, d.ld), static_cast<G*>(d.p) + r * d.ld, d.ld);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_fp8_quantize(const MatrixIn& src, bool transpose, bool square, void* codes, void* scales, cudaStream_t stream) {
  return src.type == kBF16 ? quantize<__nv_bfloat16>(src, transpose, square, codes, scales, stream) : quantize<float>(src, transpose, square, codes, scales, stream);
}

cudaError_t launch_fp8_dequantize(const Fp8& src, const MatrixOut& dst, cudaStream_t stream) {
  return dst.type == kBF16 ? dequantize<__nv_bfloat16>(src, dst, stream) : dequantize<float>(src, dst, stream);
}

}  // namespace rudra
