// Microscaled 4-bit floating point: quantization (as a matrix stands, or its transpose) and expansion.
//
// A block's scale is a power of two read off the exponent field of its largest magnitude, so scaling
// is exact and the only rounding is the one to E2M1, done by the conversion instruction.  One read and
// 17/32 byte written per value: bound by HBM for large matrices, by launch latency for small ones.  Measured:
// 4096 x 9216 floats 28.0 us = 6.1 TB/s, transposed 34.0 us = 5.0 TB/s (a thread holds 64 values, so fewer are on
// their way), expanded to bf16 13.6 us = 7.0 TB/s; 4 x 4096 bf16 1.9 us.
#include <algorithm>

#include "blocks.cuh"
#include "launch.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

constexpr int kThreads = 256;

// Rows as they stand.  Eight lanes take 128 values of a row, i.e. four blocks and one word of scale bytes.
template <typename G, bool ANY>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(Rows<G> src, uint32_t cols, Divisor kt, uint32_t items,
                                                                 uint2* codes, uint32_t* scales) {
  constexpr uint32_t U = 2, kItems = kThreads / 8;
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t lane = threadIdx.x % 8, nb = (cols + 31) / 32;
  Values<G> x[U];
  uint32_t row[U], k[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t item = blockIdx.x * (U * kItems) + u * kItems + threadIdx.x / 8;
    row[u] = kt.quotient(item);
    k[u] = item - row[u] * kt.d;
    const uint32_t c = k[u] * 128 + lane * kValues;
    const int have = item < items && c < cols ? (int)min((uint32_t)kValues, cols - c) : 0;
    x[u].template load<ANY, true>(src, have ? row[u] * src.ld + c : 0, have);
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t s = scale_byte(block_max_bits(x[u].max_bits()), 2);
    const uint2 w = e2m1_codes(x[u], s);
    uint32_t four = s << (8 * (lane / 2));
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 2);
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 4);
    if (blockIdx.x * (U * kItems) + u * kItems + threadIdx.x / 8 >= items) continue;
    if (k[u] * 4 + lane / 2 < nb) codes[(uint64_t)row[u] * nb * 2 + k[u] * 8 + lane] = w;
    if (lane == 0) scales[mx4_scale_at(row[u], k[u] * 4, kt.d) / 4] = four;
  }
}

// The transpose: a column of src is a row of the result.  A warp takes 32 rows x 64 columns, a lane two
// columns of 32 values each, so that a block lies in one thread; four warps take the four blocks that
// share a word of scale bytes, and the codes go through shared memory to leave as 64-byte rows.
template <typename G>
__global__ void __launch_bounds__(128) quantize_transposed_kernel(const G* src, uint64_t ld, uint32_t rows,
                                                                  uint32_t cols, uint32_t column_tiles, bool pairs,
                                                                  uint4* codes, uint32_t* scales) {
  admit_next_kernel();
  await_previous_kernel();
  __shared__ uint4 tile[64][5];
  __shared__ uint8_t sbytes[64][4];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t k = blockIdx.x / column_tiles;             // 128 values of a result row
  const uint32_t c0 = (blockIdx.x % column_tiles) * 64;
  const uint32_t c = c0 + lane * 2, r0 = k * 128 + warp * 32;
  const uint32_t nb = (rows + 31) / 32, kt = (nb + 3) / 4;
  float x[2][32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint64_t r = (uint64_t)r0 + i;
    x[0][i] = x[1][i] = 0.f;
    if (r < rows) {
      const G* p = src + r * ld + c;
      if (pairs && c + 1 < cols) {
        if (sizeof(G) == 4) {
          const uint2 v = read_once(reinterpret_cast<const uint2*>(p));
          x[0][i] = __uint_as_float(v.x);
          x[1][i] = __uint_as_float(v.y);
        } else {
          const uint32_t v = read_once(reinterpret_cast<const uint32_t*>(p));
          x[0][i] = __uint_as_float(v << 16);
          x[1][i] = __uint_as_float(v & 0xFFFF0000u);
        }
      } else {
        if (c < cols) x[0][i] = (float)p[0];
        if (c + 1 < cols) x[1][i] = (float)p[1];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    Values<float> v[2];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i / kValues].w[i % kValues] = __float_as_uint(x[j][i]);
    const uint32_t s = scale_byte(max(v[0].max_bits(), v[1].max_bits()), 2);
    const uint2 lo = e2m1_codes(v[0], s), hi = e2m1_codes(v[1], s);
    tile[lane * 2 + j][warp] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    sbytes[lane * 2 + j][warp] = (uint8_t)s;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t t = threadIdx.x + 128 * j, row = c0 + t / 4, b = k * 4 + t % 4;
    if (row < cols && b < nb) codes[(uint64_t)row * nb + b] = tile[t / 4][t % 4];
  }
  const uint32_t row = c0 + threadIdx.x;
  if (threadIdx.x < 64 && row < cols)
    scales[mx4_scale_at(row, (uint64_t)k * 4, kt) / 4] = *reinterpret_cast<const uint32_t*>(sbytes[threadIdx.x]);
}

// codes and dst from a launch's first row on, scales of the whole matrix.
template <typename G, bool ANY>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const uint2* codes, const uint8_t* scales,
                                                              uint32_t first_row, uint32_t cols, Divisor per_row, uint32_t kt, uint32_t units, Access access,
                                                              G* dst, uint64_t ld) {
  constexpr uint32_t U = 2;
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t nb = (cols + 31) / 32;
  uint2 w[U];
  uint32_t s[U], row[U], c[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t i = (blockIdx.x * U + u) * kThreads + threadIdx.x;
    row[u] = per_row.quotient(i);
    c[u] = (i - row[u] * per_row.d) * kValues;
    if (i < units) {
      w[u] = read_once(codes + (uint64_t)row[u] * nb * 2 + c[u] / kValues);
      s[u] = read_byte(scales + mx4_scale_at(first_row + row[u], c[u] / 32, kt));
    }
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const bool in = (blockIdx.x * U + u) * kThreads + threadIdx.x < units;
    const int have = in ? (int)min((uint32_t)kValues, cols - c[u]) : 0;
    float x[kValues] = {};
    if (in) e2m1_values(w[u], scale_value(s[u]), x);
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

template <typename G>
cudaError_t quantize(const MatrixIn& m, bool transpose, void* codes, void* scales, cudaStream_t stream) {
  const G* src = static_cast<const G*>(m.p);
  if (!transpose) {
    // as many rows to a launch as keep the count of its work below 2^31
    const uint64_t kt = (m.cols + 127) / 128, most = std::max<uint64_t>(1, 0x70000000ull / kt / 128) * 128;
    for (uint64_t r = 0; r < m.rows; r += most) {
      const uint64_t rows = std::min(most, m.rows - r);
      if (rows * kt > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
      const cudaError_t e = launch_after(
          access_of<G>(m.p, m.ld) == kByElement ? quantize_rows_kernel<G, true> : quantize_rows_kernel<G, false>, grid_of(rows * kt, 2 * kThreads / 8), kThreads, 0, 1, stream,
          Rows<G>::of(m.p, m.rows, m.cols, m.ld, r), (uint32_t)m.cols, Divisor((uint32_t)kt), (uint32_t)(rows * kt), static_cast<uint2*>(codes) + r * ((m.cols + 31) / 32) * 2,
          static_cast<uint32_t*>(scales) + mx4_scale_at(r, 0, kt) / 4);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  const uint64_t tiles = (m.cols + 63) / 64, blocks = tiles * ((m.rows + 127) / 128);
  if (blocks > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  const bool pairs = reinterpret_cast<uintptr_t>(src) % (2 * sizeof(G)) == 0 && m.ld % 2 == 0;
  return launch_after(quantize_transposed_kernel<G>, (uint32_t)blocks, 128, 0, 1, stream, src, m.ld, (uint32_t)m.rows, (uint32_t)m.cols,
                      (uint32_t)tiles, pairs, static_cast<uint4*>(codes), static_cast<uint32_t*>(scales));
}

template <typename G>
cudaError_t dequantize(const Mx4& m, const MatrixOut& d, cudaStream_t stream) {
  const uint64_t per_row = (m.cols + kValues - 1) / kValues, nb = (m.cols + 31) / 32, kt = (m.cols + 127) / 128;
  const uint64_t most = 0x70000000ull / per_row;   // rows of a launch, 14 or more: the count of its work stays below 2^31
  for (uint64_t r = 0; r < m.rows; r += most) {
    const uint64_t units = std::min(most, m.rows - r) * per_row;
    const cudaError_t e = launch_after(
        access_of<G>(d.p, d.ld) == kByElement ? dequantize_kernel<G, true> : dequantize_kernel<G, false>, grid_of(units, 2 * kThreads), kThreads, 0, 1, stream,
        static_cast<const uint2*>(m.codes) + r * nb * 2, static_cast<const uint8_t*>(m.scales), (uint32_t)r, (uint32_t)m.cols, Divisor((uint32_t)per_row), (uint32_t)kt,
        (uint32_t)units, access_of<G>(d.p, d.ld), static_cast<G*>(d.p) + r * d.ld, d.ld);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_mx4_quantize(const MatrixIn& src, bool transpose, void* codes, void* scales, cudaStream_t stream) {
  return src.type == kBF16 ? quantize<__nv_bfloat16>(src, transpose, codes, scales, stream)
                           : quantize<float>(src, transpose, codes, scales, stream);
}

cudaError_t launch_mx4_dequantize(const Mx4& src, const MatrixOut& dst, cudaStream_t stream) {
  return dst.type == kBF16 ? dequantize<__nv_bfloat16>(src, dst, stream) : dequantize<float>(src, dst, stream);
}

}  // namespace rudra
