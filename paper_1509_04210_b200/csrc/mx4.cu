// Microscaled 4-bit floating point: quantization (as a matrix stands, or its transpose) and expansion.
//
// A block's scale is a power of two read off the exponent field of its largest magnitude, so scaling
// is exact and the only rounding is the one to E2M1, done by the conversion instruction.  One read and
// 17/32 byte written per value: bound by HBM for large matrices, by launch latency for small ones.
#include "blocks.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

constexpr int kThreads = 256;

// Rows as they stand.  16 lanes take 128 values of a row, i.e. four blocks and one word of scale bytes.
template <typename G>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const G* __restrict__ src, uint64_t ld, uint32_t cols,
                                                                 uint32_t kt, uint64_t items, bool wide,
                                                                 uint32_t* __restrict__ codes, uint32_t* __restrict__ scales) {
  constexpr int U = 2;
  const uint32_t lane = threadIdx.x % 16;
  const uint32_t nb = (cols + 31) / 32;
  float x[U][8];
  uint64_t row[U];
  uint32_t k[U], c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint64_t item = (uint64_t)blockIdx.x * (U * kThreads / 16) + u * (kThreads / 16) + threadIdx.x / 16;
    const bool in = item < items;
    row[u] = in ? (uint32_t)item / kt : ~0ull;   // items < 2^32
    k[u] = (uint32_t)item % kt;
    c[u] = k[u] * 128 + lane * 8;
    const int have = in && c[u] < cols ? (int)min(8u, cols - c[u]) : 0;
    load8(src + (have ? row[u] * ld + c[u] : 0), wide && have == 8, have, x[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t s = scale_byte(block_max_bits(max_bits(x[u])), 2);
    const uint32_t w = e2m1_codes(x[u], inverse_scale(s));
    uint32_t four = s << (8 * (lane / 4));
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 4);
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 8);
    if (row[u] == ~0ull) continue;
    if (c[u] / 32 < nb) codes[row[u] * nb * 4 + c[u] / 8] = w;
    if (lane == 0) scales[mx4_scale_at(row[u], k[u] * 4, kt) / 4] = four;
  }
}

// The transpose: a column of src is a row of the result.  A warp takes 32 rows x 64 columns, a lane two
// columns of 32 values each, so that a block lies in one thread; four warps take the four blocks that
// share a word of scale bytes, and the codes go through shared memory to leave as 64-byte rows.
template <typename G>
__global__ void __launch_bounds__(128) quantize_transposed_kernel(const G* __restrict__ src, uint64_t ld, uint32_t rows,
                                                                  uint32_t cols, uint32_t column_tiles, bool pairs,
                                                                  uint4* __restrict__ codes, uint32_t* __restrict__ scales) {
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
          const float2 v = *reinterpret_cast<const float2*>(p);
          x[0][i] = v.x;
          x[1][i] = v.y;
        } else {
          const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
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
    float(&v)[4][8] = reinterpret_cast<float(&)[4][8]>(x[j]);
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) m = max(m, max_bits(v[q]));
    const uint32_t s = scale_byte(m, 2);
    const float inv = inverse_scale(s);
    tile[lane * 2 + j][warp] = make_uint4(e2m1_codes(v[0], inv), e2m1_codes(v[1], inv), e2m1_codes(v[2], inv), e2m1_codes(v[3], inv));
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

template <typename G>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                              uint32_t cols, uint32_t kt, uint64_t units, bool wide,
                                                              G* __restrict__ dst, uint64_t ld) {
  const uint32_t per_row = (cols + 7) / 8, nb = (cols + 31) / 32;
  const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= units) return;
  const uint64_t row = i / per_row;
  const uint32_t unit = (uint32_t)(i - row * per_row), c = unit * 8;
  const int have = (int)min(8u, cols - c);
  float x[8];
  e2m1_values(codes[row * nb * 4 + unit], scale_value(scales[mx4_scale_at(row, c / 32, kt)]), x);
  store8(dst + row * ld + c, wide && have == 8, have, x);
}

cudaError_t grid_of(uint64_t work, uint64_t per_block, unsigned* blocks) {
  const uint64_t b = (work + per_block - 1) / per_block;
  if (b > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  *blocks = (unsigned)b;
  return cudaSuccess;
}

template <typename G>
cudaError_t quantize(const MatrixIn& m, bool transpose, void* codes, void* scales, cudaStream_t stream) {
  const G* src = static_cast<const G*>(m.p);
  unsigned blocks;
  if (!transpose) {
    const uint64_t kt = (m.cols + 127) / 128, items = m.rows * kt;
    if (items > 0xFFFFFFFFull) return cudaErrorInvalidConfiguration;
    const cudaError_t e = grid_of(items, 2 * kThreads / 16, &blocks);
    if (e != cudaSuccess) return e;
    quantize_rows_kernel<G><<<blocks, kThreads, 0, stream>>>(src, m.ld, (uint32_t)m.cols, (uint32_t)kt, items, wide_rows<G>(src, m.ld),
                                                             static_cast<uint32_t*>(codes), static_cast<uint32_t*>(scales));
  } else {
    const uint64_t tiles = (m.cols + 63) / 64;
    const cudaError_t e = grid_of(tiles * ((m.rows + 127) / 128), 1, &blocks);
    if (e != cudaSuccess) return e;
    const bool pairs = reinterpret_cast<uintptr_t>(src) % (2 * sizeof(G)) == 0 && m.ld % 2 == 0;
    quantize_transposed_kernel<G><<<blocks, 128, 0, stream>>>(src, m.ld, (uint32_t)m.rows, (uint32_t)m.cols, (uint32_t)tiles, pairs,
                                                              static_cast<uint4*>(codes), static_cast<uint32_t*>(scales));
  }
  return cudaGetLastError();
}

template <typename G>
cudaError_t dequantize(const Mx4& m, const MatrixOut& d, cudaStream_t stream) {
  const uint64_t units = m.rows * ((m.cols + 7) / 8), kt = (m.cols + 127) / 128;
  unsigned blocks;
  const cudaError_t e = grid_of(units, kThreads, &blocks);
  if (e != cudaSuccess) return e;
  dequantize_kernel<G><<<blocks, kThreads, 0, stream>>>(static_cast<const uint32_t*>(m.codes), static_cast<const uint8_t*>(m.scales),
                                                        (uint32_t)m.cols, (uint32_t)kt, units, wide_rows<G>(d.p, d.ld), static_cast<G*>(d.p), d.ld);
  return cudaGetLastError();
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
