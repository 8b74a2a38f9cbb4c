// y = a b^T with both matrices in MX4: one output per thread, a block of 32 products at a time through
// shared memory.
#include "blocks.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

__device__ __forceinline__ void stage(const Mx4& m, uint64_t row, uint32_t b, uint32_t part, float* to) {
  const uint32_t nb = (uint32_t)((m.cols + 31) / 32);
  float x[8];
  if (row < m.rows)
    e2m1_values(static_cast<const uint32_t*>(m.codes)[(row * nb + b) * 4 + part],
                scale_value(static_cast<const uint8_t*>(m.scales)[mx4_scale_at(row, b, (nb + 3) / 4)]), x);
#pragma unroll
  for (int e = 0; e < 8; ++e) to[e] = row < m.rows ? x[e] : 0.f;
}

__global__ void __launch_bounds__(256) matmul_kernel(Mx4 a, Mx4 b, MatrixOut y) {
  __shared__ float as[16][33], bs[16][33];
  const uint32_t tiles = (uint32_t)((b.rows + 15) / 16);
  const uint64_t m0 = (uint64_t)(blockIdx.x / tiles) * 16, n0 = (uint64_t)(blockIdx.x % tiles) * 16;
  const uint32_t t = threadIdx.x, i = t / 16, j = t % 16;
  float acc = 0.f;
  for (uint32_t k = 0; k < (a.cols + 31) / 32; ++k) {
    if (t < 64) stage(a, m0 + t / 4, k, t % 4, &as[t / 4][t % 4 * 8]);
    else if (t < 128) stage(b, n0 + (t - 64) / 4, k, t % 4, &bs[(t - 64) / 4][t % 4 * 8]);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 32; ++e) acc = fmaf(as[i][e], bs[j][e], acc);
    __syncthreads();
  }
  const uint64_t m = m0 + i, n = n0 + j;
  if (m < y.rows && n < y.cols) {
    if (y.type == kBF16) static_cast<__nv_bfloat16*>(y.p)[m * y.ld + n] = __float2bfloat16_rn(acc);
    else static_cast<float*>(y.p)[m * y.ld + n] = acc;
  }
}

}  // namespace

cudaError_t launch_mx4_matmul(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream) {
  const uint64_t blocks = ((a.rows + 15) / 16) * ((b.rows + 15) / 16);
  if (blocks > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  matmul_kernel<<<(unsigned)blocks, 256, 0, stream>>>(a, b, y);
  return cudaGetLastError();
}

}  // namespace rudra
