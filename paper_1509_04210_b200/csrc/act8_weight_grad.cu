// dw = dy^T xhat with xhat from an 8-bit checkpoint: one output per thread, 32 tokens at a time through
// shared memory.
#include "blocks.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

__global__ void __launch_bounds__(256) weight_grad_kernel(MatrixIn dy, Act8 saved, MatrixOut dw) {
  __shared__ float gs[32][17], xs[32][17];
  const uint32_t tiles = (uint32_t)((dw.cols + 15) / 16);
  const uint64_t n0 = (uint64_t)(blockIdx.x / tiles) * 16, k0 = (uint64_t)(blockIdx.x % tiles) * 16;
  const uint64_t nb = (dw.cols + 31) / 32;
  const uint32_t i = threadIdx.x / 16, j = threadIdx.x % 16;
  float acc = 0.f;
  for (uint64_t t0 = 0; t0 < dy.rows; t0 += 32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t t = t0 + h * 16 + i;
      float g = 0.f, x = 0.f;
      if (t < dy.rows) {
        if (n0 + j < dy.cols)
          g = dy.type == kBF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(dy.p)[t * dy.ld + n0 + j])
                               : static_cast<const float*>(dy.p)[t * dy.ld + n0 + j];
        if (k0 + j < dw.cols)
          x = (float)static_cast<const int8_t*>(saved.codes)[t * nb * 32 + k0 + j] *
              scale_value(static_cast<const uint8_t*>(saved.scales)[t * nb + (k0 + j) / 32]);
      }
      gs[h * 16 + i][j] = g;
      xs[h * 16 + i][j] = x;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 32; ++e) acc = fmaf(gs[e][i], xs[e][j], acc);
    __syncthreads();
  }
  const uint64_t n = n0 + i, k = k0 + j;
  if (n < dw.rows && k < dw.cols) {
    if (dw.type == kBF16) static_cast<__nv_bfloat16*>(dw.p)[n * dw.ld + k] = __float2bfloat16_rn(acc);
    else static_cast<float*>(dw.p)[n * dw.ld + k] = acc;
  }
}

}  // namespace

uint64_t act8_weight_grad_workspace(const MatrixIn&) { return 0; }

cudaError_t launch_act8_weight_grad(const MatrixIn& dy, const Act8& saved, const MatrixOut& dw, void*, cudaStream_t stream) {
  const uint64_t blocks = ((dw.rows + 15) / 16) * ((dw.cols + 15) / 16);
  if (blocks > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  weight_grad_kernel<<<(unsigned)blocks, 256, 0, stream>>>(dy, saved, dw);
  return cudaGetLastError();
}

}  // namespace rudra
