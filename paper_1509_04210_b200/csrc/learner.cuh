// Launch interface between the exported learner-side operators and their sm_100a kernels.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kernels.cuh"

namespace rudra {

constexpr uint64_t kBlock = 32;   // values that share a scale, in MX4 and ACT8

// A row-major matrix; ld in elements.
struct MatrixIn {
  const void* p;
  GradType type;
  uint64_t rows, cols, ld;
};
struct MatrixOut {
  void* p;
  GradType type;
  uint64_t rows, cols, ld;
};
// A matrix in MX4: rows of 16 * ceil(cols / 32) bytes of codes, scale bytes in the tensor cores' order.
struct Mx4 {
  const void* codes;
  const void* scales;
  uint64_t rows, cols;
};
// A checkpoint: rows of 32 * ceil(cols / 32) int8 codes, rows of act8_scale_pitch(cols) scale bytes.
struct Act8 {
  void* codes;
  void* scales;
};
// Whole 16-byte pieces, which TMA can read.
inline uint64_t act8_scale_pitch(uint64_t cols) { return (cols + 511) / 512 * 16; }

enum Act : int { kNone = 0, kRelu = 1, kSilu = 2, kGelu = 3, kSwiglu = 4 };   // RUDRA_ACT_*

// All of them: sizes are not zero, arguments have been checked.
cudaError_t launch_mx4_quantize(const MatrixIn& src, bool transpose, void* codes, void* scales, cudaStream_t stream);
cudaError_t launch_mx4_dequantize(const Mx4& src, const MatrixOut& dst, cudaStream_t stream);
cudaError_t launch_mx4_matmul(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream);
cudaError_t launch_mx4_matmul_pair(const Mx4& a, const Mx4& b, const MatrixOut& y, cudaStream_t stream);   // of launch_mx4_matmul: many tiles
uint64_t mx4_linear_workspace(uint64_t m, uint64_t k);
cudaError_t launch_mx4_linear(const MatrixIn& x, const Mx4& b, const MatrixOut& y, void* workspace, cudaStream_t stream);
cudaError_t launch_act8_forward(Act act, const MatrixIn& x, const void* up, const MatrixOut& y, const Act8& saved,
                                const Act8& saved_up, cudaStream_t stream);
cudaError_t launch_act8_backward(Act act, const MatrixIn& dy, const Act8& saved, const Act8& saved_up,
                                 const MatrixOut& dx, void* dup, cudaStream_t stream);
uint64_t act8_weight_grad_workspace(const MatrixIn& dy);
cudaError_t launch_act8_weight_grad(const MatrixIn& dy, const Act8& saved, const MatrixOut& dw, void* workspace,
                                    cudaStream_t stream);

// A count that goes up where a kernel of the file gives up a wait, as the stream's work leaves it; there once the stream is done.
cudaError_t mx4_matmul_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t mx4_matmul_pair_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t act8_weight_grad_gave_up(uint32_t* count, cudaStream_t stream);

}  // namespace rudra
