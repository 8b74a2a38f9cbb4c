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
// A matrix in FP8: rows of 128 * ceil(cols / 128) bytes of codes, scale bytes in the tensor cores' order.
struct Fp8 {
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
cudaError_t launch_fp8_quantize(const MatrixIn& src, bool transpose, bool square, void* codes, void* scales, cudaStream_t stream);
cudaError_t launch_fp8_dequantize(const Fp8& src, const MatrixOut& dst, cudaStream_t stream);
cudaError_t launch_fp8_matmul(const Fp8& a, const Fp8& b, const MatrixOut& y, cudaStream_t stream);
// Of launch_fp8_matmul: many tiles; `count` blocks of 128 values from block `begin` on, added to y unless that is the first.  bf16 results
// have all blocks, in sums of `one_sum` (a multiple of four) that are gathered.
cudaError_t launch_fp8_matmul_pair(const Fp8& a, const Fp8& b, const MatrixOut& y, uint32_t begin, uint32_t count, uint32_t one_sum, cudaStream_t stream);
uint64_t fp8_linear_workspace(uint64_t m, uint64_t k);
cudaError_t launch_fp8_linear(const MatrixIn& x, const Fp8& b, const MatrixOut& y, void* workspace, cudaStream_t stream);

// Root-mean-square norm.  Matrices without memory (p null) are not given or not wanted; all have x's shape and type.
struct NormForward {
  MatrixIn x, residual;
  const void* weight;          // one for each column
  GradType weight_type;
  float eps;
  MatrixOut sum, y;
  Act8 fp8, kept;              // y in FP8, and in ACT8
};
cudaError_t launch_rms_norm(const NormForward& n, cudaStream_t stream);
struct NormBackward {
  MatrixIn dy, s, dsum;
  const void* weight;
  GradType weight_type;
  float eps;
  MatrixOut ds;                // may be dy's memory, or dsum's
  void* dw;
  GradType dw_type;
};
uint64_t rms_norm_backward_workspace(uint64_t rows, uint64_t cols);
cudaError_t launch_rms_norm_backward(const NormBackward& n, void* workspace, cudaStream_t stream);

// A list of gradients, each `size` values one after another.
struct Gradient {
  const void* p;
  void* out;                   // of grad_clip; may be p
  uint64_t size;
  GradType type, out_type;
};
uint64_t grad_norm_workspace(uint64_t count);
cudaError_t launch_grad_norm(const Gradient* grads, uint64_t count, float* norm, void* workspace, cudaStream_t stream);
// known: *norm is the norm; otherwise it is computed, left there, and the workspace needed.
cudaError_t launch_grad_clip(const Gradient* grads, uint64_t count, float* norm, float max_norm, bool known, void* workspace, cudaStream_t stream);

// A count that goes up where a kernel of the file gives up a wait, as the stream's work leaves it; there once the stream is done.
cudaError_t mx4_matmul_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t mx4_matmul_pair_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t act8_weight_grad_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t fp8_matmul_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t fp8_matmul_pair_gave_up(uint32_t* count, cudaStream_t stream);
cudaError_t rms_norm_gave_up(uint32_t* count, cudaStream_t stream);
// Where it lies on the current device.
cudaError_t mx4_matmul_count(const uint32_t** at);
cudaError_t mx4_matmul_pair_count(const uint32_t** at);
cudaError_t act8_weight_grad_count(const uint32_t** at);
cudaError_t fp8_matmul_count(const uint32_t** at);
cudaError_t fp8_matmul_pair_count(const uint32_t** at);
cudaError_t rms_norm_count(const uint32_t** at);

}  // namespace rudra
