// The exported learner-side operators: argument checks, and the launches behind them.
#include <cstdint>

#include "../../include/rudra_learner.h"
#include "host.h"
#include "learner.cuh"
#include "reports.h"

namespace {

using rudra::Act8;
using rudra::MatrixIn;
using rudra::MatrixOut;
using rudra::aligned;
using rudra::cuda_fail;
using rudra::fail;
using rudra::guarded;

bool known(int dtype) { return dtype == RUDRA_F32 || dtype == RUDRA_BF16; }
rudra::GradType type_of(int dtype) { return dtype == RUDRA_BF16 ? rudra::kBF16 : rudra::kF32; }
uint64_t size_of(int dtype) { return dtype == RUDRA_BF16 ? 2 : 4; }
uint64_t blocks_of(uint64_t cols) { return (cols + rudra::kBlock - 1) / rudra::kBlock; }

// 0, or the code of the failure it recorded.
int check_dims(const char* what, uint64_t rows, uint64_t cols) {
  if (rows > RUDRA_MAX_DIM || cols > RUDRA_MAX_DIM)
    return fail(RUDRA_E_INVAL, "%s: %llu x %llu has more than RUDRA_MAX_DIM rows or columns", what, (unsigned long long)rows, (unsigned long long)cols);
  return 0;
}
int check_matrix(const char* what, const void* p, int dtype, uint64_t rows, uint64_t cols, uint64_t ld) {
  if (!known(dtype)) return fail(RUDRA_E_INVAL, "%s: unknown dtype %d", what, dtype);
  if (const int e = check_dims(what, rows, cols)) return e;
  if (rows == 0 || cols == 0) return 0;
  if (p == nullptr || reinterpret_cast<uintptr_t>(p) % size_of(dtype)) return fail(RUDRA_E_INVAL, "%s is null or not aligned to its elements", what);
  if (ld < cols) return fail(RUDRA_E_INVAL, "%s: rows of %llu elements are %llu apart", what, (unsigned long long)cols, (unsigned long long)ld);
  if (ld > (1ull << 60) / rows) return fail(RUDRA_E_INVAL, "%s: ld of %llu is out of range", what, (unsigned long long)ld);
  return 0;
}
int check_blocks(const char* what, const void* codes, const void* scales, uint64_t rows, uint64_t cols) {
  if (const int e = check_dims(what, rows, cols)) return e;
  if (rows && cols && (!aligned(codes) || !aligned(scales))) return fail(RUDRA_E_INVAL, "%s: codes or scales are null or not 32-byte aligned", what);
  return 0;
}
int done(cudaError_t e, const char* what) { return e == cudaSuccess ? 0 : cuda_fail(e, what); }
cudaStream_t stream_of(void* s) { return static_cast<cudaStream_t>(s); }

rudra::Reports g_reports;   // of rudra_learner_sync

}  // namespace

extern "C" {

uint64_t rudra_mx4_codes_bytes(uint64_t rows, uint64_t cols) { return rows * blocks_of(cols) * 16; }
uint64_t rudra_mx4_scales_bytes(uint64_t rows, uint64_t cols) { return (rows + 127) / 128 * ((blocks_of(cols) + 3) / 4) * 512; }

int rudra_mx4_quantize(const void* src_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int transpose, void* codes_dev,
                       void* scales_dev, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("source", src_dev, dtype, rows, cols, ld)) return e;
    if (const int e = check_blocks("MX4 matrix", codes_dev, scales_dev, rows, cols)) return e;
    if (rows == 0 || cols == 0) return 0;
    const MatrixIn src = {src_dev, type_of(dtype), rows, cols, ld};
    return done(rudra::launch_mx4_quantize(src, transpose != 0, codes_dev, scales_dev, stream_of(cuda_stream)), "quantization kernel launch");
  });
}

int rudra_mx4_dequantize(const void* codes_dev, const void* scales_dev, uint64_t rows, uint64_t cols, void* dst_dev, int dtype,
                         uint64_t ld, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("destination", dst_dev, dtype, rows, cols, ld)) return e;
    if (const int e = check_blocks("MX4 matrix", codes_dev, scales_dev, rows, cols)) return e;
    if (rows == 0 || cols == 0) return 0;
    const MatrixOut dst = {dst_dev, type_of(dtype), rows, cols, ld};
    return done(rudra::launch_mx4_dequantize({codes_dev, scales_dev, rows, cols}, dst, stream_of(cuda_stream)), "expansion kernel launch");
  });
}

int rudra_mx4_matmul(const void* a_codes_dev, const void* a_scales_dev, uint64_t m, const void* b_codes_dev, const void* b_scales_dev,
                     uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_blocks("first factor", a_codes_dev, a_scales_dev, m, k)) return e;
    if (const int e = check_blocks("second factor", b_codes_dev, b_scales_dev, n, k)) return e;
    if (const int e = check_matrix("product", y_dev, y_dtype, m, n, ldy)) return e;
    if (m == 0 || n == 0) return 0;
    return done(rudra::launch_mx4_matmul({a_codes_dev, a_scales_dev, m, k}, {b_codes_dev, b_scales_dev, n, k}, {y_dev, type_of(y_dtype), m, n, ldy},
                                         stream_of(cuda_stream)),
                "4-bit product kernel launch");
  });
}

uint64_t rudra_mx4_linear_workspace(uint64_t m, uint64_t k) { return rudra::mx4_linear_workspace(m, k); }

int rudra_mx4_linear(const void* x_dev, int x_dtype, uint64_t ldx, uint64_t m, const void* w_codes_dev, const void* w_scales_dev,
                     uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy, void* workspace_dev, uint64_t workspace_bytes,
                     void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("input", x_dev, x_dtype, m, k, ldx)) return e;
    if (const int e = check_blocks("weights", w_codes_dev, w_scales_dev, n, k)) return e;
    if (const int e = check_matrix("product", y_dev, y_dtype, m, n, ldy)) return e;
    if (m == 0 || n == 0) return 0;
    const uint64_t need = rudra_mx4_linear_workspace(m, k);
    if (need && (!aligned(workspace_dev) || workspace_bytes < need))
      return fail(RUDRA_E_INVAL, "workspace is null, not 32-byte aligned or smaller than %llu bytes", (unsigned long long)need);
    return done(rudra::launch_mx4_linear({x_dev, type_of(x_dtype), m, k, ldx}, {w_codes_dev, w_scales_dev, n, k},
                                         {y_dev, type_of(y_dtype), m, n, ldy}, workspace_dev, stream_of(cuda_stream)),
                "4-bit product kernel launch");
  });
}

uint64_t rudra_act8_codes_bytes(uint64_t tokens, uint64_t channels) { return tokens * blocks_of(channels) * 32; }
uint64_t rudra_act8_scales_bytes(uint64_t tokens, uint64_t channels) { return tokens * rudra::act8_scale_pitch(channels); }

int rudra_act8_forward(int act, const void* x_dev, const void* up_dev, int dtype, uint64_t tokens, uint64_t channels, uint64_t ldx,
                       void* y_dev, uint64_t ldy, void* codes_dev, void* scales_dev, void* up_codes_dev, void* up_scales_dev,
                       void* cuda_stream) {
  return guarded([&]() -> int {
    if (act < RUDRA_ACT_NONE || act > RUDRA_ACT_SWIGLU) return fail(RUDRA_E_INVAL, "unknown activation %d", act);
    const bool two = act == RUDRA_ACT_SWIGLU;
    if (const int e = check_matrix("input", x_dev, dtype, tokens, channels, ldx)) return e;
    if (const int e = check_blocks("checkpoint", codes_dev, scales_dev, tokens, channels)) return e;
    if (two) {
      if (const int e = check_matrix("second input", up_dev, dtype, tokens, channels, ldx)) return e;
      if (const int e = check_blocks("second checkpoint", up_codes_dev, up_scales_dev, tokens, channels)) return e;
    } else if (up_dev || up_codes_dev || up_scales_dev) {
      return fail(RUDRA_E_INVAL, "only RUDRA_ACT_SWIGLU has a second input");
    }
    if (act != RUDRA_ACT_NONE) {
      if (const int e = check_matrix("output", y_dev, dtype, tokens, channels, ldy)) return e;
    } else if (y_dev) {
      return fail(RUDRA_E_INVAL, "RUDRA_ACT_NONE writes no output");
    }
    if (tokens == 0 || channels == 0) return 0;
    const rudra::GradType t = type_of(dtype);
    return done(rudra::launch_act8_forward(static_cast<rudra::Act>(act), {x_dev, t, tokens, channels, ldx}, up_dev, {y_dev, t, tokens, channels, ldy},
                                           {codes_dev, scales_dev}, {up_codes_dev, up_scales_dev}, stream_of(cuda_stream)),
                "activation kernel launch");
  });
}

int rudra_act8_backward(int act, const void* dy_dev, int dtype, uint64_t tokens, uint64_t channels, uint64_t lddy, const void* codes_dev,
                        const void* scales_dev, const void* up_codes_dev, const void* up_scales_dev, void* dx_dev, void* dup_dev,
                        uint64_t lddx, void* cuda_stream) {
  return guarded([&]() -> int {
    if (act < RUDRA_ACT_NONE || act > RUDRA_ACT_SWIGLU) return fail(RUDRA_E_INVAL, "unknown activation %d", act);
    const bool two = act == RUDRA_ACT_SWIGLU;
    if (const int e = check_matrix("gradient of the input", dx_dev, dtype, tokens, channels, lddx)) return e;
    if (const int e = check_blocks("checkpoint", codes_dev, scales_dev, tokens, channels)) return e;
    if (act != RUDRA_ACT_NONE) {
      if (const int e = check_matrix("gradient of the output", dy_dev, dtype, tokens, channels, lddy)) return e;
    } else if (dy_dev) {
      return fail(RUDRA_E_INVAL, "RUDRA_ACT_NONE expands the checkpoint and takes no gradient");
    }
    if (two) {
      if (const int e = check_matrix("gradient of the second input", dup_dev, dtype, tokens, channels, lddx)) return e;
      if (const int e = check_blocks("second checkpoint", up_codes_dev, up_scales_dev, tokens, channels)) return e;
    } else if (dup_dev || up_codes_dev || up_scales_dev) {
      return fail(RUDRA_E_INVAL, "only RUDRA_ACT_SWIGLU has a second input");
    }
    if (tokens == 0 || channels == 0) return 0;
    const rudra::GradType t = type_of(dtype);
    const Act8 saved = {const_cast<void*>(codes_dev), const_cast<void*>(scales_dev)};
    const Act8 saved_up = {const_cast<void*>(up_codes_dev), const_cast<void*>(up_scales_dev)};
    return done(rudra::launch_act8_backward(static_cast<rudra::Act>(act), {dy_dev, t, tokens, channels, lddy}, saved, saved_up,
                                            {dx_dev, t, tokens, channels, lddx}, dup_dev, stream_of(cuda_stream)),
                "activation gradient kernel launch");
  });
}

uint64_t rudra_act8_weight_grad_workspace(const void* dy_dev, int dy_dtype, uint64_t tokens, uint64_t n, uint64_t lddy) {
  if (!known(dy_dtype) || tokens > RUDRA_MAX_DIM || n > RUDRA_MAX_DIM) return 0;
  return rudra::act8_weight_grad_workspace({dy_dev, type_of(dy_dtype), tokens, n, lddy});
}

int rudra_act8_weight_grad(const void* dy_dev, int dy_dtype, uint64_t lddy, uint64_t tokens, uint64_t n, const void* codes_dev,
                           const void* scales_dev, uint64_t k, void* dw_dev, int dw_dtype, uint64_t lddw, void* workspace_dev,
                           uint64_t workspace_bytes, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("gradient of the output", dy_dev, dy_dtype, tokens, n, lddy)) return e;
    if (const int e = check_blocks("checkpoint", codes_dev, scales_dev, tokens, k)) return e;
    if (const int e = check_matrix("weight gradient", dw_dev, dw_dtype, n, k, lddw)) return e;
    if (n == 0 || k == 0) return 0;
    const MatrixIn dy = {dy_dev, type_of(dy_dtype), tokens, n, lddy};
    const uint64_t need = rudra::act8_weight_grad_workspace(dy);
    if (need && (!aligned(workspace_dev) || workspace_bytes < need))
      return fail(RUDRA_E_INVAL, "workspace is null, not 32-byte aligned or smaller than %llu bytes", (unsigned long long)need);
    const Act8 saved = {const_cast<void*>(codes_dev), const_cast<void*>(scales_dev)};
    return done(rudra::launch_act8_weight_grad(dy, saved, {dw_dev, type_of(dw_dtype), n, k, lddw}, workspace_dev, stream_of(cuda_stream)),
                "weight gradient kernel launch");
  });
}

int rudra_learner_sync(void* cuda_stream) {
  return guarded([&]() -> int {
    const cudaStream_t stream = stream_of(cuda_stream);
    rudra::Reports::Counts counts = {};
    unsigned long long id = 0;
    int device = 0;
    cudaError_t e = cudaStreamSynchronize(stream);      // first: a stream that is being captured refuses, and takes no copies to `counts`
    if (e == cudaSuccess) e = rudra::mx4_matmul_gave_up(&counts[0], stream);
    if (e == cudaSuccess) e = rudra::mx4_matmul_pair_gave_up(&counts[1], stream);
    if (e == cudaSuccess) e = rudra::act8_weight_grad_gave_up(&counts[2], stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e == cudaSuccess) e = cudaStreamGetId(stream, &id);
    if (e == cudaSuccess) e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_fail(e, "learner-side operators");
    if (g_reports.fresh(device, id, counts)) return fail(RUDRA_E_CUDA, "a product kernel on this device gave up a wait: its result is not valid");
    return 0;
  });
}

}  // extern "C"
