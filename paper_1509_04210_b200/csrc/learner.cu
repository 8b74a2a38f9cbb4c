// The exported learner-side operators: argument checks, and the launches behind them.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

#include "../../include/rudra_learner.h"
#include "host.h"
#include "learner.cuh"
#include "reports.h"

namespace {

using rudra::Act8;
using rudra::Gradient;
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
int check_vector(const char* what, const void* p, int dtype, uint64_t n) { return check_matrix(what, p, dtype, 1, n, n); }

// 0, or the refusal of a list of gradients; fills `list` where `out` gradients are written.
int gradients(const void* const* grads, const int* dtypes, const uint64_t* sizes, uint64_t count, void* const* outs, const int* out_dtypes, std::vector<Gradient>* list) {
  constexpr uint64_t kMost = 1ull << 24, kValues = 1ull << 43;
  if (count > kMost) return fail(RUDRA_E_INVAL, "%llu gradients are more than a list may have", (unsigned long long)count);
  if (count && (!grads || !dtypes || !sizes || !outs != !out_dtypes)) return fail(RUDRA_E_INVAL, "a list of gradients is null");
  uint64_t total = 0;
  list->reserve(count);
  for (uint64_t i = 0; i < count; ++i) {
    if (sizes[i] > kValues || (total += sizes[i]) > kValues) return fail(RUDRA_E_INVAL, "gradients of more than 2^43 values");
    if (!known(dtypes[i]) || (outs && !known(out_dtypes[i]))) return fail(RUDRA_E_INVAL, "gradient %llu: unknown dtype", (unsigned long long)i);
    void* const out = outs ? outs[i] : const_cast<void*>(grads[i]);
    const int out_dtype = outs ? out_dtypes[i] : dtypes[i];
    if (sizes[i] && (!grads[i] || reinterpret_cast<uintptr_t>(grads[i]) % size_of(dtypes[i]) || !out || reinterpret_cast<uintptr_t>(out) % size_of(out_dtype)))
      return fail(RUDRA_E_INVAL, "gradient %llu is null or not aligned to its elements", (unsigned long long)i);
    list->push_back({grads[i], out, sizes[i], type_of(dtypes[i]), type_of(out_dtype)});
  }
  return 0;
}

// Whether what is written overlaps: an output another output, the norm or another gradient, or its own gradient other than in its
// place; the norm, where it is `computed`, a gradient.
bool overlapping(const std::vector<Gradient>& list, const float* norm, bool computed) {
  struct Span {
    uintptr_t from, to;
    bool operator<(const Span& o) const { return from < o.from; }
  };
  std::vector<Span> written;
  written.reserve(list.size());
  uintptr_t low = UINTPTR_MAX, high = 0;
  bool sorted = true;
  for (const Gradient& g : list) {
    if (!g.size) continue;
    const uintptr_t out = reinterpret_cast<uintptr_t>(g.out), end = out + g.size * (g.out_type == rudra::kBF16 ? 2 : 4);
    sorted = sorted && (written.empty() || written.back().from <= out);
    written.push_back({out, end});
    low = std::min(low, out);
    high = std::max(high, end);
  }
  if (!sorted) std::sort(written.begin(), written.end());
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].from < written[i - 1].to) return true;
  const auto meets = [&](uintptr_t p, uintptr_t end) {
    if (p >= high || end <= low) return false;
    // the first output that begins behind the first byte, and the one before it
    const auto at = std::upper_bound(written.begin(), written.end(), Span{p, 0});
    return (at != written.end() && at->from < end) || (at != written.begin() && (at - 1)->to > p);
  };
  const uintptr_t n = reinterpret_cast<uintptr_t>(norm), n_end = reinterpret_cast<uintptr_t>(norm + 1);
  for (const Gradient& g : list) {
    if (!g.size || (g.p == g.out && g.type == g.out_type)) continue;
    const uintptr_t p = reinterpret_cast<uintptr_t>(g.p), end = p + g.size * (g.type == rudra::kBF16 ? 2 : 4);
    if (meets(p, end) || (computed && p < n_end && n < end)) return true;
  }
  return meets(n, n_end);
}

int done(cudaError_t e, const char* what) { return e == cudaSuccess ? 0 : cuda_fail(e, what); }
cudaStream_t stream_of(void* s) { return static_cast<cudaStream_t>(s); }

rudra::Reports g_reports;   // of rudra_learner_sync
// Where calls gather the counts on the device, so that one copy brings them: to ordinary memory of the host every copy waits for itself
// (a call took 50 us with six of them, 17 this way).
constexpr int kCounts = rudra::Reports::kKernels;
rudra::Places g_places;
__device__ uint32_t g_gathered[rudra::Places::kMost][kCounts];

struct Addresses {
  const uint32_t* of[kCounts];
};
__global__ void gather_kernel(const __grid_constant__ Addresses counts, int place) {
  if (threadIdx.x < kCounts) g_gathered[place][threadIdx.x] = *counts.of[threadIdx.x];
}
cudaError_t gather(int place, rudra::Reports::Counts& told, cudaStream_t stream) {
  Addresses at = {};
  cudaError_t e = rudra::mx4_matmul_count(&at.of[0]);
  if (e == cudaSuccess) e = rudra::mx4_matmul_pair_count(&at.of[1]);
  if (e == cudaSuccess) e = rudra::act8_weight_grad_count(&at.of[2]);
  if (e == cudaSuccess) e = rudra::fp8_matmul_count(&at.of[3]);
  if (e == cudaSuccess) e = rudra::fp8_matmul_pair_count(&at.of[4]);
  if (e == cudaSuccess) e = rudra::rms_norm_count(&at.of[5]);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1);
  cfg.blockDim = dim3(32);
  cfg.stream = stream;
  e = cudaLaunchKernelEx(&cfg, gather_kernel, at, place);
  if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(told.data(), g_gathered, sizeof(told), place * sizeof(told), cudaMemcpyDeviceToHost, stream);
  return e;
}

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

uint64_t rudra_fp8_codes_bytes(uint64_t rows, uint64_t cols) { return rows * ((cols + 127) / 128) * 128; }
uint64_t rudra_fp8_scales_bytes(uint64_t rows, uint64_t cols) { return (rows + 127) / 128 * (((cols + 127) / 128 + 3) / 4) * 512; }

int rudra_fp8_quantize(const void* src_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int transpose, int square, void* codes_dev,
                       void* scales_dev, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("source", src_dev, dtype, rows, cols, ld)) return e;
    if (const int e = check_blocks("FP8 matrix", codes_dev, scales_dev, rows, cols)) return e;
    if (rows == 0 || cols == 0) return 0;
    const MatrixIn src = {src_dev, type_of(dtype), rows, cols, ld};
    return done(rudra::launch_fp8_quantize(src, transpose != 0, square != 0, codes_dev, scales_dev, stream_of(cuda_stream)), "quantization kernel launch");
  });
}

int rudra_fp8_dequantize(const void* codes_dev, const void* scales_dev, uint64_t rows, uint64_t cols, void* dst_dev, int dtype,
                         uint64_t ld, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("destination", dst_dev, dtype, rows, cols, ld)) return e;
    if (const int e = check_blocks("FP8 matrix", codes_dev, scales_dev, rows, cols)) return e;
    if (rows == 0 || cols == 0) return 0;
    const MatrixOut dst = {dst_dev, type_of(dtype), rows, cols, ld};
    return done(rudra::launch_fp8_dequantize({codes_dev, scales_dev, rows, cols}, dst, stream_of(cuda_stream)), "expansion kernel launch");
  });
}

int rudra_fp8_matmul(const void* a_codes_dev, const void* a_scales_dev, uint64_t m, const void* b_codes_dev, const void* b_scales_dev,
                     uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy, void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_blocks("first factor", a_codes_dev, a_scales_dev, m, k)) return e;
    if (const int e = check_blocks("second factor", b_codes_dev, b_scales_dev, n, k)) return e;
    if (const int e = check_matrix("product", y_dev, y_dtype, m, n, ldy)) return e;
    if (m == 0 || n == 0) return 0;
    return done(rudra::launch_fp8_matmul({a_codes_dev, a_scales_dev, m, k}, {b_codes_dev, b_scales_dev, n, k}, {y_dev, type_of(y_dtype), m, n, ldy},
                                         stream_of(cuda_stream)),
                "8-bit product kernel launch");
  });
}

uint64_t rudra_fp8_linear_workspace(uint64_t m, uint64_t k) { return rudra::fp8_linear_workspace(m, k); }

int rudra_fp8_linear(const void* x_dev, int x_dtype, uint64_t ldx, uint64_t m, const void* w_codes_dev, const void* w_scales_dev,
                     uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy, void* workspace_dev, uint64_t workspace_bytes,
                     void* cuda_stream) {
  return guarded([&]() -> int {
    if (const int e = check_matrix("input", x_dev, x_dtype, m, k, ldx)) return e;
    if (const int e = check_blocks("weights", w_codes_dev, w_scales_dev, n, k)) return e;
    if (const int e = check_matrix("product", y_dev, y_dtype, m, n, ldy)) return e;
    if (m == 0 || n == 0) return 0;
    const uint64_t need = rudra_fp8_linear_workspace(m, k);
    if (need && (!aligned(workspace_dev) || workspace_bytes < need))
      return fail(RUDRA_E_INVAL, "workspace is null, not 32-byte aligned or smaller than %llu bytes", (unsigned long long)need);
    return done(rudra::launch_fp8_linear({x_dev, type_of(x_dtype), m, k, ldx}, {w_codes_dev, w_scales_dev, n, k},
                                         {y_dev, type_of(y_dtype), m, n, ldy}, workspace_dev, stream_of(cuda_stream)),
                "8-bit product kernel launch");
  });
}

int rudra_rms_norm(const void* x_dev, uint64_t ldx, const void* residual_dev, uint64_t ldr, int dtype, uint64_t tokens, uint64_t channels,
                   const void* weight_dev, int weight_dtype, float eps, void* sum_dev, uint64_t ldsum, void* y_dev, uint64_t ldy,
                   void* fp8_codes_dev, void* fp8_scales_dev, void* act8_codes_dev, void* act8_scales_dev, void* cuda_stream) {
  return guarded([&]() -> int {
    const rudra::GradType t = type_of(dtype);
    if (const int e = check_matrix("input", x_dev, dtype, tokens, channels, ldx)) return e;
    if (const int e = check_vector("weight", tokens ? weight_dev : nullptr, weight_dtype, tokens ? channels : 0)) return e;
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(RUDRA_E_INVAL, "eps is negative or not finite");
    if (!residual_dev != !sum_dev && tokens && channels) return fail(RUDRA_E_INVAL, "a residual and the sum with it go together");
    if (residual_dev) {
      if (const int e = check_matrix("residual", residual_dev, dtype, tokens, channels, ldr)) return e;
      if (const int e = check_matrix("sum", sum_dev, dtype, tokens, channels, ldsum)) return e;
    }
    if (y_dev)
      if (const int e = check_matrix("output", y_dev, dtype, tokens, channels, ldy)) return e;
    if (y_dev && y_dev == sum_dev) return fail(RUDRA_E_INVAL, "output and sum are one matrix");
    if (fp8_codes_dev || fp8_scales_dev)
      if (const int e = check_blocks("FP8 output", fp8_codes_dev, fp8_scales_dev, tokens, channels)) return e;
    if (act8_codes_dev || act8_scales_dev)
      if (const int e = check_blocks("checkpoint", act8_codes_dev, act8_scales_dev, tokens, channels)) return e;
    if (tokens == 0 || channels == 0) return 0;
    if (!y_dev && !fp8_codes_dev && !act8_codes_dev) return fail(RUDRA_E_INVAL, "no output is wanted");
    return done(rudra::launch_rms_norm({{x_dev, t, tokens, channels, ldx}, {residual_dev, t, tokens, channels, ldr}, weight_dev, type_of(weight_dtype), eps,
                                        {sum_dev, t, tokens, channels, ldsum}, {y_dev, t, tokens, channels, ldy}, {fp8_codes_dev, fp8_scales_dev},
                                        {act8_codes_dev, act8_scales_dev}}, stream_of(cuda_stream)),
                "norm kernel launch");
  });
}

uint64_t rudra_rms_norm_backward_workspace(uint64_t tokens, uint64_t channels) {
  if (tokens == 0 || channels == 0 || tokens > RUDRA_MAX_DIM || channels > RUDRA_MAX_DIM) return 0;
  return rudra::rms_norm_backward_workspace(tokens, channels);
}

int rudra_rms_norm_backward(const void* dy_dev, uint64_t lddy, const void* s_dev, uint64_t lds, const void* dsum_dev, uint64_t lddsum, int dtype,
                            uint64_t tokens, uint64_t channels, const void* weight_dev, int weight_dtype, float eps, void* ds_dev, uint64_t ldds,
                            void* dweight_dev, int dweight_dtype, void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream) {
  return guarded([&]() -> int {
    const rudra::GradType t = type_of(dtype);
    if (const int e = check_matrix("gradient of the output", dy_dev, dtype, tokens, channels, lddy)) return e;
    if (const int e = check_matrix("normed input", s_dev, dtype, tokens, channels, lds)) return e;
    if (dsum_dev)
      if (const int e = check_matrix("gradient of the sum", dsum_dev, dtype, tokens, channels, lddsum)) return e;
    if (const int e = check_vector("weight", tokens ? weight_dev : nullptr, weight_dtype, tokens ? channels : 0)) return e;
    if (const int e = check_matrix("gradient of the input", ds_dev, dtype, tokens, channels, ldds)) return e;
    if (const int e = check_vector("weight gradient", dweight_dev, dweight_dtype, channels)) return e;
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(RUDRA_E_INVAL, "eps is negative or not finite");
    if (channels == 0) return 0;
    if (tokens == 0) return done(cudaMemsetAsync(dweight_dev, 0, channels * size_of(dweight_dtype), stream_of(cuda_stream)), "clearing the weight gradient");
    const uint64_t need = rudra_rms_norm_backward_workspace(tokens, channels);
    if (need && (!aligned(workspace_dev) || workspace_bytes < need))
      return fail(RUDRA_E_INVAL, "workspace is null, not 32-byte aligned or smaller than %llu bytes", (unsigned long long)need);
    return done(rudra::launch_rms_norm_backward({{dy_dev, t, tokens, channels, lddy}, {s_dev, t, tokens, channels, lds}, {dsum_dev, t, tokens, channels, lddsum},
                                                 weight_dev, type_of(weight_dtype), eps, {ds_dev, t, tokens, channels, ldds}, dweight_dev, type_of(dweight_dtype)},
                                                workspace_dev, stream_of(cuda_stream)),
                "norm gradient kernel launch");
  });
}

uint64_t rudra_grad_norm_workspace(uint64_t count) { return rudra::grad_norm_workspace(count); }

int rudra_grad_norm(const void* const* grads_dev, const int* dtypes, const uint64_t* sizes, uint64_t count, float* norm_dev, void* workspace_dev,
                    uint64_t workspace_bytes, void* cuda_stream) {
  return guarded([&]() -> int {
    std::vector<Gradient> list;
    if (const int e = gradients(grads_dev, dtypes, sizes, count, nullptr, nullptr, &list)) return e;
    if (const int e = check_vector("norm", norm_dev, RUDRA_F32, 1)) return e;
    const uint64_t need = rudra_grad_norm_workspace(count);
    if (!aligned(workspace_dev) || workspace_bytes < need)
      return fail(RUDRA_E_INVAL, "workspace is null, not 32-byte aligned or smaller than %llu bytes", (unsigned long long)need);
    return done(rudra::launch_grad_norm(list.data(), list.size(), norm_dev, workspace_dev, stream_of(cuda_stream)), "gradient norm kernel launch");
  });
}

int rudra_grad_clip(const void* const* grads_dev, const int* dtypes, const uint64_t* sizes, uint64_t count, float* norm_dev, int norm_known,
                    float max_norm, void* const* outs_dev, const int* out_dtypes, void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream) {
  return guarded([&]() -> int {
    std::vector<Gradient> list;
    if (count && !outs_dev) return fail(RUDRA_E_INVAL, "a list of outputs is null");
    if (const int e = gradients(grads_dev, dtypes, sizes, count, outs_dev, out_dtypes, &list)) return e;
    if (const int e = check_vector("norm", norm_dev, RUDRA_F32, 1)) return e;
    if (!(max_norm >= 0.f)) return fail(RUDRA_E_INVAL, "max_norm is negative or not a number");
    const uint64_t need = norm_known ? 0 : rudra_grad_norm_workspace(count);
    if (need && (!aligned(workspace_dev) || workspace_bytes < need))
      return fail(RUDRA_E_INVAL, "workspace is null, not 32-byte aligned or smaller than %llu bytes", (unsigned long long)need);
    if (overlapping(list, norm_dev, norm_known == 0)) return fail(RUDRA_E_INVAL, "outputs overlap each other, other gradients or the norm, or it a gradient");
    return done(rudra::launch_grad_clip(list.data(), list.size(), norm_dev, max_norm, norm_known != 0, workspace_dev, stream_of(cuda_stream)),
                "gradient clipping kernel launch");
  });
}

int rudra_learner_sync(void* cuda_stream) {
  return guarded([&]() -> int {
    const cudaStream_t stream = stream_of(cuda_stream);
    rudra::Reports::Counts counts = {};
    unsigned long long id = 0;
    int device = 0;
    cudaError_t e = cudaStreamSynchronize(stream);      // first: a stream that is being captured refuses, and takes no copies to `counts`
    const rudra::Places::Place place(g_places);
    if (place.number >= 0) {
      if (e == cudaSuccess) e = gather(place.number, counts, stream);
    } else {      // more calls at once than there are places
      if (e == cudaSuccess) e = rudra::mx4_matmul_gave_up(&counts[0], stream);
      if (e == cudaSuccess) e = rudra::mx4_matmul_pair_gave_up(&counts[1], stream);
      if (e == cudaSuccess) e = rudra::act8_weight_grad_gave_up(&counts[2], stream);
      if (e == cudaSuccess) e = rudra::fp8_matmul_gave_up(&counts[3], stream);
      if (e == cudaSuccess) e = rudra::fp8_matmul_pair_gave_up(&counts[4], stream);
      if (e == cudaSuccess) e = rudra::rms_norm_gave_up(&counts[5], stream);
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e == cudaSuccess) e = cudaStreamGetId(stream, &id);
    if (e == cudaSuccess) e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_fail(e, "learner-side operators");
    if (g_reports.fresh(device, id, counts)) return fail(RUDRA_E_CUDA, "a kernel on this device gave up a wait: its result is not valid");
    return 0;
  });
}

}  // extern "C"
