// Activation functions with an 8-bit checkpoint of their input: forward (value and checkpoint in one
// pass) and backward (slope from the checkpoint).  Element-wise but for a block's shared scale, so bound
// by HBM: per value and input 2G + 33/32 bytes each way (G = 2 bf16, 4 f32).  Sigmoids are formed from the
// fast exponential and reciprocal, each within about 2 ulp in 32 bits.
#include "blocks.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float sigmoid(float x) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.f + __expf(-x)));   // exp may reach infinity: the reciprocal is 0
  return r;
}

constexpr float kGeluA = 1.5957691216057308f;   // 2 sqrt(2 / pi): gelu(x) = x sigmoid(A (x + B x^3))
constexpr float kGeluB = 0.044715f;

template <Act A> __device__ __forceinline__ float value(float x) {
  if (A == kRelu) return x > 0.f ? x : x != x ? x : 0.f;
  if (A == kGelu) return x * sigmoid(kGeluA * fmaf(kGeluB * x, x * x, x));
  return x * sigmoid(x);
}

// f'(x); `f`: f(x), from the same sigmoid.
template <Act A> __device__ __forceinline__ float slope(float x, float& f) {
  if (A == kRelu) { f = x; return x > 0.f ? 1.f : x != x ? x : 0.f; }
  if (A == kGelu) {
    const float s = sigmoid(kGeluA * fmaf(kGeluB * x, x * x, x));
    const float t = s * (1.f - s);
    f = x * s;
    // where the sigmoid is 0 or 1 its slope is nothing, however far x^3 has run
    return t == 0.f ? s : fmaf(x * t, kGeluA * fmaf(3.f * kGeluB * x, x, 1.f), s);
  }
  const float s = sigmoid(x);
  f = x * s;
  return fmaf(f, 1.f - s, s);
}

struct Saved {
  uint2* codes;
  uint8_t* scales;
};

__device__ __forceinline__ void save(const Saved& to, uint64_t unit, const float (&x)[8], bool in) {
  const uint32_t s = scale_byte(block_max_bits(max_bits(x)), 6);
  const uint2 w = int8_codes(x, inverse_scale(s));
  if (!in) return;
  to.codes[unit] = w;
  if (unit % 4 == 0) to.scales[unit / 4] = (uint8_t)s;
}

__device__ __forceinline__ void restore(const Saved& from, uint64_t unit, float (&x)[8]) {
  int8_values(__ldg(from.codes + unit), scale_value(__ldg(from.scales + unit / 4)), x);
}

// A unit is 8 values; checkpoint rows are whole blocks of four units, so unit numbers run through the
// checkpoint without gaps and four neighbouring lanes always share a block.
template <typename G, Act A>
__global__ void __launch_bounds__(kThreads) forward_kernel(const G* __restrict__ x, const G* __restrict__ up, uint64_t ldx,
                                                           uint32_t cols, uint64_t units, bool wide_in, bool wide_out,
                                                           G* __restrict__ y, uint64_t ldy, Saved saved, Saved saved_up) {
  const uint32_t per_row = (cols + 31) / 32 * 4;
  const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  const uint64_t row = i / per_row;
  const uint32_t c = (uint32_t)(i - row * per_row) * 8;
  const bool in = i < units;
  const int have = in && c < cols ? (int)min(8u, cols - c) : 0;
  const uint64_t at = have ? row * ldx + c : 0;
  float a[8], b[8];
  load8(x + at, wide_in && have == 8, have, a);
  if (A == kSwiglu) load8(up + at, wide_in && have == 8, have, b);
  save(saved, i, a, in);
  if (A == kSwiglu) save(saved_up, i, b, in);
  if constexpr (A != kNone) {
    if (!have) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = A == kSwiglu ? value<A>(a[e]) * b[e] : value<A>(a[e]);
    store8(y + row * ldy + c, wide_out && have == 8, have, a);
  }
}

template <typename G, Act A>
__global__ void __launch_bounds__(kThreads) backward_kernel(const G* dy, uint64_t lddy, uint32_t cols, uint64_t units, bool wide_in,
                                                            bool wide_out, Saved saved, Saved saved_up, G* dx, G* dup, uint64_t lddx) {
  const uint32_t per_row = (cols + 31) / 32 * 4;
  const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= units) return;
  const uint64_t row = i / per_row;
  const uint32_t c = (uint32_t)(i - row * per_row) * 8;
  if (c >= cols) return;
  const int have = (int)min(8u, cols - c);
  float g[8], x[8], u[8];
  if (A != kNone) load8(dy + row * lddy + c, wide_in && have == 8, have, g);
  restore(saved, i, x);
  if (A == kSwiglu) restore(saved_up, i, u);
  if constexpr (A != kNone) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f;
      const float d = slope<A>(x[e], f);
      x[e] = A == kSwiglu ? g[e] * u[e] * d : g[e] * d;
      if (A == kSwiglu) u[e] = g[e] * f;
    }
  }
  store8(dx + row * lddx + c, wide_out && have == 8, have, x);
  if (A == kSwiglu) store8(dup + row * lddx + c, wide_out && have == 8, have, u);
}

cudaError_t shape(uint64_t rows, uint64_t cols, uint64_t* units, unsigned* blocks) {
  *units = rows * ((cols + 31) / 32 * 4);
  const uint64_t b = (*units + kThreads - 1) / kThreads;
  if (b > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  *blocks = (unsigned)b;
  return cudaSuccess;
}

Saved saved_of(const Act8& a) { return Saved{static_cast<uint2*>(a.codes), static_cast<uint8_t*>(a.scales)}; }

template <typename G, Act A>
cudaError_t forward(const MatrixIn& x, const void* up, const MatrixOut& y, const Act8& saved, const Act8& saved_up, cudaStream_t stream) {
  uint64_t units;
  unsigned blocks;
  const cudaError_t e = shape(x.rows, x.cols, &units, &blocks);
  if (e != cudaSuccess) return e;
  const bool wide_in = wide_rows<G>(x.p, x.ld) && (A != kSwiglu || wide_rows<G>(up, x.ld));
  forward_kernel<G, A><<<blocks, kThreads, 0, stream>>>(static_cast<const G*>(x.p), static_cast<const G*>(up), x.ld, (uint32_t)x.cols,
                                                        units, wide_in, wide_rows<G>(y.p, y.ld), static_cast<G*>(y.p), y.ld,
                                                        saved_of(saved), saved_of(saved_up));
  return cudaGetLastError();
}

template <typename G, Act A>
cudaError_t backward(const MatrixIn& dy, const Act8& saved, const Act8& saved_up, const MatrixOut& dx, void* dup, cudaStream_t stream) {
  uint64_t units;
  unsigned blocks;
  const cudaError_t e = shape(dx.rows, dx.cols, &units, &blocks);
  if (e != cudaSuccess) return e;
  const bool wide_out = wide_rows<G>(dx.p, dx.ld) && (A != kSwiglu || wide_rows<G>(dup, dx.ld));
  backward_kernel<G, A><<<blocks, kThreads, 0, stream>>>(static_cast<const G*>(dy.p), dy.ld, (uint32_t)dx.cols, units, wide_rows<G>(dy.p, dy.ld),
                                                         wide_out, saved_of(saved), saved_of(saved_up), static_cast<G*>(dx.p),
                                                         static_cast<G*>(dup), dx.ld);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_act8_forward(Act act, const MatrixIn& x, const void* up, const MatrixOut& y, const Act8& saved,
                                const Act8& saved_up, cudaStream_t stream) {
  const bool h = x.type == kBF16;
  switch (act) {
    case kNone: return h ? forward<__nv_bfloat16, kNone>(x, up, y, saved, saved_up, stream) : forward<float, kNone>(x, up, y, saved, saved_up, stream);
    case kRelu: return h ? forward<__nv_bfloat16, kRelu>(x, up, y, saved, saved_up, stream) : forward<float, kRelu>(x, up, y, saved, saved_up, stream);
    case kSilu: return h ? forward<__nv_bfloat16, kSilu>(x, up, y, saved, saved_up, stream) : forward<float, kSilu>(x, up, y, saved, saved_up, stream);
    case kGelu: return h ? forward<__nv_bfloat16, kGelu>(x, up, y, saved, saved_up, stream) : forward<float, kGelu>(x, up, y, saved, saved_up, stream);
    default: return h ? forward<__nv_bfloat16, kSwiglu>(x, up, y, saved, saved_up, stream) : forward<float, kSwiglu>(x, up, y, saved, saved_up, stream);
  }
}

cudaError_t launch_act8_backward(Act act, const MatrixIn& dy, const Act8& saved, const Act8& saved_up, const MatrixOut& dx, void* dup,
                                 cudaStream_t stream) {
  const bool h = dx.type == kBF16;
  switch (act) {
    case kNone: return h ? backward<__nv_bfloat16, kNone>(dy, saved, saved_up, dx, dup, stream) : backward<float, kNone>(dy, saved, saved_up, dx, dup, stream);
    case kRelu: return h ? backward<__nv_bfloat16, kRelu>(dy, saved, saved_up, dx, dup, stream) : backward<float, kRelu>(dy, saved, saved_up, dx, dup, stream);
    case kSilu: return h ? backward<__nv_bfloat16, kSilu>(dy, saved, saved_up, dx, dup, stream) : backward<float, kSilu>(dy, saved, saved_up, dx, dup, stream);
    case kGelu: return h ? backward<__nv_bfloat16, kGelu>(dy, saved, saved_up, dx, dup, stream) : backward<float, kGelu>(dy, saved, saved_up, dx, dup, stream);
    default: return h ? backward<__nv_bfloat16, kSwiglu>(dy, saved, saved_up, dx, dup, stream) : backward<float, kSwiglu>(dy, saved, saved_up, dx, dup, stream);
  }
}

}  // namespace rudra
