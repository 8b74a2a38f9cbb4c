// Activation functions with an 8-bit checkpoint of their input: forward (value and checkpoint in one
// pass) and backward (slope from the checkpoint).  Element-wise but for a block's shared scale, so bound
// by HBM: per value and input 2G + 33/32 bytes each way (G = 2 bf16, 4 f32).  Sigmoids are formed from the
// approximate base-2 exponential and reciprocal, each within about 2 units in the last place of 32 bits; the exponent is
// rounded before that (x log2 e to 32 bits), so far out a sigmoid is off by some |x| 2^-24 of itself (gelu in f32: 1.8e-7 over a
// normal x, 1.6e-7 with the plain exponential).
// Measured at 8192 x 4096: silu in f32 46.3 us each way = 6.5 TB/s, swiglu in bf16 42.9 and 44.1 us = 6.3 and 6.2 TB/s,
// gelu in bf16 27.4 and 28.5 us = 6.2 and 5.9 TB/s (with the plain exponential, reciprocal and a clamp of
// each value by itself 35 and 39 us: the instructions were the bound); the checkpoint alone of bf16 18.7 us.
#include <algorithm>

#include "blocks.cuh"
#include "launch.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

constexpr int kThreads = 128;   // swiglu backward 45.6 us; 48.4 with 256

constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + 2^t).  2^t may reach infinity, whose reciprocal is 0; results below 2^-126 count as 0.
__device__ __forceinline__ float sigmoid2(float t) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}

constexpr float kGeluA = 1.5957691216057308f;   // 2 sqrt(2 / pi): gelu(x) = x sigmoid(A (x + B x^3))
constexpr float kGeluB = 0.044715f;

// The sigmoid that f(x) = x * sigmoid is made with.
template <Act A> __device__ __forceinline__ float gate(float x) {
  if (A == kGelu) return sigmoid2(x * fmaf(-kLog2e * kGeluA * kGeluB * x, x, -kLog2e * kGeluA));
  return sigmoid2(-kLog2e * x);
}

template <Act A> __device__ __forceinline__ float value(float x) {
  if (A == kRelu) return x > 0.f ? x : x != x ? x : 0.f;
  return x * gate<A>(x);
}

// f'(x); `f`: f(x), from the same sigmoid.
template <Act A> __device__ __forceinline__ float slope(float x, float& f) {
  if (A == kRelu) { f = x; return x > 0.f ? 1.f : x != x ? x : 0.f; }
  const float s = gate<A>(x);
  f = x * s;
  if (A == kGelu) {
    const float t = f * (1.f - s);
    // where the sigmoid is 0 or 1 its slope is nothing, however far x^2 has run
    return t == 0.f ? s : fmaf(t, fmaf(3.f * kGeluA * kGeluB * x, x, kGeluA), s);
  }
  return fmaf(f, 1.f - s, s);
}

struct Saved {
  uint4* codes;
  uint8_t* scales;
  uint32_t pitch;     // of the scale bytes
};

template <typename G> __device__ __forceinline__ void save(const Saved& to, uint32_t unit, uint32_t row, uint32_t block, const Values<G>& x, bool in) {
  const uint32_t s = scale_byte(block_max_bits(x.max_bits()), 6);
  const uint4 w = int8_codes(x, s);
  if (!in) return;
  to.codes[unit] = w;
  if (unit % 2 == 0) to.scales[(uint64_t)row * to.pitch + block] = (uint8_t)s;
}

struct Restored {
  uint4 w;
  uint32_t s;
  __device__ __forceinline__ void load(const Saved& from, uint32_t unit, uint32_t row, uint32_t block) {
    w = read_once(from.codes + unit);
    s = read_byte(from.scales + (uint64_t)row * from.pitch + block);
  }
  __device__ __forceinline__ void values(float (&x)[kValues]) const { int8_values(w, scale_value(s), x); }
};

template <bool ANY, typename G> __device__ __forceinline__ void write(G* p, Access access, int have, const float (&x)[kValues]) {
  if constexpr (ANY) {
    __shared__ Meeting meeting[kThreads / 32];
    store_values_anyhow(meeting[threadIdx.x / 32], p, have, x);
  } else {
    store_values(p, access, have, x);
  }
}

// Checkpoint rows are whole blocks of two units (of a thread's values), so unit numbers run through the
// checkpoint without gaps and neighbouring lanes share a block.
template <typename G, Act A, bool ANY>
__global__ void __launch_bounds__(kThreads) forward_kernel(Rows<G> x, Rows<G> up, uint32_t cols, Divisor per_row, uint32_t units,
                                                           Access access_out, G* y, uint64_t ldy, Saved saved, Saved saved_up) {
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x, row = per_row.quotient(i), c = (i - row * per_row.d) * kValues;
  const bool in = i < units;
  const int have = in && c < cols ? (int)min((uint32_t)kValues, cols - c) : 0;
  const uint64_t at = have ? row * x.ld + c : 0;
  Values<G> a, b;
  a.template load<ANY>(x, at, have);
  if (A == kSwiglu) b.template load<ANY>(up, at, have);
  save(saved, i, row, c / 32, a, in);
  if (A == kSwiglu) save(saved_up, i, row, c / 32, b, in);
  if constexpr (A != kNone) {
    float v[kValues];
#pragma unroll
    for (int e = 0; e < kValues; ++e) v[e] = A == kSwiglu ? value<A>(a.get(e)) * b.get(e) : value<A>(a.get(e));
    write<ANY>(y + (have ? row * ldy + c : 0), access_out, have, v);
  }
}

template <typename G, Act A, bool ANY>
__global__ void __launch_bounds__(kThreads) backward_kernel(Rows<G> dy, uint32_t cols, Divisor per_row, uint32_t units, Access access_out, Saved saved,
                                                            Saved saved_up, G* dx, G* dup, uint64_t lddx) {
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x, row = per_row.quotient(i), c = (i - row * per_row.d) * kValues;
  const int have = i < units && c < cols ? (int)min((uint32_t)kValues, cols - c) : 0;
  Values<G> g;
  Restored rx = {}, ru = {};
  if (have) {
    if (A != kNone) g.template load<ANY>(dy, row * dy.ld + c, have);
    rx.load(saved, i, row, c / 32);
    if (A == kSwiglu) ru.load(saved_up, i, row, c / 32);
  }
  float x[kValues], u[kValues];
  rx.values(x);
  if (A == kSwiglu) ru.values(u);
  if constexpr (A != kNone) {
#pragma unroll
    for (int e = 0; e < kValues; ++e) {
      float f;
      const float d = slope<A>(x[e], f);
      x[e] = A == kSwiglu ? g.get(e) * u[e] * d : g.get(e) * d;
      if (A == kSwiglu) u[e] = g.get(e) * f;
    }
  }
  const uint64_t at = have ? row * lddx + c : 0;
  write<ANY>(dx + at, access_out, have, x);
  if (A == kSwiglu) write<ANY>(dup + at, access_out, have, u);
}

// Rows of a launch: as many as keep the number of its units below 2^31.
struct Part {
  uint64_t per_row, most;
  Part(uint64_t cols) : per_row((cols + 31) / 32 * 2), most(std::max<uint64_t>(1, 0x70000000ull / per_row)) {}
};

// A checkpoint of `cols` channels from row `r` on.
Saved from_row(const Act8& a, uint64_t cols, uint64_t r) {
  const uint64_t pitch = act8_scale_pitch(cols);
  if (!a.codes) return Saved{nullptr, nullptr, 0};
  return Saved{static_cast<uint4*>(a.codes) + r * ((cols + 31) / 32 * 2), static_cast<uint8_t*>(a.scales) + r * pitch, (uint32_t)pitch};
}

template <typename G, Act A>
cudaError_t forward(const MatrixIn& x, const void* up, const MatrixOut& y, const Act8& saved, const Act8& saved_up, cudaStream_t stream) {
  const Part part(x.cols);
  const Access in = A == kSwiglu ? both(access_of<G>(x.p, x.ld), access_of<G>(up, x.ld)) : access_of<G>(x.p, x.ld);
  const Access out = access_of<G>(y.p, A == kNone ? 0 : y.ld);
  const bool anyhow = in == kByElement || out == kByElement;
  for (uint64_t r = 0; r < x.rows; r += part.most) {
    const uint64_t units = std::min(part.most, x.rows - r) * part.per_row;
    if (units > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_after(
        anyhow ? forward_kernel<G, A, true> : forward_kernel<G, A, false>, (uint32_t)((units + kThreads - 1) / kThreads), kThreads, 0, 1, stream, Rows<G>::of(x.p, x.rows, x.cols, x.ld, r),
        Rows<G>::of(up, x.rows, x.cols, x.ld, r), (uint32_t)x.cols, Divisor((uint32_t)part.per_row), (uint32_t)units, out,
        static_cast<G*>(y.p) + (y.p ? r * y.ld : 0), y.ld, from_row(saved, x.cols, r), from_row(saved_up, x.cols, r));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <typename G, Act A>
cudaError_t backward(const MatrixIn& dy, const Act8& saved, const Act8& saved_up, const MatrixOut& dx, void* dup, cudaStream_t stream) {
  const Part part(dx.cols);
  const Access out = A == kSwiglu ? both(access_of<G>(dx.p, dx.ld), access_of<G>(dup, dx.ld)) : access_of<G>(dx.p, dx.ld);
  const bool anyhow = out == kByElement || (A != kNone && access_of<G>(dy.p, dy.ld) == kByElement);
  for (uint64_t r = 0; r < dx.rows; r += part.most) {
    const uint64_t units = std::min(part.most, dx.rows - r) * part.per_row;
    if (units > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_after(
        anyhow ? backward_kernel<G, A, true> : backward_kernel<G, A, false>, (uint32_t)((units + kThreads - 1) / kThreads), kThreads, 0, 1, stream, Rows<G>::of(dy.p, dx.rows, dx.cols, dy.ld, r),
        (uint32_t)dx.cols, Divisor((uint32_t)part.per_row), (uint32_t)units, out, from_row(saved, dx.cols, r), from_row(saved_up, dx.cols, r),
        static_cast<G*>(dx.p) + r * dx.ld, static_cast<G*>(dup) + (dup ? r * dx.ld : 0), dx.ld);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
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
