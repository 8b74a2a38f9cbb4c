// The norm of many gradients taken together, and their scaling to a largest norm.
//
// The gradients are cut into chunks of kChunk values, each within one gradient; a block takes every gridDim-th chunk.  Where they
// lie comes as a kernel parameter, so a list costs no copy.  Squares are added in 32 bits over 16 values, everything beyond
// that in 64, in an order that depends on the list alone; 16 values whose squares leave the range of a float are
// squared in 64 bits.  One read for the norm, one read and one write for the scaling: bound by HBM.
#include <algorithm>

#include "blocks.cuh"
#include "launch.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

constexpr uint32_t kThreads = 256, kPieces = 2, kChunk = kThreads * kPieces * kValues;
constexpr uint32_t kBlocks = 148 * 8;    // at most; a partial sum each

// Part of a list, as a kernel takes it.
template <uint32_t MOST> struct List {
  const void* p[MOST];
  void* out[MOST];
  uint64_t size[MOST];
  uint32_t end[MOST];        // chunks up to and with this gradient's last
  uint8_t wide[MOST];        // bit 0: f32, bit 1: its output is
  uint32_t count;
};

// The gradient that chunk c is of: the first whose chunks end behind it.
template <uint32_t MOST> __device__ __forceinline__ uint32_t gradient_of(const List<MOST>& list, uint32_t c) {
  uint32_t lo = 0, hi = list.count - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (list.end[mid] > c) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

template <typename G> __device__ __forceinline__ Rows<G> rows_of(const void* p, uint64_t size) {
  const G* g = static_cast<const G*>(p);
  return Rows<G>{g, 0, g + size, access_of<G>(p, 0)};
}

// Sum of a thread's squares.
template <typename G> __device__ __forceinline__ double squares(const Values<G>& v) {
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int i = 0; i < kValues; i += 2) {
    a = fmaf(v.get(i), v.get(i), a);
    b = fmaf(v.get(i + 1), v.get(i + 1), b);
  }
  const float s = a + b;
  if (s > 1e-24f && s < 1e38f) return (double)s;      // what squares below 2^-126 lost is nothing next to it
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < kValues; ++i) d = fma((double)v.get(i), (double)v.get(i), d);
  return d;
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double room[kThreads / 32];
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if (threadIdx.x % 32 == 0) room[threadIdx.x / 32] = v;
  __syncthreads();
  v = room[0];
  for (uint32_t i = 1; i < kThreads / 32; ++i) v += room[i];
  return v;
}

template <typename G> __device__ __forceinline__ double chunk_squares(const void* p, uint64_t size, uint64_t at) {
  const Rows<G> m = rows_of<G>(p, size);
  Values<G> v[kPieces];
#pragma unroll
  for (uint32_t u = 0; u < kPieces; ++u) {
    const uint64_t c = at + (u * kThreads + threadIdx.x) * kValues;
    v[u].template load<true>(m, c < size ? c : 0, c < size ? (int)min((uint64_t)kValues, size - c) : 0);
  }
  double s = 0.0;
#pragma unroll
  for (uint32_t u = 0; u < kPieces; ++u) s += squares(v[u]);
  return s;
}

template <uint32_t MOST> __global__ void __launch_bounds__(kThreads) squares_kernel(const __grid_constant__ List<MOST> list, double* parts) {
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t chunks = list.end[list.count - 1];
  double s = 0.0;
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const uint32_t g = gradient_of(list, c);
    const uint64_t at = (uint64_t)(c - (g ? list.end[g - 1] : 0)) * kChunk;
    s += list.wide[g] & 1 ? chunk_squares<float>(list.p[g], list.size[g], at) : chunk_squares<__nv_bfloat16>(list.p[g], list.size[g], at);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* parts, uint64_t count, float* norm) {
  admit_next_kernel();
  await_previous_kernel();
  double s = 0.0;
  for (uint64_t i = threadIdx.x; i < count; i += kThreads) s += parts[i];
  s = block_sum(s);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <typename G, typename D> __device__ __forceinline__ void scale_chunk(Meeting* meeting, const void* p, void* out, uint64_t size, uint64_t at, float by) {
  const Rows<G> m = rows_of<G>(p, size);
  D* const to = static_cast<D*>(out);
  const Access access = access_of<D>(out, 0);
  Values<G> v[kPieces];
#pragma unroll
  for (uint32_t u = 0; u < kPieces; ++u) {
    const uint64_t c = at + (u * kThreads + threadIdx.x) * kValues;
    v[u].template load<true>(m, c < size ? c : 0, c < size ? (int)min((uint64_t)kValues, size - c) : 0);
  }
#pragma unroll
  for (uint32_t u = 0; u < kPieces; ++u) {
    const uint64_t c = at + (u * kThreads + threadIdx.x) * kValues;
    const int have = c < size ? (int)min((uint64_t)kValues, size - c) : 0;
    float x[kValues];
#pragma unroll
    for (int i = 0; i < kValues; ++i) x[i] = v[u].get(i) * by;
    if (access == kByElement) store_values_anyhow(meeting[threadIdx.x / 32], to + (have ? c : 0), have, x);
    else store_values(to + (have ? c : 0), access, have, x);
  }
}

template <uint32_t MOST, bool IN_PLACE> __global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ List<MOST> list, const float* norm, float max_norm) {
  __shared__ Meeting meeting[kThreads / 32];
  admit_next_kernel();
  await_previous_kernel();
  const float n = *const_cast<const volatile float*>(norm), by = n <= max_norm ? 1.f : max_norm / n;
  if (IN_PLACE && by == 1.f) return;
  const uint32_t chunks = list.end[list.count - 1];
  for (uint32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const uint32_t c = chunks - 1 - i, g = gradient_of(list, c);      // what the norm read last is still in L2
    const uint64_t at = (uint64_t)(c - (g ? list.end[g - 1] : 0)) * kChunk;
    const void* p = list.p[g];
    void* out = list.out[g];
    switch (list.wide[g]) {
      case 0: scale_chunk<__nv_bfloat16, __nv_bfloat16>(meeting, p, out, list.size[g], at, by); break;
      case 1: scale_chunk<float, __nv_bfloat16>(meeting, p, out, list.size[g], at, by); break;
      case 2: scale_chunk<__nv_bfloat16, float>(meeting, p, out, list.size[g], at, by); break;
      default: scale_chunk<float, float>(meeting, p, out, list.size[g], at, by);
    }
  }
}

// The list in parts that a kernel takes, empty gradients left out: body(part, blocks).  At most 2^43 values in all, so that
// chunks count in 32 bits.
template <uint32_t MOST, typename F> cudaError_t in_parts(const Gradient* grads, uint64_t count, F&& body) {
  List<MOST> list;
  list.count = 0;
  uint32_t chunks = 0;
  for (uint64_t i = 0; i < count; ++i) {
    if (!grads[i].size) continue;
    const uint32_t k = list.count++;
    list.p[k] = grads[i].p;
    list.out[k] = grads[i].out;
    list.size[k] = grads[i].size;
    list.wide[k] = (uint8_t)((grads[i].type == kF32) | (grads[i].out_type == kF32) << 1);
    chunks += (uint32_t)((grads[i].size + kChunk - 1) / kChunk);
    list.end[k] = chunks;
    if (list.count < MOST) continue;
    const cudaError_t e = body(list, std::min(chunks, kBlocks));
    if (e != cudaSuccess) return e;
    list.count = chunks = 0;
  }
  return list.count ? body(list, std::min(chunks, kBlocks)) : cudaSuccess;
}

constexpr uint32_t kFew = 64, kMany = 960;    // gradients that one launch takes: 2 KB of parameters, and what 32 KB hold
static_assert(sizeof(List<kMany>) + 64 <= 32764, "more than kernel parameters may be");

template <uint32_t MOST> cudaError_t norm_of(const Gradient* grads, uint64_t count, float* norm, double* parts, cudaStream_t stream) {
  uint64_t used = 0;
  const cudaError_t e = in_parts<MOST>(grads, count, [&](const List<MOST>& list, uint32_t blocks) {
    double* const to = parts + used;
    used += blocks;
    return launch_overlapped(squares_kernel<MOST>, blocks, kThreads, 0, 1, stream, list, to);
  });
  return e != cudaSuccess ? e : launch_overlapped(norm_kernel, 1, kThreads, 0, 1, stream, (const double*)parts, used, norm);
}

template <uint32_t MOST> cudaError_t scale(const Gradient* grads, uint64_t count, const float* norm, float max_norm, bool in_place, cudaStream_t stream) {
  return in_parts<MOST>(grads, count, [&](const List<MOST>& list, uint32_t blocks) {
    return launch_overlapped(in_place ? scale_kernel<MOST, true> : scale_kernel<MOST, false>, blocks, kThreads, 0, 1, stream, list, norm, max_norm);
  });
}

}  // namespace

uint64_t grad_norm_workspace(uint64_t count) { return (count / kMany + 1) * kBlocks * sizeof(double); }

cudaError_t launch_grad_norm(const Gradient* grads, uint64_t count, float* norm, void* workspace, cudaStream_t stream) {
  double* parts = static_cast<double*>(workspace);
  return count <= kFew ? norm_of<kFew>(grads, count, norm, parts, stream) : norm_of<kMany>(grads, count, norm, parts, stream);
}

cudaError_t launch_grad_clip(const Gradient* grads, uint64_t count, const float* norm, float max_norm, cudaStream_t stream) {
  bool in_place = true;
  for (uint64_t i = 0; i < count; ++i) in_place = in_place && grads[i].p == grads[i].out;
  return count <= kFew ? scale<kFew>(grads, count, norm, max_norm, in_place, stream) : scale<kMany>(grads, count, norm, max_norm, in_place, stream);
}

}  // namespace rudra
