// The norm of many gradients taken together, and their scaling to a largest norm.
//
// The gradients are cut into units of consecutive values, each within one gradient, which blocks (of a small list: warps) take in
// turn.  Where the gradients lie comes as a kernel parameter, so a list costs no copy.  Squares are added in 32 bits over 16
// values, everything beyond that in 64, in an order that depends on the list alone; 16 values whose squares leave the range of a
// float are squared in 64 bits.  One read for the norm, one read and one write for the scaling: bound by HBM, less what the
// second read finds in L2; small lists by launches, and have one for both.  Measured, norm and scaling: 61 million f32 in 16
// gradients 119 us (244 MB read, 200 read again and 244 written: 5.8 TB/s; a copy reaches 6.5), 20 million bf16 in 301 gradients to
// f32 32 us, 90 thousand f32 in 48 gradients 7.2 us in one launch, 20 thousand 4.4.
#include <algorithm>

#include "launch.cuh"
#include "learner.cuh"
#include "pairs.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

// Two blocks of 512 threads to an SM, 32 values to a thread: 61 million f32 117 us, 20 million bf16 to f32 in 301 gradients 30 us; six of 256
// threads 120 and 36, eight of 256 with 16 values 124 and 33.
constexpr uint32_t kThreads = 512, kPieces = 2, kBlocksPerSm = 2, kLargeUnit = kThreads * kPieces * kValues;
constexpr uint32_t kBlocks = 148 * kBlocksPerSm;    // at most; a partial sum each
// Units that are read to stay in L2 until they are scaled: 48 MB of f32, 24 of bf16 (61 million f32 123.9 us without, 120.3 with 48 to 80 MB,
// 121.2 with 100; 20 million bf16 in their place 32.1 without, 29.3 with 24 MB, more was not measured).
constexpr uint32_t kHotUnits = 732;
constexpr uint32_t kFusedBlocks = 8, kFusedThreads = 512, kSmallUnit = 32 * kValues;   // one cluster

// Part of a list, as a kernel takes it.
template <uint32_t MOST> struct List {
  const void* p[MOST];
  void* out[MOST];
  uint64_t size[MOST];
  uint32_t end[MOST];        // units up to and with this gradient's last
  uint8_t wide[MOST];        // bit 0: f32, bit 1: its output is
  uint32_t count;
  uint32_t hot;              // units from here on are to stay in L2 between the norm and the scaling
};

// Where the gradients' units end, in shared memory: a warp finds a unit's gradient by two votes.
template <uint32_t MOST> struct Ends {
  uint32_t end[MOST];
  __device__ __forceinline__ void fill(const List<MOST>& list) {
    for (uint32_t i = threadIdx.x; i < list.count; i += blockDim.x) end[i] = list.end[i];
    __syncthreads();
  }
  // Whole warps; c is the same to them and below the last end.
  __device__ __forceinline__ uint32_t of(uint32_t count, uint32_t c, uint32_t& begin) const {
    static_assert(MOST <= 1024, "two votes of 32");
    const uint32_t lane = threadIdx.x % 32;
    const uint32_t of32 = MOST <= 32 ? 0 : __ffs(__ballot_sync(0xFFFFFFFFu, end[min(lane * 32 + 31, count - 1)] > c)) - 1;
    const uint32_t g = of32 * 32 + __ffs(__ballot_sync(0xFFFFFFFFu, end[min(of32 * 32 + lane, count - 1)] > c)) - 1;
    begin = g ? end[g - 1] : 0;
    return g;
  }
};

// Elements by which p lies past a boundary of 32 bytes.  Units begin at the boundary before a gradient, and every thread's 16 values
// at one; values before the gradient's first do not exist.
template <typename G> __device__ __host__ __forceinline__ uint32_t past_boundary(const void* p) { return (uint32_t)(reinterpret_cast<uintptr_t>(p) % 32 / sizeof(G)); }

// What of 16 values from `at` (which may be negative) on exists.
struct Span {
  int lo, hi;
  __device__ __forceinline__ Span(int64_t at, uint64_t size) {
    lo = at < 0 ? (int)-at : 0;
    hi = (int)max((int64_t)0, min((int64_t)kValues, (int64_t)size - at));
  }
  __device__ __forceinline__ bool whole() const { return lo == 0 && hi == kValues; }
};

// Sum of a thread's squares.
template <typename G> __device__ __forceinline__ double squares(const Values<G>& x) {
  Pair s(0.f);
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const Pair v(x.get(2 * i), x.get(2 * i + 1));
    s = fma(v, v, s);
  }
  const float f = s.sum();
  if (f > 1e-24f && f < 1e38f) return (double)f;      // what squares below 2^-126 lost is nothing next to it
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < kValues; ++i) d = ::fma((double)x.get(i), (double)x.get(i), d);
  return d;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
template <uint32_t THREADS> __device__ __forceinline__ double block_sum(double v) {
  __shared__ double room[THREADS / 32];
  v = warp_sum(v);
  if (threadIdx.x % 32 == 0) room[threadIdx.x / 32] = v;
  __syncthreads();
  v = room[0];
#pragma unroll
  for (uint32_t i = 1; i < THREADS / 32; ++i) v += room[i];
  return v;
}

__device__ __forceinline__ void load_to_stay(const uint32_t* q, uint32_t* r) {
  asm volatile("ld.global.L2::evict_last.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(q) : "memory");
}
__device__ __forceinline__ void store_first_out(uint32_t* q, const uint32_t* r) {
  asm volatile("st.global.L2::evict_first.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               :: "l"(q), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// Values on a boundary of 32 bytes that are read to stay in L2, to leave it first, or by themselves at a gradient's ends.
template <typename G> __device__ __forceinline__ void load_aligned(Values<G>& v, const G* p, Span span, bool hot) {
  if (span.whole()) {
    const uint32_t* const q = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < Values<G>::kWords; i += 8) {
      if (hot) load_to_stay(q + i, v.w + i);
      else Values<G>::template load32<true>(q + i, v.w + i);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < Values<G>::kWords; ++i) {
    if constexpr (sizeof(G) == 4) {
      v.w[i] = i >= span.lo && i < span.hi ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    } else {
      const uint32_t lo = 2 * i >= span.lo && 2 * i < span.hi ? reinterpret_cast<const uint16_t*>(p)[2 * i] : 0u;
      const uint32_t hi = 2 * i + 1 >= span.lo && 2 * i + 1 < span.hi ? reinterpret_cast<const uint16_t*>(p)[2 * i + 1] : 0u;
      v.w[i] = lo | hi << 16;
    }
  }
}

// Squares of PIECES times 16 values of a thread, `step` apart.
template <typename G, uint32_t PIECES> __device__ __forceinline__ double unit_squares(const void* p, uint64_t size, int64_t at, uint32_t step, bool hot) {
  at -= past_boundary<G>(p);
  Values<G> x[PIECES];
#pragma unroll
  for (uint32_t u = 0; u < PIECES; ++u) load_aligned(x[u], static_cast<const G*>(p) + (at + u * step), Span(at + u * step, size), hot);
  double s = 0.0;
#pragma unroll
  for (uint32_t u = 0; u < PIECES; ++u) s += squares(x[u]);
  return s;
}
template <uint32_t PIECES, uint32_t MOST> __device__ __forceinline__ double squares_of(const List<MOST>& list, uint32_t g, int64_t at, uint32_t step, bool hot) {
  return list.wide[g] & 1 ? unit_squares<float, PIECES>(list.p[g], list.size[g], at, step, hot) : unit_squares<__nv_bfloat16, PIECES>(list.p[g], list.size[g], at, step, hot);
}

// Outputs lie on boundaries, gradients anyhow.
template <typename G, typename D, uint32_t PIECES>
__device__ __forceinline__ void scale_unit(const void* p, void* out, uint64_t size, int64_t at, uint32_t step, float by) {
  at -= past_boundary<D>(out);
  const G* const from = static_cast<const G*>(p);
  const bool aligned = reinterpret_cast<uintptr_t>(from + at) % 32 == 0;
  Values<G> x[PIECES];
#pragma unroll
  for (uint32_t u = 0; u < PIECES; ++u) {
    const Span span(at + u * step, size);
    if (aligned || !span.whole()) load_aligned(x[u], from + (at + u * step), span, false);
    else x[u].template load<true>(Rows<G>{from, 0, from + size, kByElement}, at + u * step, kValues);
  }
#pragma unroll
  for (uint32_t u = 0; u < PIECES; ++u) {
    const Span span(at + u * step, size);
    D* const to = static_cast<D*>(out) + (at + u * step);
    Piece<D, kBy32s> y;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) y.set(i, Pair(x[u].get(2 * i), x[u].get(2 * i + 1)) * Pair(by));
    if (span.whole()) {
#pragma unroll
      for (int i = 0; i < Values<D>::kWords; i += 8) store_first_out(reinterpret_cast<uint32_t*>(to) + i, y.v.w + i);
    } else {
#pragma unroll
      for (int i = 0; i < kValues; ++i)
        if (i >= span.lo && i < span.hi) {
          if constexpr (sizeof(D) == 4) reinterpret_cast<uint32_t*>(to)[i] = y.v.w[i];
          else reinterpret_cast<uint16_t*>(to)[i] = (uint16_t)(y.v.w[i / 2] >> i % 2 * 16);
        }
    }
  }
}
template <uint32_t PIECES, uint32_t MOST> __device__ __forceinline__ void scale_of(const List<MOST>& list, uint32_t g, int64_t at, uint32_t step, float by) {
  const void* const p = list.p[g];
  void* const out = list.out[g];
  const uint64_t size = list.size[g];
  switch (list.wide[g]) {
    case 0: scale_unit<__nv_bfloat16, __nv_bfloat16, PIECES>(p, out, size, at, step, by); break;
    case 1: scale_unit<float, __nv_bfloat16, PIECES>(p, out, size, at, step, by); break;
    case 2: scale_unit<__nv_bfloat16, float, PIECES>(p, out, size, at, step, by); break;
    default: scale_unit<float, float, PIECES>(p, out, size, at, step, by);
  }
}

// Lines of a unit that were asked to stay in L2 leave it like any others; they would not otherwise, even once they are read and written first to
// leave.  (12 M values read and written over and over took 15.2 us after a clipping instead of 12.8.  Releasing costs 0.5 us where 61 million
// f32 are scaled, 0.8 with 20 million bf16.)  Whole lines: what is left of a gradient's ends is next to nothing.
template <uint32_t MOST> __device__ __forceinline__ void release(const List<MOST>& list, uint32_t g, uint64_t at) {
  constexpr uint32_t kLine = 128;
  const uint32_t element = list.wide[g] & 1 ? 4 : 2;
  const uintptr_t p = reinterpret_cast<uintptr_t>(list.p[g]), end = p + list.size[g] * element, from = (p & ~(uintptr_t)31) + at * element;
  for (uint32_t i = threadIdx.x * kLine; i < kLargeUnit * element; i += kThreads * kLine) {
    const uintptr_t line = (from & ~(uintptr_t)(kLine - 1)) + i;
    if (line >= p && line + kLine <= end) asm volatile("applypriority.global.L2::evict_normal [%0], 128;" :: "l"(line) : "memory");
  }
}

__device__ __forceinline__ float factor(float norm, float max_norm) { return norm <= max_norm ? 1.f : max_norm / norm; }

template <uint32_t MOST> __global__ void __launch_bounds__(kThreads, kBlocksPerSm) squares_kernel(const __grid_constant__ List<MOST> list, double* parts) {
  __shared__ Ends<MOST> ends;
  admit_next_kernel();
  ends.fill(list);
  const uint32_t units = list.end[list.count - 1];
  await_previous_kernel();
  double s = 0.0;
  for (uint32_t c = blockIdx.x; c < units; c += gridDim.x) {
    uint32_t begin;
    const uint32_t g = ends.of(list.count, c, begin);
    s += squares_of<kPieces>(list, g, (int64_t)(c - begin) * kLargeUnit + threadIdx.x * kValues, kThreads * kValues, c >= list.hot);
  }
  s = block_sum<kThreads>(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The norm from the parts; every thread gets it.
__device__ __forceinline__ float norm_of_parts(const double* parts, uint32_t count) {
  double s = 0.0;
  for (uint32_t i = threadIdx.x; i < count; i += kThreads) s += parts[i];
  return (float)sqrt(block_sum<kThreads>(s));
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* parts, uint32_t count, float* norm) {
  admit_next_kernel();
  await_previous_kernel();
  const float n = norm_of_parts(parts, count);
  if (threadIdx.x == 0) *norm = n;
}

// parts: the norm is their sum's and is left in *norm; null: it is there already.
template <uint32_t MOST, bool IN_PLACE>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) scale_kernel(const __grid_constant__ List<MOST> list, const double* parts, uint32_t count, float* norm, float max_norm) {
  __shared__ Ends<MOST> ends;
  admit_next_kernel();
  ends.fill(list);
  const uint32_t units = list.end[list.count - 1];
  await_previous_kernel();
  const float n = parts ? norm_of_parts(parts, count) : *const_cast<volatile float*>(norm), by = factor(n, max_norm);
  if (parts && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  const bool nothing = IN_PLACE && by == 1.f;
  const uint32_t first = nothing ? parts ? list.hot : units : 0;      // of those that there is something to do for
  for (uint32_t i = blockIdx.x; i < units - first; i += gridDim.x) {
    const uint32_t c = units - 1 - i;      // backwards: what the norm read last is still in L2
    uint32_t begin;
    const uint32_t g = ends.of(list.count, c, begin);
    if (parts && c >= list.hot) release(list, g, (uint64_t)(c - begin) * kLargeUnit);      // before it is written: results leave first
    if (!nothing) scale_of<kPieces>(list, g, (int64_t)(c - begin) * kLargeUnit + threadIdx.x * kValues, kThreads * kValues, by);
  }
}

// Both by one cluster, a warp to a unit of 512 values.
template <uint32_t MOST, bool IN_PLACE>
__global__ void __launch_bounds__(kFusedThreads) clip_kernel(const __grid_constant__ List<MOST> list, float* norm, float max_norm) {
  __shared__ Ends<MOST> ends;
  __shared__ double part;
  admit_next_kernel();
  ends.fill(list);
  const uint32_t units = list.end[list.count - 1], first = blockIdx.x * (kFusedThreads / 32) + threadIdx.x / 32, step = kFusedBlocks * (kFusedThreads / 32);
  await_previous_kernel();
  double s = 0.0;
  uint32_t begin;
  for (uint32_t c = first; c < units; c += step) {
    const uint32_t g = ends.of(list.count, c, begin);
    s += squares_of<1>(list, g, (int64_t)(c - begin) * kSmallUnit + threadIdx.x % 32 * kValues, 0, true);      // half a megabyte at most
  }
  s = block_sum<kFusedThreads>(s);
  if (threadIdx.x == 0) part = s;
  cluster_arrive();
  cluster_wait();
  s = 0.0;
#pragma unroll
  for (uint32_t r = 0; r < kFusedBlocks; ++r) s += peer_double(smem_address(&part), r);
  const float n = (float)sqrt(s), by = factor(n, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  if (!IN_PLACE || by != 1.f)
    for (uint32_t c = first; c < units; c += step) {
      const uint32_t g = ends.of(list.count, c, begin);
      scale_of<1>(list, g, (int64_t)(c - begin) * kSmallUnit + threadIdx.x % 32 * kValues, 0, by);
    }
  cluster_arrive();      // the parts stay until all have read them
  cluster_wait();
}

// The list in parts that a kernel takes, empty gradients left out: body(part, units).  At most 2^43 values in all, so that
// units count in 32 bits.
template <uint32_t MOST, typename F> cudaError_t in_parts(const Gradient* grads, uint64_t count, uint32_t unit, F&& body) {
  List<MOST> list;
  list.count = list.hot = 0;
  uint32_t units = 0;
  for (uint64_t i = 0; i < count; ++i) {
    const Gradient& g = grads[i];
    if (!g.size) continue;
    const uint32_t k = list.count++;
    list.p[k] = g.p;
    list.out[k] = g.out;
    list.size[k] = g.size;
    list.wide[k] = (uint8_t)((g.type == kF32) | (g.out_type == kF32) << 1);
    // up to 15 values more, for where units begin before it
    units += (uint32_t)((g.size + 15 + unit - 1) / unit);
    list.end[k] = units;
    if (list.count < MOST) continue;
    const cudaError_t e = body(list, units);
    if (e != cudaSuccess) return e;
    list.count = units = 0;
  }
  return list.count ? body(list, units) : cudaSuccess;
}

// Gradients that one launch takes: 1.9, 9.3 and 27.8 KB of parameters.
constexpr uint32_t kFew = 64, kSome = 320, kMany = 960;
static_assert(sizeof(List<kMany>) + 64 <= 32764, "more than kernel parameters may be");

uint32_t hot_from(uint32_t units) { return units > kHotUnits ? units - kHotUnits : 0; }

// again: the values are read once more.  Else nothing is asked to stay in L2.
template <uint32_t MOST> cudaError_t squares_to(const Gradient* grads, uint64_t count, bool again, double* parts, uint32_t* used, cudaStream_t stream) {
  *used = 0;
  return in_parts<MOST>(grads, count, kLargeUnit, [&](List<MOST>& list, uint32_t units) {
    const uint32_t blocks = std::min(units, kBlocks);
    double* const to = parts + *used;
    *used += blocks;
    list.hot = again ? hot_from(units) : units;
    return launch_overlapped(squares_kernel<MOST>, blocks, kThreads, 0, 1, stream, list, to);
  });
}
template <uint32_t MOST> cudaError_t norm_of(const Gradient* grads, uint64_t count, float* norm, double* parts, cudaStream_t stream) {
  uint32_t used;
  const cudaError_t e = squares_to<MOST>(grads, count, false, parts, &used, stream);
  return e != cudaSuccess ? e : launch_overlapped(norm_kernel, 1, kThreads, 0, 1, stream, (const double*)parts, used, norm);
}

// Units of 512 values up to which one cluster takes norm and norm's use in one launch: two to a warp.  On the GPU 20 thousand values take 4.4 us
// that way and 5.8 in two launches, 90 thousand 5.9 and 6.0, or 7.5 and 5.7 in 48 gradients, 200 thousand 8.6 and 6.3; one call after another
// from the host, whose second launch takes 1.5 us, 90 thousand in 48 gradients 7.2 and 8.7.  The rule is the host's: a captured graph of a list of 100
// to 256 units would be faster with two.
constexpr uint64_t kFusedMost = 256;

template <uint32_t MOST, bool IN_PLACE> cudaError_t clip(const Gradient* grads, uint64_t count, float* norm, float max_norm, bool known, double* parts, cudaStream_t stream) {
  uint32_t used = 0;
  if (!known) {
    uint64_t units = 0;
    for (uint64_t i = 0; i < count; ++i) units += grads[i].size ? (grads[i].size + 15 + kSmallUnit - 1) / kSmallUnit : 0;
    if (units && units <= kFusedMost && count <= MOST)
      return in_parts<MOST>(grads, count, kSmallUnit, [&](const List<MOST>& list, uint32_t) {
        return launch_overlapped(clip_kernel<MOST, IN_PLACE>, kFusedBlocks, kFusedThreads, 0, kFusedBlocks, stream, list, norm, max_norm);
      });
    if (!units) return launch_overlapped(norm_kernel, 1, kThreads, 0, 1, stream, (const double*)parts, 0u, norm);
    const cudaError_t e = squares_to<MOST>(grads, count, true, parts, &used, stream);
    if (e != cudaSuccess) return e;
  }
  return in_parts<MOST>(grads, count, kLargeUnit, [&](List<MOST>& list, uint32_t units) {
    list.hot = hot_from(units);
    return launch_overlapped(scale_kernel<MOST, IN_PLACE>, std::min(units, kBlocks), kThreads, 0, 1, stream, list, known ? (const double*)nullptr : (const double*)parts, used, norm,
                             max_norm);
  });
}

}  // namespace

uint64_t grad_norm_workspace(uint64_t count) { return (count / kSome + 1) * kBlocks * sizeof(double); }

cudaError_t launch_grad_norm(const Gradient* grads, uint64_t count, float* norm, void* workspace, cudaStream_t stream) {
  double* parts = static_cast<double*>(workspace);
  return count <= kFew ? norm_of<kFew>(grads, count, norm, parts, stream)
         : count <= kSome ? norm_of<kSome>(grads, count, norm, parts, stream) : norm_of<kMany>(grads, count, norm, parts, stream);
}

cudaError_t launch_grad_clip(const Gradient* grads, uint64_t count, float* norm, float max_norm, bool known, void* workspace, cudaStream_t stream) {
  bool in_place = true;
  for (uint64_t i = 0; i < count; ++i) in_place = in_place && grads[i].p == grads[i].out;
  double* parts = static_cast<double*>(workspace);
  const auto run = count <= kFew ? in_place ? clip<kFew, true> : clip<kFew, false>
                   : count <= kSome ? in_place ? clip<kSome, true> : clip<kSome, false> : in_place ? clip<kMany, true> : clip<kMany, false>;
  return run(grads, count, norm, max_norm, known, parts, stream);
}

}  // namespace rudra
