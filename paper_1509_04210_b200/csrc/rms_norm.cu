// Root-mean-square norm with the residual's addition, forward and backward.
//
//   s = x + residual, rounded to the matrices' dtype;  rms = sqrt(mean(s^2) + eps);  y = s w / rms
//   ds = (w dy - s m / rms^2) / rms + dsum,  m = mean(w dy s);  dw = sum over the tokens of dy s / rms
//
// The norm is taken of the rounded s, so that the backward pass, which reads s, has the forward's values; statistics and
// sums are in 32 bits.  Both passes read and write each matrix once and multiply nothing: they are bound by HBM for
// many tokens, by launch latency for few.
#include <algorithm>

#include "fp8.cuh"
#include "launch.cuh"
#include "learner.cuh"

namespace rudra {
namespace {

constexpr uint32_t kMostThreads = 512;

// Sum over the threads of a block in a fixed order; every thread gets it.  `room`: 32 floats.
__device__ __forceinline__ float block_sum(float v, float* room) {
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  __syncthreads();
  if (threadIdx.x % 32 == 0) room[threadIdx.x / 32] = v;
  __syncthreads();
  float s = threadIdx.x % 32 < blockDim.x / 32 ? room[threadIdx.x % 32] : 0.f;
#pragma unroll
  for (int d = 16; d; d /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  return s;
}

template <typename G> __device__ __forceinline__ float rounded(float v) {
  if constexpr (sizeof(G) == 4) return v;
  else return __bfloat162float(__float2bfloat16_rn(v));
}

template <typename G, bool ANY> __device__ __forceinline__ void store_any(Meeting* meeting, G* p, Access access, int have, const float (&x)[kValues]) {
  if constexpr (ANY) store_values_anyhow(meeting[threadIdx.x / 32], p, have, x);
  else store_values(p, access, have, x);
}

template <typename G, typename W> struct Forward {
  Rows<G> x, residual;     // residual.p null: none
  Rows<W> w;
  G *sum, *y;              // each null: not wanted
  uint64_t ldsum, ldy;
  uint4* codes;            // FP8 of y
  uint8_t* scales;
  uint4* kept;             // ACT8 of y
  uint8_t* kept_scales;
  uint32_t cols, nb, kt, kept_blocks, kept_pitch;
  float eps, columns;      // cols as a float
};

// What leaves of a thread's 16 values of y: column `c` of `row`, `have` of them in the row.  Whole warps.
template <typename G, typename W, bool ANY>
__device__ __forceinline__ void put_outputs(const Forward<G, W>& p, Meeting* meeting, uint64_t row, uint32_t c, int have, const float (&y)[kValues]) {
  if (p.y) store_any<G, ANY>(meeting, p.y + (have ? row * p.ldy + c : 0), access_of<G>(p.y, p.ldy), have, y);
  if (!p.codes && !p.kept) return;
  Values<float> v;
#pragma unroll
  for (int i = 0; i < kValues; ++i) v.w[i] = i < have ? __float_as_uint(y[i]) : 0u;
  const uint32_t most = block_max_bits(v.max_bits());     // of 32 values
  if (p.codes) {
    uint32_t all = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
    all = max(all, __shfl_xor_sync(0xFFFFFFFFu, all, 4));
    const uint32_t s = fp8_scale_byte(all), b = c / kFp8Block;
    const uint4 w = e4m3_codes([&](int i) { return v.get(i); }, s);
    if (b < p.nb) {
      p.codes[(row * p.nb + b) * 8 + c / kValues % 8] = w;
      if (c % kFp8Block == 0) put_fp8_scale(p.scales, row, b, p.nb, p.kt, s);
    }
  }
  if (p.kept) {
    const uint32_t s = scale_byte(most, 6), b = c / 32;
    const uint4 w = int8_codes(v, s);
    if (b < p.kept_blocks) {
      p.kept[(row * p.kept_blocks + b) * 2 + c / kValues % 2] = w;
      if (c % 32 == 0) p.kept_scales[row * p.kept_pitch + b] = (uint8_t)s;
    }
  }
}

// A block to a row of any length, read twice: the second time s where it was written.
template <typename G, typename W, bool ANY> __global__ void __launch_bounds__(kMostThreads) norm_long_kernel(const __grid_constant__ Forward<G, W> p) {
  __shared__ Meeting meeting[ANY ? kMostThreads / 32 : 1];
  __shared__ float room[32];
  admit_next_kernel();
  await_previous_kernel();
  const uint64_t row = blockIdx.x;
  const uint32_t lane = threadIdx.x % 32, step = blockDim.x * kValues;
  const uint32_t padded = max(p.nb * kFp8Block, p.kept_blocks * 32);      // columns that outputs in blocks have
  const uint64_t end = max(padded, p.cols);
  float total = 0.f;
  for (uint64_t c0 = threadIdx.x / 32 * 32 * kValues; c0 < p.cols; c0 += step) {
    const uint64_t c = c0 + lane * kValues;
    const int have = c < p.cols ? (int)min((uint64_t)kValues, p.cols - c) : 0;
    Values<G> x, r;
    x.template load<ANY>(p.x, have ? row * p.x.ld + c : 0, have);
    if (p.residual.p) r.template load<ANY>(p.residual, have ? row * p.residual.ld + c : 0, have);
    float s[kValues], part = 0.f;
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      s[i] = p.residual.p ? rounded<G>(x.get(i) + r.get(i)) : x.get(i);
      part = fmaf(s[i], s[i], part);
    }
    total += part;
    if (p.sum) store_any<G, ANY>(meeting, p.sum + (have ? row * p.ldsum + c : 0), access_of<G>(p.sum, p.ldsum), have, s);
  }
  const float inv = __frsqrt_rn(block_sum(total, room) / p.columns + p.eps);     // its barriers: s is there for all to read
  const Rows<G> again = p.sum ? Rows<G>{p.sum, p.ldsum, p.sum + (gridDim.x - 1) * p.ldsum + p.cols, access_of<G>(p.sum, p.ldsum)} : p.x;
  for (uint64_t c0 = threadIdx.x / 32 * 32 * kValues; c0 < end; c0 += step) {
    const uint64_t c = c0 + lane * kValues;
    const int have = c < p.cols ? (int)min((uint64_t)kValues, p.cols - c) : 0;
    Values<G> s;
    Values<W> w;
    s.template load<ANY>(again, have ? row * again.ld + c : 0, have);
    w.template load<ANY>(p.w, have ? c : 0, have);
    float y[kValues];
#pragma unroll
    for (int i = 0; i < kValues; ++i) y[i] = s.get(i) * inv * w.get(i);
    put_outputs<G, W, ANY>(p, meeting, row, (uint32_t)c, have, y);
  }
}

template <typename G, typename W> struct Backward {
  Rows<G> dy, s, dsum;     // dsum.p null: none
  Rows<W> w;
  G* ds;
  uint64_t ldds;
  uint64_t rows;
  uint32_t cols;
  float eps, columns;
  float2* stats;           // of a row: 1 / rms and m / rms^2
};

// A row's statistics, by a block.
template <typename G, typename W, bool ANY> __global__ void __launch_bounds__(kMostThreads) norm_stats_kernel(const __grid_constant__ Backward<G, W> p) {
  __shared__ float room[32];
  admit_next_kernel();
  await_previous_kernel();
  const uint64_t row = blockIdx.x;
  float q = 0.f, m = 0.f;
  for (uint64_t c = (uint64_t)threadIdx.x * kValues; c < p.cols; c += blockDim.x * kValues) {
    const int have = (int)min((uint64_t)kValues, p.cols - c);
    Values<G> s, dy;
    Values<W> w;
    s.template load<ANY>(p.s, row * p.s.ld + c, have);
    dy.template load<ANY>(p.dy, row * p.dy.ld + c, have);
    w.template load<ANY>(p.w, c, have);
    float q1 = 0.f, m1 = 0.f;
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      q1 = fmaf(s.get(i), s.get(i), q1);
      m1 = fmaf(dy.get(i) * w.get(i), s.get(i), m1);
    }
    q += q1;
    m += m1;
  }
  q = block_sum(q, room);
  m = block_sum(m, room);
  const float inv = __frsqrt_rn(q / p.columns + p.eps);
  if (threadIdx.x == 0) p.stats[row] = make_float2(inv, m / p.columns * inv * inv);
}

// Sums over the tokens of a strip of 32 columns: eight warps take rows in turn; strip blockIdx.x % strips, share
// blockIdx.x / strips of the rows.
template <typename G, typename W> __global__ void __launch_bounds__(256) norm_weight_kernel(const __grid_constant__ Backward<G, W> p, uint32_t strips, uint32_t shares, float* parts) {
  __shared__ float room[8][32];
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, share = blockIdx.x / strips;
  const uint64_t c = (uint64_t)(blockIdx.x % strips) * 32 + lane;
  float total = 0.f;
  if (c < p.cols)
    for (uint64_t r = share * 8 + warp; r < p.rows; r += shares * 8)
      total = fmaf((float)p.dy.p[r * p.dy.ld + c], (float)p.s.p[r * p.s.ld + c] * p.stats[r].x, total);
  room[warp][lane] = total;
  __syncthreads();
  if (warp == 0 && c < p.cols) {
    for (int i = 1; i < 8; ++i) total += room[i][lane];
    parts[(uint64_t)share * p.cols + c] = total;
  }
}

// The gradient of s from the statistics, by a block to a row.
template <typename G, typename W, bool ANY> __global__ void __launch_bounds__(kMostThreads) norm_input_kernel(const __grid_constant__ Backward<G, W> p) {
  __shared__ Meeting meeting[ANY ? kMostThreads / 32 : 1];
  admit_next_kernel();
  await_previous_kernel();
  const uint64_t row = blockIdx.x;
  const float2 stats = p.stats[row];
  for (uint64_t c0 = threadIdx.x / 32 * 32 * kValues; c0 < p.cols; c0 += blockDim.x * kValues) {
    const uint64_t c = c0 + threadIdx.x % 32 * kValues;
    const int have = c < p.cols ? (int)min((uint64_t)kValues, p.cols - c) : 0;
    Values<G> s, dy, more;
    Values<W> w;
    s.template load<ANY>(p.s, have ? row * p.s.ld + c : 0, have);
    dy.template load<ANY>(p.dy, have ? row * p.dy.ld + c : 0, have);
    w.template load<ANY>(p.w, have ? c : 0, have);
    if (p.dsum.p) more.template load<ANY>(p.dsum, have ? row * p.dsum.ld + c : 0, have);
    float d[kValues];
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      d[i] = (dy.get(i) * w.get(i) - s.get(i) * stats.y) * stats.x;
      if (p.dsum.p) d[i] += more.get(i);
    }
    store_any<G, ANY>(meeting, p.ds + (have ? row * p.ldds + c : 0), access_of<G>(p.ds, p.ldds), have, d);
  }
}

// dw: the parts of all shares added in order, by eight warps in turn.
template <typename D> __global__ void __launch_bounds__(256) norm_join_kernel(const float* parts, uint32_t shares, uint32_t cols, D* dw) {
  __shared__ float room[8][32];
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
  float total = 0.f;
  if (c < cols)
    for (uint32_t i = warp; i < shares; i += 8) total += parts[(uint64_t)i * cols + c];
  room[warp][lane] = total;
  __syncthreads();
  if (warp == 0 && c < cols) {
    for (int i = 1; i < 8; ++i) total += room[i][lane];
    if constexpr (sizeof(D) == 4) dw[c] = total;
    else dw[c] = __float2bfloat16_rn(total);
  }
}

uint32_t threads_for(uint64_t cols) {   // of a row: 16 values each
  return (uint32_t)std::min<uint64_t>(kMostThreads, ((cols + kValues - 1) / kValues + 31) / 32 * 32);
}

template <typename G, typename W> cudaError_t forward(const NormForward& n, cudaStream_t stream) {
  const uint64_t rows = n.x.rows, cols = n.x.cols;
  Forward<G, W> p = {};
  p.x = Rows<G>::of(n.x.p, rows, cols, n.x.ld, 0);
  p.residual = Rows<G>::of(n.residual.p, rows, cols, n.residual.ld, 0);
  p.w = Rows<W>::of(n.weight, 1, cols, cols, 0);
  p.sum = static_cast<G*>(n.sum.p);
  p.ldsum = n.sum.ld;
  p.y = static_cast<G*>(n.y.p);
  p.ldy = n.y.ld;
  p.codes = static_cast<uint4*>(n.fp8.codes);
  p.scales = static_cast<uint8_t*>(n.fp8.scales);
  p.kept = static_cast<uint4*>(n.kept.codes);
  p.kept_scales = static_cast<uint8_t*>(n.kept.scales);
  p.cols = (uint32_t)cols;
  p.nb = p.codes ? (uint32_t)((cols + kFp8Block - 1) / kFp8Block) : 0;
  p.kt = (p.nb + 3) / 4;
  p.kept_blocks = p.kept ? (uint32_t)((cols + 31) / 32) : 0;
  p.kept_pitch = (uint32_t)act8_scale_pitch(cols);
  p.eps = n.eps;
  p.columns = (float)cols;
  Access all = both(p.x.access, p.w.access);
  if (p.residual.p) all = both(all, p.residual.access);
  if (p.sum) all = both(all, access_of<G>(p.sum, p.ldsum));
  if (p.y) all = both(all, access_of<G>(p.y, p.ldy));
  return launch_overlapped(all == kByElement ? norm_long_kernel<G, W, true> : norm_long_kernel<G, W, false>, (uint32_t)rows,
                           threads_for(std::max<uint64_t>(cols, (uint64_t)p.nb * kFp8Block)), 0, 1, stream, p);
}

constexpr uint64_t kMostShares = 296;
// Shares of the rows whose sums for the weight are taken side by side: two blocks to an SM.
uint64_t shares_for(uint64_t rows, uint64_t cols) {
  const uint64_t strips = (cols + 31) / 32;
  return std::max<uint64_t>(1, std::min(kMostShares / std::min(strips, kMostShares), (rows + 7) / 8));
}

template <typename G, typename W> cudaError_t backward(const NormBackward& n, void* workspace, cudaStream_t stream) {
  const uint64_t rows = n.s.rows, cols = n.s.cols;
  Backward<G, W> p = {};
  p.dy = Rows<G>::of(n.dy.p, rows, cols, n.dy.ld, 0);
  p.s = Rows<G>::of(n.s.p, rows, cols, n.s.ld, 0);
  p.dsum = Rows<G>::of(n.dsum.p, rows, cols, n.dsum.ld, 0);
  p.w = Rows<W>::of(n.weight, 1, cols, cols, 0);
  p.ds = static_cast<G*>(n.ds.p);
  p.ldds = n.ds.ld;
  p.rows = rows;
  p.cols = (uint32_t)cols;
  p.eps = n.eps;
  p.columns = (float)cols;
  p.stats = static_cast<float2*>(workspace);
  Access all = both(both(p.dy.access, p.s.access), both(p.w.access, access_of<G>(p.ds, p.ldds)));
  if (p.dsum.p) all = both(all, p.dsum.access);
  const uint64_t strips = (cols + 31) / 32, shares = shares_for(rows, cols);
  float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + (rows * sizeof(float2) + 31) / 32 * 32);
  const bool any = all == kByElement;
  cudaError_t e = launch_overlapped(any ? norm_stats_kernel<G, W, true> : norm_stats_kernel<G, W, false>, (uint32_t)rows, threads_for(cols), 0, 1, stream, p);
  if (e == cudaSuccess) e = launch_overlapped(norm_weight_kernel<G, W>, (uint32_t)(strips * shares), 256, 0, 1, stream, p, (uint32_t)strips, (uint32_t)shares, parts);
  // only now: it may be written over dy
  if (e == cudaSuccess) e = launch_overlapped(any ? norm_input_kernel<G, W, true> : norm_input_kernel<G, W, false>, (uint32_t)rows, threads_for(cols), 0, 1, stream, p);
  if (e != cudaSuccess) return e;
  return n.dw_type == kBF16 ? launch_overlapped(norm_join_kernel<__nv_bfloat16>, (uint32_t)strips, 256, 0, 1, stream, parts, (uint32_t)shares, (uint32_t)cols, static_cast<__nv_bfloat16*>(n.dw))
                            : launch_overlapped(norm_join_kernel<float>, (uint32_t)strips, 256, 0, 1, stream, parts, (uint32_t)shares, (uint32_t)cols, static_cast<float*>(n.dw));
}

}  // namespace

cudaError_t launch_rms_norm(const NormForward& n, cudaStream_t stream) {
  if (n.x.type == kBF16) return n.weight_type == kBF16 ? forward<__nv_bfloat16, __nv_bfloat16>(n, stream) : forward<__nv_bfloat16, float>(n, stream);
  return n.weight_type == kBF16 ? forward<float, __nv_bfloat16>(n, stream) : forward<float, float>(n, stream);
}

uint64_t rms_norm_backward_workspace(uint64_t rows, uint64_t cols) {
  return (rows * sizeof(float2) + 31) / 32 * 32 + shares_for(rows, cols) * cols * sizeof(float);
}

cudaError_t launch_rms_norm_backward(const NormBackward& n, void* workspace, cudaStream_t stream) {
  if (n.s.type == kBF16) return n.weight_type == kBF16 ? backward<__nv_bfloat16, __nv_bfloat16>(n, workspace, stream) : backward<__nv_bfloat16, float>(n, workspace, stream);
  return n.weight_type == kBF16 ? backward<float, __nv_bfloat16>(n, workspace, stream) : backward<float, float>(n, workspace, stream);
}

}  // namespace rudra
