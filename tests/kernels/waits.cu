// Kernels of a test: the product kernels' waits and copies by themselves, with limits short enough to run out.
#include <cstdint>

#include "../../paper_1509_04210_b200/csrc/reports.h"
#include "../../paper_1509_04210_b200/csrc/tensor.cuh"

namespace rudra {
namespace {

__device__ void pass_cycles(long long n) {
  const long long begin = clock64();
  while (clock64() - begin < n) {}
}

// Warp 0 waits for what warp 1 does after `after` cycles (never if that is 0); the upper half of its lanes would wait longer.
__global__ void uneven_wait(long long low, long long high, long long after, uint32_t* answers) {
  __shared__ uint64_t bar;
  if (threadIdx.x == 0) barrier_init(smem_address(&bar), 1);
  __syncthreads();
  const uint32_t lane = threadIdx.x % 32;
  if (threadIdx.x < 32) {
    const bool ok = barrier_wait(smem_address(&bar), 0, lane < 16 ? low : high);
    const uint32_t all = __ballot_sync(0xFFFFFFFFu, ok);
    if (lane == 0) answers[0] = all;
  } else if (after) {
    pass_cycles(after);
    if (lane == 0) barrier_arrive(smem_address(&bar));
  }
  __syncthreads();
}

constexpr uint32_t kRing = 4, kPiece = 1024;

// Warp 0 brings `stages` pieces into a ring of four; warp 1 uses the first `used` of them and then gives up.  `arrivals`: what
// a stage's barrier counts, one of which is the loading warp's.  Out: bytes of the last pieces that have not landed once
// the loading warp is at its end, and how many cycles that end took.
__global__ void load_and_end(const uint8_t* from, uint32_t stages, uint32_t used, uint32_t arrivals, long long limit, uint32_t* missing, long long* took) {
  __shared__ alignas(128) uint8_t ring[kRing * kPiece];
  __shared__ uint64_t bars[2 * kRing];
  const uint32_t full = smem_address(bars), empty = full + 8 * kRing, lane = threadIdx.x % 32;
  for (uint32_t i = threadIdx.x; i < kRing * kPiece; i += 64) ring[i] = 0;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < kRing; ++s) {
      barrier_init(full + 8 * s, arrivals);
      barrier_init(empty + 8 * s, 1);
    }
    barrier_init_fence();
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncthreads();
  if (threadIdx.x < 32) {
    const uint32_t elected = elect();
    uint32_t issued = 0;
    for (; issued < stages; ++issued) {
      const uint32_t s = issued % kRing;
      if (!barrier_wait(empty + 8 * s, (issued / kRing & 1) ^ 1, limit)) break;
      barrier_expect(full + 8 * s, kPiece, elected);
      copy_bulk(smem_address(ring) + s * kPiece, from + issued * kPiece, kPiece, full + 8 * s, elected);
    }
    const long long begin = clock64();
    await_copies(full, issued, kRing, limit);
    if (lane == 0) *took = clock64() - begin;
    uint32_t bad = issued == stages ? 0 : 1u << 30;
    for (uint32_t j = stages > kRing ? stages - kRing : 0; j < stages; ++j)
      for (uint32_t i = lane; i < kPiece; i += 32)
        bad += reinterpret_cast<volatile uint8_t*>(ring)[j % kRing * kPiece + i] != from[j * kPiece + i];
    atomicAdd(missing, bad);
  } else {
    for (uint32_t j = 0; j < used; ++j) {
      if (!barrier_wait(full + 8 * (j % kRing), j / kRing & 1, limit)) break;
      if (lane == 0) barrier_arrive(empty + 8 * (j % kRing));
      __syncwarp();
    }
  }
  __syncthreads();
}

__device__ uint32_t g_count;

// Whether a stream is told of the count, as rudra_learner_sync does it; < 0: a CUDA error.
int told(Reports& reports, cudaStream_t stream) {
  Reports::Counts counts = {};
  unsigned long long id = 0;
  cudaError_t e = read_count(g_count, &counts[1], stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  if (e == cudaSuccess) e = cudaStreamGetId(stream, &id);
  return e == cudaSuccess ? (int)reports.fresh(0, id, counts) : -(int)e;
}

}  // namespace
}  // namespace rudra

extern "C" int run_uneven_wait(long long low, long long high, long long after, uint32_t* answers) {
  rudra::uneven_wait<<<1, 64>>>(low, high, after, answers);
  cudaError_t e = cudaGetLastError();
  return (int)(e == cudaSuccess ? cudaDeviceSynchronize() : e);
}

// from: at least 1024 * stages bytes; stages <= used + 4.
extern "C" int run_load_and_end(const uint8_t* from, uint32_t stages, uint32_t used, uint32_t arrivals, long long limit, uint32_t* missing,
                                long long* took) {
  if (stages > used + rudra::kRing) return -1;
  rudra::load_and_end<<<1, 64>>>(from, stages, used, arrivals, limit, missing, took);
  cudaError_t e = cudaGetLastError();
  return (int)(e == cudaSuccess ? cudaDeviceSynchronize() : e);
}

// Asks for two streams and the legacy one after the host set the count to `count`; a bit for each that is told.
extern "C" int run_told(uint32_t count, void* a, void* b) {
  static rudra::Reports reports;
  if (cudaMemcpyToSymbol(rudra::g_count, &count, sizeof(count)) != cudaSuccess) return -1;
  int bits = 0;
  void* const streams[3] = {a, b, nullptr};
  for (int i = 0; i < 3; ++i) {
    const int t = rudra::told(reports, static_cast<cudaStream_t>(streams[i]));
    if (t < 0) return t;
    bits |= t << i;
  }
  return bits;
}
