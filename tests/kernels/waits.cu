// Kernels of a test: the product kernels' waits and copies by themselves, with limits short enough to run out.
#include <cstdint>

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

}  // namespace
}  // namespace rudra

extern "C" int run_uneven_wait(long long low, long long high, long long after, uint32_t* answers) {
  rudra::uneven_wait<<<1, 64>>>(low, high, after, answers);
  cudaError_t e = cudaGetLastError();
  return (int)(e == cudaSuccess ? cudaDeviceSynchronize() : e);
}
