// Launches of the learner-side kernels: as clusters, and each allowed to start while the kernel before it ends.
#pragma once
#include <cstdint>
#include <utility>

#include <cuda_runtime.h>

namespace rudra {
namespace {

// A kernel launched this way is set up while the one before it still runs, and waits here, before it touches
// global memory, until that one and all it wrote is done.
__device__ __forceinline__ void await_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Reads, each by one instruction, of what the kernel before may have written.  They are ordered after the wait above; a
// read-only load (__ldg, or through a const __restrict__ pointer) promises that nobody writes there for as long as the
// kernel runs, which does not hold here, and may be moved above the wait.
__device__ __forceinline__ uint32_t read_byte(const uint8_t* p) {
  uint32_t v;
  asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// The same of what is read once, first to leave the caches.
__device__ __forceinline__ uint32_t read_once(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.global.cs.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint2 read_once(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.cs.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint4 read_once(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
// From here on the next kernel may be set up.
__device__ __forceinline__ void admit_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), uint32_t blocks, uint32_t threads, uint32_t smem, uint32_t cluster, cudaStream_t stream, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = cluster;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}
// The same, under the name that the 8-bit, norm and clipping kernels use; the rules hold for either.
template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kernel)(P...), uint32_t blocks, uint32_t threads, uint32_t smem, uint32_t cluster, cudaStream_t stream, A&&... args) {
  return launch_after(kernel, blocks, threads, smem, cluster, stream, std::forward<A>(args)...);
}

}  // namespace
}  // namespace rudra
