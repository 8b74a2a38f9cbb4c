// sm_100a building blocks of the two products: barriers with bounded waits, TMA and bulk copies, tensor
// memory, and the descriptors of tcgen05.mma.
#pragma once
#include <atomic>
#include <cstdint>
#include <mutex>

#include <cuda.h>
#include <cuda_bf16.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

namespace rudra {
namespace {

// ---------------------------------------------------------------------------------------- warps

// One lane of a converged warp.  The warps that issue copies and tensor operations run whole, with this lane's
// predicate on the operation alone: descriptors and addresses then live in uniform registers, where the operations
// take them from.  (Issued from a branch of one lane, a stage of the 256 x 256 tile took 1150 cycles.)
__device__ __forceinline__ uint32_t elect() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p;
}
// The same to every lane of a warp: the compiler knows that what comes out is uniform.
__device__ __forceinline__ uint32_t warp_index() { return __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0); }
__device__ __forceinline__ bool all_lanes(bool ok) { return __all_sync(0xFFFFFFFFu, ok); }

// ------------------------------------------------------------------------------------ barriers

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" :: "r"(bar), "r"(bytes), "r"(elected) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Arrives on another block's barrier; `remote`: its address in the cluster.  What stands behind such an arrival is
// read by the tensor cores, from memory that this thread has fenced for them (fence.proxy.async, or
// tcgen05.fence before and after for tensor memory), not by the thread that waits; so neither side
// asks for more than block scope.  At cluster scope every arrival drains the SM's memory traffic: the
// weight gradient of 8192 x 4096 x 4096 took 415 us instead of 241.
__device__ __forceinline__ void barrier_arrive_cluster(uint32_t remote) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(remote) : "memory");
}
// A wait of a whole warp that gives up after about two seconds.  All lanes get one answer, whichever of them gives up first:
// what follows (shuffles, tensor memory) takes whole warps.  The caller then stops issuing work and the block ends
// through its ordinary exit; the count it raises is read by rudra_learner_sync.
constexpr long long kWaitCycles = 4000000000ll;
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, long long limit = kWaitCycles) {
  if (all_lanes(barrier_try(bar, parity))) return true;
  const long long begin = clock64();
  while (!all_lanes(barrier_try(bar, parity)))
    if (!all_lanes(clock64() - begin <= limit)) return false;
  return true;
}
// The end of a loading warp that issued `issued` stages of copies over a ring of barriers at `full`: the last ones land while
// their block still has its shared memory, even if the warps that should have used them gave up and this one did
// not.  Costs nothing otherwise, for their users wait for the same.  Copies take microseconds; where a barrier waits
// for more than copies and this wait runs out too, two seconds have passed since the last of them was issued.
__device__ __forceinline__ void await_copies(uint32_t full, uint32_t issued, uint32_t ring, long long limit = kWaitCycles) {
  for (uint32_t j = issued > ring ? issued - ring : 0; j < issued; ++j)
    if (!barrier_wait(full + 8 * (j % ring), j / ring & 1, limit)) break;
}
__device__ __forceinline__ void barrier_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

// A warpgroup's registers per thread, out of those the block was launched with.
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N)); }
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N)); }

// -------------------------------------------------------------------------------------- clusters

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Whole warps.  What a thread wrote before it arrives is seen by whoever has waited.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Where another block of the cluster has what is at `at` here.
__device__ __forceinline__ uint32_t peer_address(uint32_t at, uint32_t rank) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(rank));
  return remote;
}
// Four floats from another block's shared memory, at what is address `at` here.
__device__ __forceinline__ float4 peer_load(uint32_t at, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(peer_address(at, rank)) : "memory");
  return v;
}
__device__ __forceinline__ double peer_double(uint32_t at, uint32_t rank) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(peer_address(at, rank)) : "memory");
  return v;
}
__device__ __forceinline__ float peer_value(uint32_t at, uint32_t rank) {      // one of them
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer_address(at, rank)) : "memory");
  return v;
}

// -------------------------------------------------------------------------------------- copies

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" :: "l"(m) : "memory");
}
// One box; x in elements of the map's type and a multiple of 16 bytes.
__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap* m, int x, int y, uint32_t bar, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t"
               "@q cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
               :: "r"(to), "l"(m), "r"(x), "r"(y), "r"(bar), "r"(elected) : "memory");
}
// `bytes` (a multiple of 16) from a 16-byte boundary.
__device__ __forceinline__ void copy_bulk(uint32_t to, const void* from, uint32_t bytes, uint32_t bar, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %4, 0;\n\t"
               "@q cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
               :: "r"(to), "l"(from), "r"(bytes), "r"(bar), "r"(elected) : "memory");
}

// For a pair of blocks that issue their tensor operations together (cta_group::2): a box into this block's shared
// memory that counts on the barrier at cluster address `bar`, which may be the other's.
__device__ __forceinline__ void copy_box_pair(uint32_t to, const CUtensorMap* m, int x, int y, uint32_t bar, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t"
               "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
               :: "r"(to), "l"(m), "r"(x), "r"(y), "r"(bar), "r"(elected) : "memory");
}

// ------------------------------------------------------------------------------- tensor memory

__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {   // a whole warp; slot: shared address
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(slot), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {    // a whole warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(columns));
}
// The same by a warp of both blocks of a pair.
__device__ __forceinline__ void tmem_alloc_pair(uint32_t slot, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(slot), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t base, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(columns));
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Arrives on the barrier once every tcgen05 operation this thread issued has finished.
__device__ __forceinline__ void tensor_commit(uint32_t bar, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
               :: "r"(bar), "r"(elected) : "memory");
}
// The same on the barrier at this address in both blocks of a pair (ranks 0 and 1 of a cluster of two).
__device__ __forceinline__ void tensor_commit_pair(uint32_t bar, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}"
               :: "r"(bar), "r"(elected), "h"((uint16_t)3) : "memory");
}
// 16 columns of this warp's 32 lanes: register i is column i.
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                 "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(at));
}
__device__ __forceinline__ void tmem_load8(uint32_t at, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// 128 rows of four scale bytes (512 bytes in shared memory) to four columns, repeated for the four lane groups.
__device__ __forceinline__ void scales_to_tmem(uint32_t at, uint64_t desc, uint32_t elected) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" :: "r"(at), "l"(desc), "r"(elected) : "memory");
}
__device__ __forceinline__ void scales_to_tmem_pair(uint32_t at, uint64_t desc, uint32_t elected) {   // in both blocks of a pair, each from its own
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" :: "r"(at), "l"(desc), "r"(elected) : "memory");
}

// ------------------------------------------------------------------------------------- results

template <typename G> __device__ __forceinline__ void put(G* to, float v) {
  if constexpr (sizeof(G) == 2) *to = __float2bfloat16_rn(v);
  else *to = v;
}
// For results that are larger than L2 more often than not (151 MB of weight gradients: 32.4 us against 34.5).
template <typename G> __device__ __forceinline__ void put_streaming(G* to, float v) {
  if constexpr (sizeof(G) == 2) __stcs(to, __float2bfloat16_rn(v));
  else __stcs(to, v);
}

// The end of a tile whose sum was split over the blocks of a cluster, each of which holds its part as
// [column][128 lanes] at `part`: this block adds the parts of every split-th column in rank order and writes
// them as rows of `out`.  `rows` columns and `lanes` lanes exist.  Every thread of every block calls it.
template <typename G>
__device__ __forceinline__ void join_parts(uint32_t part, uint32_t split, uint32_t rank, uint32_t rows, uint32_t lanes, G* out, uint64_t ld, bool add = false) {
  cluster_arrive();
  cluster_wait();
  const uint32_t lane = threadIdx.x % 32 * 4, step = blockDim.x / 32 * split;
  constexpr uint32_t kMost = 8;
  const bool whole = reinterpret_cast<uintptr_t>(out) % (4 * sizeof(G)) == 0 && ld % 4 == 0;
  for (uint32_t c = threadIdx.x / 32 * split + rank; c < rows; c += step) {
    float4 v[kMost];
#pragma unroll
    for (uint32_t r = 0; r < kMost; ++r)
      if (r < split) v[r] = peer_load(part + c * 512 + lane * 4, r);
    float4 s = v[0];
#pragma unroll
    for (uint32_t r = 1; r < kMost; ++r)
      if (r < split) s = make_float4(s.x + v[r].x, s.y + v[r].y, s.z + v[r].z, s.w + v[r].w);
    G* to = out + c * ld + lane;
    if (add) {      // to what is there
      if (lane < lanes) s.x += (float)to[0];
      if (lane + 1 < lanes) s.y += (float)to[1];
      if (lane + 2 < lanes) s.z += (float)to[2];
      if (lane + 3 < lanes) s.w += (float)to[3];
    }
    if (whole && lane + 3 < lanes) {      // four at once: 128x1000x4096 in 8 bits 5.5 -> 5.3 us
      if constexpr (sizeof(G) == 4) {
        *reinterpret_cast<float4*>(to) = s;
      } else {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(s.x, s.y), hi = __floats2bfloat162_rn(s.z, s.w);
        *reinterpret_cast<uint2*>(to) = make_uint2(reinterpret_cast<const uint32_t&>(lo), reinterpret_cast<const uint32_t&>(hi));
      }
      continue;
    }
    if (lane < lanes) put(to, s.x);
    if (lane + 1 < lanes) put(to + 1, s.y);
    if (lane + 2 < lanes) put(to + 2, s.z);
    if (lane + 3 < lanes) put(to + 3, s.w);
  }
  cluster_arrive();      // the parts stay until all have read them
  cluster_wait();
}

// --------------------------------------------------------------------------------- descriptors

// A shared-memory matrix in rows of 128 bytes, swizzled, 8-row groups 1024 bytes apart.  Along the
// rows: an operand whose reduction index is contiguous.
__device__ __forceinline__ uint64_t swizzled_rows(uint32_t at) {
  return (uint64_t)((at >> 4) & 0x3FFF) | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// The same rows, across them: an operand whose reduction index counts rows.  A row is 64 values wide;
// the next 64 lie `chunk` bytes on.
__device__ __forceinline__ uint64_t swizzled_columns(uint32_t at, uint32_t chunk) {
  return (uint64_t)((at >> 4) & 0x3FFF) | (uint64_t)(chunk >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// 32 rows of 16 bytes, as tcgen05.cp takes them.
__device__ __forceinline__ uint64_t scale_rows(uint32_t at) {
  return (uint64_t)((at >> 4) & 0x3FFF) | (uint64_t)(128 >> 4) << 32 | 1ull << 46;
}

// ---------------------------------------------------------------------------------------- host

constexpr uint64_t kSms = 148;   // of a B200

// cuTensorMapEncodeTiled, looked up in the driver once.
inline PFN_cuTensorMapEncodeTiled map_encoder() {
  static const PFN_cuTensorMapEncodeTiled fn = []() -> PFN_cuTensorMapEncodeTiled {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled>(p);
  }();
  return fn;
}

// What a launch asks of the current device, asked once per device: its multiprocessors, `kernel`'s leave to use
// `bytes` of shared memory, and how many clusters of 2, 4 and 8 of its blocks run at once (of 8 fewer than
// an eighth of the multiprocessors, because a cluster does not leave its part of the chip).  One static
// instance per kernel.
class Device {
 public:
  struct Facts {
    int sms;
    int clusters[4];   // of 1, 2, 4 and 8 blocks
  };
  // `registers`: those of a thread that the kernel hands around between its warpgroups, 0 if it does not.  A build that gave it
  // fewer would wait for registers that never come, and is refused.
  template <typename K> cudaError_t prepare(K* kernel, uint32_t threads, uint32_t bytes, int registers, const Facts** facts) {
    int d = 0;
    cudaError_t e = cudaGetDevice(&d);
    if (e != cudaSuccess) return e;
    if (d < 0 || d >= kMost) return cudaErrorInvalidDevice;
    if (!known_[d].load(std::memory_order_acquire)) {
      std::lock_guard<std::mutex> lock(mutex_);
      if (!known_[d].load(std::memory_order_relaxed)) {
        Facts f = {};
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&f.sms, cudaDevAttrMultiProcessorCount, d);
        cudaFuncAttributes attributes = {};
        if (e == cudaSuccess && registers) e = cudaFuncGetAttributes(&attributes, kernel);
        if (e == cudaSuccess && registers && attributes.numRegs != registers) e = cudaErrorInvalidKernelImage;
        f.clusters[0] = f.sms;
        for (int i = 1; e == cudaSuccess && i < 4; ++i) {
          cudaLaunchConfig_t cfg = {};
          cfg.gridDim = dim3(1u << i);
          cfg.blockDim = dim3(threads);
          cfg.dynamicSmemBytes = bytes;
          cudaLaunchAttribute cluster;
          cluster.id = cudaLaunchAttributeClusterDimension;
          cluster.val.clusterDim.x = 1u << i;
          cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
          cfg.attrs = &cluster;
          cfg.numAttrs = 1;
          e = cudaOccupancyMaxActiveClusters(&f.clusters[i], kernel, &cfg);
        }
        if (e != cudaSuccess) return e;
        facts_[d] = f;
        known_[d].store(true, std::memory_order_release);
      }
    }
    *facts = &facts_[d];
    return cudaSuccess;
  }

 private:
  static constexpr int kMost = 64;
  std::mutex mutex_;
  std::atomic<bool> known_[kMost] = {};
  Facts facts_[kMost];
};

// Blocks of a cluster that share a tile: the count that is done soonest, where a block's stages are its time and
// joining the parts takes as long as `join` stages.
inline uint32_t pick_split(const Device::Facts& f, uint64_t tiles, uint32_t stages, uint32_t join) {
  uint32_t best = 1, time = stages;
  for (uint32_t i = 1; i < 4; ++i) {
    const uint32_t split = 1u << i, t = (stages + split - 1) / split + join;
    if (split <= stages && tiles <= (uint64_t)f.clusters[i] && t < time) best = split, time = t;
  }
  return best;
}

// The count that kernels raise when they give up a wait, on its way to `count` behind the stream's work; and where it lies.
template <typename F> cudaError_t read_count(const F& symbol, uint32_t* count, cudaStream_t stream) {
  return cudaMemcpyFromSymbolAsync(count, symbol, sizeof(*count), 0, cudaMemcpyDeviceToHost, stream);
}
template <typename F> cudaError_t count_address(const F& symbol, const uint32_t** at) {
  void* p = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&p, symbol);
  *at = static_cast<const uint32_t*>(p);
  return e;
}

// A row-major matrix, read in boxes as it lies; what lies outside reads as zero.
inline cudaError_t encode_plain(CUtensorMap* map, CUtensorMapDataType type, const void* p, uint64_t cols, uint64_t rows, uint64_t pitch_bytes,
                                uint32_t box_cols, uint32_t box_rows) {
  const PFN_cuTensorMapEncodeTiled fn = map_encoder();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch_bytes};
  const cuuint32_t box[2] = {box_cols, box_rows}, steps[2] = {1, 1};
  return fn(map, type, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// The same in 128-byte wide boxes with the 128-byte swizzle.
inline cudaError_t encode_rows(CUtensorMap* map, CUtensorMapDataType type, uint32_t element, const void* p, uint64_t cols, uint64_t rows,
                               uint64_t pitch_bytes, uint32_t box_rows) {
  const PFN_cuTensorMapEncodeTiled fn = map_encoder();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch_bytes};
  const cuuint32_t box[2] = {128 / element, box_rows}, steps[2] = {1, 1};
  return fn(map, type, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace
}  // namespace rudra
