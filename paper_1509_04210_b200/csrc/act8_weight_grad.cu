// dw = dy^T xhat, the weight gradient of a linear layer, with xhat from its 8-bit checkpoint, on the bf16
// tensor cores.
//
// A code times its block's power of two is a bf16 number exactly, so the checkpoint is expanded to
// bf16 on its way into shared memory (eight warps, integer and bf16 instructions only) and never exists
// wide in memory.  Both operands run along tokens, the reduction, so both sit in shared memory as they
// sit in global memory, tokens as rows ("transposed" operands for the tensor core): dy arrives by TMA.
// Inputs of the layer (k) are the 128 lanes of an accumulator, outputs (n) its columns, so a warp
// writes 32 neighbouring weights whatever the alignment of dw.
//
// One block per SM walks over its tiles with two accumulators: while one is taken out the other is
// filled.  With few tiles the tokens are split over the blocks of a cluster, which add their parts in
// rank order through distributed shared memory.
//
// The tensor core truncates where it adds to an accumulator, which costs half a unit in the last place
// every 16 tokens, always towards zero.  For an f32 result an accumulator is therefore taken out every
// kChain stages and the parts are added in registers, rounding to nearest; a bf16 result keeps 16 bits
// fewer and is taken out once.
//
// dy in f32 is first cut into three bf16 matrices whose sum it is (8 bits of the significand each, an exact split),
// and dy whose rows TMA cannot read is copied to rows it can; both go through the workspace.
#include <algorithm>

#include "blocks.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

constexpr uint32_t kLanes = 128, kColumns = 256, kTokens = 64;      // a tile, and a stage of it
constexpr uint32_t kStages = 4, kStageX = kLanes * kTokens * 2, kStageDy = kColumns * kTokens * 2, kStage = kStageX + kStageDy;
// Warpgroups: 0 manages (warp 0 loads dy, warp 1 issues), 1 and 2 take results out, 3 and 4 expand, each
// every second stage.
constexpr uint32_t kThreads = 640;
constexpr uint32_t kChain = 4;       // stages in one accumulator where the result is f32
// Registers of a thread by its group, of the 96 each that the block is launched with (640 x 96 in all).
constexpr int kManageRegisters = 32, kTakeRegisters = 152, kExpandRegisters = 72;
static_assert(128 * (kManageRegisters + 2 * kTakeRegisters + 2 * kExpandRegisters) <= 640 * 96, "more registers than the block has");
constexpr uint32_t kSmem = 1024 + kStages * kStage + 256;
constexpr uint32_t kChunk = 64 * 2 * kTokens;                       // 64 values wide, kTokens rows of 128 bytes
static_assert(kLanes * kColumns * 4 <= kStages * kStage, "the parts of a split sum are kept where the stages were");

struct Params {
  const uint8_t* codes;
  const uint8_t* scales;
  void* dw;
  uint64_t lddw;
  uint32_t tokens, n, k;
  uint32_t blocks;          // of 32 values in a row of the checkpoint
  uint32_t token_stages;    // ceil(tokens / kTokens)
  uint32_t stages;          // of the whole reduction: token_stages for each of dy's planes
  uint32_t lane_tiles, tiles;
  uint32_t chain;           // stages in one accumulator
  uint32_t split;
};

__device__ uint32_t g_wait_failed;

// kind::f16: bf16 x bf16 -> f32, both operands with the reduction across rows, 128 x 256.
constexpr uint32_t kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (kColumns / 8) << 17 | (kLanes / 16) << 24;

__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t add, uint32_t elected) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(kInstruction), "r"(add), "r"(elected) : "memory");
}

// Four int8 codes to two pairs of bf16 under a scale (a pair of equal bf16).  With u the byte, its low
// seven bits set into 128 = 0x4300 give 128 + u % 128, and 0x4300 with bit 7 of u gives 128 or 256:
// their difference is the signed code.
__device__ __forceinline__ uint32_t scaled(uint32_t bytes, uint32_t scale) {   // bytes 0 and 2
  const uint32_t low = (bytes & 0x007F007Fu) | 0x43004300u, base = (bytes & 0x00800080u) | 0x43004300u;
  const __nv_bfloat162 d = __hsub2(reinterpret_cast<const __nv_bfloat162&>(low), reinterpret_cast<const __nv_bfloat162&>(base));
  const __nv_bfloat162 r = __hmul2(d, reinterpret_cast<const __nv_bfloat162&>(scale));
  return reinterpret_cast<const uint32_t&>(r);
}
__device__ __forceinline__ uint2 expand4(uint32_t w, uint32_t scale) {
  return make_uint2(scaled(__byte_perm(w, 0, 0x4140), scale), scaled(__byte_perm(w, 0, 0x4342), scale));
}
__device__ __forceinline__ uint32_t scale_pair(uint32_t s) {
  const uint32_t h = s == 255u ? 0x7FC0u : s ? s << 7 : 0x0040u;
  return h | h << 16;
}

struct Unit {   // 32 codes of one token, and their scale
  uint32_t w[8];
  uint32_t s;
};
__device__ __forceinline__ void fetch(Unit& u, const Params& p, uint32_t token, uint32_t block) {
  if (token < p.tokens && block < p.blocks) {
    const uint64_t at = (uint64_t)token * p.blocks + block;
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(u.w[0]), "=r"(u.w[1]), "=r"(u.w[2]), "=r"(u.w[3]), "=r"(u.w[4]), "=r"(u.w[5]), "=r"(u.w[6]), "=r"(u.w[7])
                 : "l"(p.codes + at * 32));
    u.s = __ldg(p.scales + at);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) u.w[i] = 0;
    u.s = 0;
  }
}

template <typename G>
__global__ void __launch_bounds__(kThreads, 1) weight_grad_kernel(const __grid_constant__ CUtensorMap dy_map, const __grid_constant__ Params p) {
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_address(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * kStage);
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages, drained = ready + 16;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 4);

  const uint32_t warp = warp_index(), lane = threadIdx.x % 32;
  const uint32_t rank = p.split > 1 ? cluster_rank() : 0;
  const uint32_t tile0 = blockIdx.x / p.split, tile_step = gridDim.x / p.split;
  const uint32_t first = (uint32_t)((uint64_t)p.stages * rank / p.split), last = (uint32_t)((uint64_t)p.stages * (rank + 1) / p.split);

  if (threadIdx.x == 0) {
    prefetch_map(&dy_map);
    for (uint32_t s = 0; s < kStages; ++s) {
      barrier_init(full + 8 * s, 1 + 4);
      barrier_init(empty + 8 * s, 1);
    }
    for (uint32_t b = 0; b < 2; ++b) {
      barrier_init(ready + 8 * b, 1);
      barrier_init(drained + 8 * b, 8);
    }
    barrier_init_fence();
  }
  if (warp == 2) tmem_alloc(smem_address(slot), 2 * kColumns);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *slot;
  bool ok = true;

  if (warp < 4) {
    give_registers<kManageRegisters>();
    if (warp == 0 && lane == 0) {
      uint32_t c = 0;
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
        const int n0 = (int)(tile / p.lane_tiles * kColumns);
        for (uint32_t i = first; i < last; ++i, ++c) {
          const uint32_t s = c % kStages, bar = full + 8 * s, at = stage0 + s * kStage + kStageX;
          if (!(ok = barrier_wait(empty + 8 * s, (c / kStages & 1) ^ 1))) break;
          barrier_expect(bar, kStageDy);
#pragma unroll
          for (uint32_t q = 0; q < kColumns / 64; ++q) copy_box(at + q * kChunk, &dy_map, n0 + 64 * (int)q, (int)(i * kTokens), bar);
        }
      }
      // given up: what is on its way has landed once every copy issued has had its time
      if (!ok)
        for (uint32_t j = c > kStages ? c - kStages : 0; j < c; ++j) barrier_wait(full + 8 * (j % kStages), j / kStages & 1);
    } else if (warp == 1) {
      const uint32_t elected = elect();
      uint32_t q = 0, s = 0, parity = 0;     // accumulators so far; stage
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
        for (uint32_t i = first; ok && i < last; ++q) {
          const uint32_t buffer = q & 1, d = tmem + buffer * kColumns, begin = i, end = min(last, i + p.chain);
          if (!(ok = all_lanes(barrier_wait(drained + 8 * buffer, (q / 2 & 1) ^ 1)))) break;
          tmem_fence_after();
          for (; i < end; ++i) {
            if (!(ok = all_lanes(barrier_wait(full + 8 * s, parity)))) break;
            tmem_fence_after();
            const uint32_t at = stage0 + s * kStage;
            const uint64_t x = swizzled_columns(at, kChunk), dy = swizzled_columns(at + kStageX, kChunk);
#pragma unroll
            for (uint32_t j = 0; j < kTokens / 16; ++j) multiply(d, x + j * (2048 / 16), dy + j * (2048 / 16), i != begin || j, elected);
            tensor_commit(empty + 8 * s, elected);
            if (++s == kStages) s = 0, parity ^= 1;
          }
          if (ok) tensor_commit(ready + 8 * buffer, elected);
        }
      }
    }
  } else if (warp < 12) {
    take_registers<kTakeRegisters>();
    const uint32_t group = warp % 4, half = (warp - 4) / 4 * 128;   // the lanes a warp may read; its columns
    const uint32_t at = tmem + (group * 32 << 16) + half;
    float* part = reinterpret_cast<float*>(smem) + half * kLanes + group * 32 + lane;   // [column][lane], once the stages are done with
    uint32_t q = 0;
    for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
      const uint32_t k = tile % p.lane_tiles * kLanes + group * 32 + lane, n = tile / p.lane_tiles * kColumns + half;
      const uint32_t have = n < p.n ? min(128u, p.n - n) : 0;
      float acc[128];
      for (uint32_t i = first; i < last; i += p.chain, ++q) {
        const uint32_t buffer = q & 1;
        if (!(ok = barrier_wait(ready + 8 * buffer, q / 2 & 1))) break;
        tmem_fence_after();
#pragma unroll
        for (uint32_t c = 0; c < 128; c += 8) {
          uint32_t r[8];
          tmem_load8(at + buffer * kColumns + c, r);
          tmem_load_wait();
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j) acc[c + j] = i == first ? __uint_as_float(r[j]) : acc[c + j] + __uint_as_float(r[j]);
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) barrier_arrive(drained + 8 * buffer);
      }
      if (p.split > 1) {
#pragma unroll
        for (uint32_t c = 0; c < 128; ++c) part[c * kLanes] = acc[c];
      } else if (k < p.k) {
        G* to = static_cast<G*>(p.dw) + (uint64_t)n * p.lddw + k;
        if (have == 128) {
#pragma unroll
          for (uint32_t c = 0; c < 128; ++c, to += p.lddw) put(to, acc[c]);
        } else {
#pragma unroll
          for (uint32_t c = 0; c < 128; ++c, to += p.lddw)
            if (c < have) put(to, acc[c]);
        }
      }
    }
  } else {
    give_registers<kExpandRegisters>();
    // a thread expands two blocks of 32 values: tokens t and t + 32 of a stage, block b
    const uint32_t mine = (warp - 12) / 4, t = warp % 4 * 8 + lane % 8, b = lane / 8;
    const uint32_t to = stage0 + (b / 2) * kChunk + t * 128, x = t % 8, u0 = b % 2 * 4, length = last - first;
    uint32_t tile = tile0, i = first;       // the next to be fetched
    auto step = [&](uint32_t by) {
      for (i += by; i >= last && tile < p.tiles; i -= length) tile += tile_step;
    };
    auto next = [&](Unit (&u)[2]) {
      if (tile < p.tiles) {
        const uint32_t token = i % p.token_stages * kTokens + t, block = tile % p.lane_tiles * (kLanes / 32) + b;
        fetch(u[0], p, token, block);
        fetch(u[1], p, token + 32, block);
      }
      step(2);
    };
    const uint32_t total = tile0 < p.tiles ? ((p.tiles - tile0 + tile_step - 1) / tile_step) * length : 0;
    Unit u[2];
    step(mine);
    next(u);
    for (uint32_t c = mine; c < total; c += 2) {
      // expanded in registers, and the next codes on their way, before the stage is free
      uint32_t w[2][16];
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h) {
        const uint32_t scale = scale_pair(u[h].s);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          const uint2 e = expand4(u[h].w[j], scale);
          w[h][2 * j] = e.x;
          w[h][2 * j + 1] = e.y;
        }
      }
      next(u);
      const uint32_t s = c % kStages;
      if (!(ok = barrier_wait(empty + 8 * s, (c / kStages & 1) ^ 1))) break;
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};"
                       :: "r"(to + s * kStage + h * 32 * 128 + ((u0 + j) ^ x) * 16), "r"(w[h][4 * j]), "r"(w[h][4 * j + 1]), "r"(w[h][4 * j + 2]),
                          "r"(w[h][4 * j + 3]) : "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) barrier_arrive(full + 8 * s);
    }
  }
  if (!ok) g_wait_failed = 1;
  __syncwarp();
  if (p.split > 1) {   // one tile to a cluster
    const uint32_t k0 = tile0 % p.lane_tiles * kLanes, n0 = tile0 / p.lane_tiles * kColumns;
    join_parts(stage0, p.split, rank, min(kColumns, p.n - n0), min(kLanes, p.k - k0), static_cast<G*>(p.dw) + (uint64_t)n0 * p.lddw + k0, p.lddw);
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 2) {
    tmem_fence_after();
    tmem_free(tmem, 2 * kColumns);
  }
}

// ------------------------------------------------------------------------------ dy that TMA can read

// Planes of bf16 with rows of `pitch` values (whole threads) and `rows` of them (whole stages, the last
// ones zero): dy itself, or the three parts of a float's significand.
template <typename G>
__global__ void __launch_bounds__(256) planes_kernel(const G* __restrict__ dy, uint64_t ld, uint32_t tokens, uint32_t n, uint32_t pitch,
                                                     uint64_t rows, Access access, uint4* __restrict__ out) {
  const uint32_t per_row = pitch / kValues;
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t row = i / per_row;
  if (row >= rows) return;
  const uint32_t c = (uint32_t)(i - row * per_row) * kValues;
  const int have = row < tokens && c < n ? (int)min((uint32_t)kValues, n - c) : 0;
  Values<G> v;
  v.load(dy + (have ? row * ld + c : 0), access, have);
  if constexpr (sizeof(G) == 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) out[row * per_row * 2 + c / 8 + h] = make_uint4(v.w[4 * h], v.w[4 * h + 1], v.w[4 * h + 2], v.w[4 * h + 3]);
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      uint32_t w[kValues / 2];
#pragma unroll
      for (int e = 0; e < kValues; ++e) {
        const uint32_t bits = v.w[e], top = bits & 0xFFFF0000u;
        // a number loses its upper eight bits to this plane; an infinity or NaN goes there whole
        const bool number = (bits & 0x7F800000u) != 0x7F800000u;
        const uint32_t mine = number ? top : top | ((bits & 0xFFFFu) ? 0x00400000u : 0u);
        v.w[e] = number ? __float_as_uint(__uint_as_float(bits) - __uint_as_float(top)) : 0u;
        w[e / 2] = e % 2 ? w[e / 2] | mine : mine >> 16;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        out[((uint64_t)q * rows + row) * per_row * 2 + c / 8 + h] = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
    }
  }
}

uint64_t plane_pitch(uint64_t n) { return (n + kValues - 1) / kValues * kValues; }
uint64_t plane_rows(uint64_t tokens) { return (tokens + kTokens - 1) / kTokens * kTokens; }
bool readable(const MatrixIn& dy) {
  return dy.type == kBF16 && reinterpret_cast<uintptr_t>(dy.p) % 16 == 0 && (dy.ld % 8 == 0 || dy.rows <= 1) && dy.ld < (1ull << 32);
}

template <typename G>
cudaError_t launch(const CUtensorMap& map, Params& p, cudaStream_t stream) {
  static Device device;
  int sms;
  const cudaError_t e = device.prepare(reinterpret_cast<const void*>(weight_grad_kernel<G>), kSmem, &sms);
  if (e != cudaSuccess) return e;
  p.chain = sizeof(G) == 4 ? kChain : p.stages;
  p.split = 1;
  while (p.split < 8 && (uint64_t)p.tiles * p.split * 2 <= (uint64_t)sms && p.stages >= p.split * 2) p.split *= 2;
  const unsigned grid = p.split > 1 ? p.tiles * p.split : std::min<unsigned>(p.tiles, (unsigned)sms);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute cluster;
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = p.split;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cfg.attrs = &cluster;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, weight_grad_kernel<G>, map, p);
}

}  // namespace

uint64_t act8_weight_grad_workspace(const MatrixIn& dy) {
  if (dy.rows == 0 || dy.cols == 0 || readable(dy)) return 0;
  return (dy.type == kF32 ? 3 : 1) * plane_rows(dy.rows) * plane_pitch(dy.cols) * 2;
}

cudaError_t launch_act8_weight_grad(const MatrixIn& dy, const Act8& saved, const MatrixOut& dw, void* workspace, cudaStream_t stream) {
  const uint64_t size = dw.type == kBF16 ? 2 : 4;
  if (dy.rows == 0) return cudaMemset2DAsync(dw.p, dw.ld * size, 0, dw.cols * size, dw.rows, stream);   // a sum over nothing
  const bool direct = readable(dy);
  const uint64_t planes = direct || dy.type == kBF16 ? 1 : 3;
  const void* from = dy.p;
  uint64_t pitch = dy.rows > 1 ? dy.ld : plane_pitch(dy.cols), rows = dy.rows;
  if (!direct) {
    from = workspace;
    pitch = plane_pitch(dy.cols);
    rows = plane_rows(dy.rows);
    const uint64_t blocks = (rows * (pitch / kValues) + 255) / 256;
    if (blocks > 0x7FFFFFFFull || planes * rows > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    if (dy.type == kF32)
      planes_kernel<float><<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const float*>(dy.p), dy.ld, (uint32_t)dy.rows, (uint32_t)dy.cols,
                                                                 (uint32_t)pitch, rows, access_of<float>(dy.p, dy.ld), static_cast<uint4*>(workspace));
    else
      planes_kernel<__nv_bfloat16><<<(unsigned)blocks, 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(dy.p), dy.ld, (uint32_t)dy.rows,
                                                                         (uint32_t)dy.cols, (uint32_t)pitch, rows,
                                                                         access_of<__nv_bfloat16>(dy.p, dy.ld), static_cast<uint4*>(workspace));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  CUtensorMap map;
  cudaError_t e = encode_rows(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, from, dy.cols, planes * rows, pitch * 2, kTokens);
  if (e != cudaSuccess) return e;
  Params p = {};
  p.codes = static_cast<const uint8_t*>(saved.codes);
  p.scales = static_cast<const uint8_t*>(saved.scales);
  p.dw = dw.p;
  p.lddw = dw.ld;
  p.tokens = (uint32_t)dy.rows;
  p.n = (uint32_t)dw.rows;
  p.k = (uint32_t)dw.cols;
  p.blocks = (p.k + 31) / 32;
  p.token_stages = (p.tokens + kTokens - 1) / kTokens;
  p.stages = p.token_stages * (uint32_t)planes;
  p.lane_tiles = (p.k + kLanes - 1) / kLanes;
  const uint64_t tiles = (uint64_t)p.lane_tiles * ((p.n + kColumns - 1) / kColumns);
  if (tiles > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
  p.tiles = (uint32_t)tiles;
  return dw.type == kBF16 ? launch<__nv_bfloat16>(map, p, stream) : launch<float>(map, p, stream);
}

}  // namespace rudra
