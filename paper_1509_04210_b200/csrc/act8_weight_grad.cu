// dw = dy^T xhat, the weight gradient of a linear layer, with xhat from its 8-bit checkpoint, on the bf16
// tensor cores.
//
// A code times its block's power of two is a bf16 number exactly, so the checkpoint is expanded to
// bf16 between two places in shared memory (12 or 16 warps, integer and bf16 instructions only) and never exists
// wide in memory.  Both operands run along tokens, the reduction, so both sit in shared memory as they
// sit in global memory, tokens as rows ("transposed" operands for the tensor core).  Inputs of the layer
// (k) are the 128 lanes of an accumulator, outputs (n) its columns, so a warp writes 32 neighbouring
// weights whatever the alignment of dw.
//
// What bounds a large product is shared memory: codes in and out, xhat in, dy in, and both operands read by
// the tensor core.  Two SMs therefore share a tile of 256 x 256 (each expands 128 inputs and loads
// 128 outputs' gradients), where there are enough tiles; else a block takes 128 x 128 by itself, and with few
// of those the tokens are split over the blocks of a cluster, which add their parts in rank order.
// Codes come by TMA, seven stages ahead of their use: as ordinary loads of the expanding warps they cost 100 of 315
// us at 8192 x 4096 x 4096.
//
// A block (or pair) walks over its tiles with two accumulators: while one is taken out the other is
// filled.  The tensor core truncates where it adds to an accumulator, which costs half a unit in the
// last place every 16 tokens, always towards zero.  For an f32 result an accumulator is therefore taken
// out every few stages and the parts are added in registers, rounding to nearest (509 tokens in three planes: an
// error of 8e-8 instead of 2.6e-6); a bf16 result keeps 16 bits fewer and is taken out
// once, up to 65 536 tokens.
//
// Measured: 8192 x 4096 x 4096 to bf16 212 us = 1.29 PFLOP/s, 0.78 of the measured bf16 rate (171 us if nothing had to
// be expanded; 256 tiles are 3.5 rounds of 74 pairs, which cost 4), to f32 234 us; repeated for long both run into the
// power cap (1.56 GHz) and take 248 and 274 us.  128 x 4096 x 9216 to f32 31.7 us = 4.8 TB/s of its 151 MB of results, which
// a kernel that only stores them writes in 22.8 us (6.6 TB/s): the bound is here, where loads from tensor memory and stores of
// a warp take turns, not HBM.
//
// The kernels that gather hold 64 or 128 parts of sums in a thread's registers and spill beside them: 24 bytes a thread in
// single blocks, 88 (f32 results) or 96 (bf16) in pairs.
//
// dy in f32 is first cut into three bf16 matrices whose sum it is (8 bits of the significand each, an
// exact split down to 2^-133, the last bit of bf16), and dy whose rows TMA cannot read is copied to rows it can; both go through the workspace.  The three meet
// one expansion of xhat (4096 x 2048 x 2048 to bf16 76 us; 86 with an expansion for each).
#include <algorithm>
#include <type_traits>

#include "blocks.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

constexpr uint32_t kBlockK = 128, kBlockN = 128, kTokens = 64;      // what a block holds of a stage: inputs, outputs, tokens
constexpr uint32_t kChunk = 64 * 2 * kTokens;                       // 64 values wide, kTokens rows of 128 bytes
constexpr uint32_t kStage = 2 * kChunk, kStages = 5;                // of either operand: each has its own ring of five
constexpr uint32_t kCodes = kBlockK * kTokens, kScales = 16 * kTokens, kSlots = 7;   // of the checkpoint; stages of it on their way
constexpr uint32_t kSmem = 1024 + 2 * kStages * kStage + kSlots * (kCodes + kScales) + 384;
static_assert(kSmem <= 227 * 1024, "does not fit an SM");
static_assert(kBlockN * 512 <= 2 * kStages * kStage, "the parts of a split sum are kept where the stages were");
// Stages in one accumulator where the result is f32: 8192 x 4096 x 4096 takes 259, 235 and 225 us with 4, 8 and 16, and is
// off by 1.4e-7, 2.0e-7 and 4.0e-7.
constexpr uint32_t kChain = 8;      // 2 where dy comes in three planes
// Stages, times planes, from which on a bf16 result is gathered too, at 16 % more time (2048 x 1024 positive terms: 65 536
// tokens 304 and 354 us, too small by 1.7e-4 if not gathered; 262 144 tokens 1.14 and 1.35 ms, 8.8e-4, half of what bf16 rounds off).
constexpr uint64_t kLongest = 1024;

// Warpgroups: 0 manages (warp 0 loads dy, 1 issues, 2 allocates, 3 loads codes), 1 and 2 take results out, the
// others expand, each every third or fourth stage; and the registers of a thread by its group, of those
// that the block is launched with.  GATHER: the parts of a sum are
// added in up to 128 registers of a thread.
template <bool GATHER> struct Groups {
  static constexpr uint32_t kExpanders = GATHER ? 3 : 4, kThreads = 128 * (3 + kExpanders);
  static constexpr int kLaunch = GATHER ? 80 : 72, kManage = GATHER ? 40 : 56, kTake = GATHER ? 144 : 72, kExpand = GATHER ? 48 : 72;
  static_assert(kManage + 2 * kTake + kExpanders * kExpand <= (3 + kExpanders) * kLaunch && kThreads * kLaunch <= 65536,
                "more registers than the block has");
};

// PAIR: two blocks, one tile.
template <bool PAIR> struct Tile {
  static constexpr uint32_t kK = PAIR ? 2 * kBlockK : kBlockK, kN = PAIR ? 2 * kBlockN : kBlockN;
  // kind::f16: bf16 x bf16 -> f32, both operands with the reduction across rows
  static constexpr uint32_t kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (kN / 8) << 17 | (kK / 16) << 24;
};

struct Params {
  void* dw;
  uint64_t lddw;
  uint32_t n, k;
  uint32_t stages;          // ceil(tokens / kTokens)
  uint32_t lane_tiles, tiles;
  uint32_t chain;           // stages in one accumulator
  uint32_t split;           // blocks of a cluster that share a tile's tokens
};

// dy's planes, the largest part first.
template <uint32_t PLANES> struct Planes {
  CUtensorMap map[PLANES];
};

__device__ uint32_t g_gave_up;   // counts up

template <bool PAIR> __device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t add, uint32_t elected) {
  if (PAIR)
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(Tile<PAIR>::kInstruction), "r"(add), "r"(elected) : "memory");
  else
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(Tile<PAIR>::kInstruction), "r"(add), "r"(elected) : "memory");
}
template <bool PAIR> __device__ __forceinline__ void commit(uint32_t bar, uint32_t elected) {
  if (PAIR) tensor_commit_pair(bar, elected);
  else tensor_commit(bar, elected);
}
template <bool PAIR> __device__ __forceinline__ void arrive(uint32_t bar) {   // at the first block's barrier
  if (PAIR) barrier_arrive_cluster(bar);
  else barrier_arrive(bar);
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
__device__ __forceinline__ uint32_t scale_pair(uint32_t s) {
  const uint32_t h = s == 255u ? 0x7FC0u : s ? s << 7 : 0x0040u;
  return h | h << 16;
}

// PLANES: matrices that dy is the sum of, 1 or 3.  Two stages of xhat meet all three before they are left, the smallest
// part first: added to an accumulator that already holds the largest it would be cut off (errors of 6e-7).
// Where there is one, the stages of both operands share their barriers (two sets cost a stage 0.1 us).
template <typename G, bool PAIR, uint32_t PLANES, bool GATHER>
__global__ void __launch_bounds__(Groups<GATHER>::kThreads, 1)
weight_grad_kernel(const __grid_constant__ Planes<PLANES> dy_planes, const __grid_constant__ CUtensorMap codes_map,
                   const __grid_constant__ CUtensorMap scales_map, const __grid_constant__ Params p) {
  using T = Tile<PAIR>;
  using R = Groups<GATHER>;
  constexpr uint32_t kExpanders = R::kExpanders, kGroup = PLANES == 1 ? 1 : 2;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t x0 = smem_address(smem), dy0 = x0 + kStages * kStage, codes0 = dy0 + kStages * kStage, scales0 = codes0 + kSlots * kCodes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 2 * kStages * kStage + kSlots * (kCodes + kScales));
  const uint32_t x_full = smem_address(bars), x_empty = x_full + 8 * kStages, dy_full = PLANES == 1 ? x_full : x_empty + 8 * kStages,
                 dy_empty = PLANES == 1 ? x_empty : dy_full + 8 * kStages, ready = x_empty + 24 * kStages, drained = ready + 16, coded = drained + 16, taken = coded + 8 * kSlots;
  uint32_t* slot = reinterpret_cast<uint32_t*>(bars + 4 * kStages + 4 + 2 * kSlots);

  const uint32_t warp = warp_index(), lane = threadIdx.x % 32;
  const uint32_t rank = PAIR || p.split > 1 ? cluster_rank() : 0;
  const uint32_t together = PAIR ? 2 : p.split, tile0 = blockIdx.x / together, tile_step = gridDim.x / together;
  const uint32_t first = PAIR ? 0 : (uint32_t)((uint64_t)p.stages * rank / p.split);
  const uint32_t last = PAIR ? p.stages : (uint32_t)((uint64_t)p.stages * (rank + 1) / p.split);

  if (threadIdx.x == 0) {
#pragma unroll
    for (uint32_t q = 0; q < PLANES; ++q) prefetch_map(&dy_planes.map[q]);
    prefetch_map(&codes_map);
    prefetch_map(&scales_map);
    for (uint32_t s = 0; s < kStages; ++s) {
      barrier_init(x_full + 8 * s, (PAIR ? 8 : 4) + (PLANES == 1));      // the four warps of a group of each block, and dy
      barrier_init(x_empty + 8 * s, 1);
      if (PLANES > 1) {
        barrier_init(dy_full + 8 * s, 1);
        barrier_init(dy_empty + 8 * s, 1);
      }
    }
    for (uint32_t b = 0; b < 2; ++b) {
      barrier_init(ready + 8 * b, 1);
      barrier_init(drained + 8 * b, PAIR ? 16 : 8);
    }
    for (uint32_t s = 0; s < kSlots; ++s) {
      barrier_init(coded + 8 * s, 1);
      barrier_init(taken + 8 * s, 4);
    }
    barrier_init_fence();
  }
  if (warp == 2) {
    if (PAIR) tmem_alloc_pair(smem_address(slot), 2 * T::kN);
    else tmem_alloc(smem_address(slot), 2 * T::kN);
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (PAIR) {
    cluster_arrive();
    cluster_wait();
  }
  const uint32_t tmem = *slot;
  bool ok = true;
  admit_next_kernel();
  await_previous_kernel();

  if (warp < 4) {
    give_registers<R::kManage>();
    if (warp == 0) {
      const uint32_t elected = elect(), first_full = PAIR ? peer_address(dy_full, 0) : dy_full;
      uint32_t s = 0, parity = 1, issued = 0;
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
        const int n0 = (int)(tile / p.lane_tiles * T::kN + (PAIR ? rank * kBlockN : 0));
        for (uint32_t i = first; ok && i < last; i += kGroup) {
          for (uint32_t turn = 0; ok && turn < PLANES; ++turn) {      // the smallest part first
            const CUtensorMap* dy_map = &dy_planes.map[PLANES - 1 - turn];
            for (uint32_t t = i; t < min(last, i + kGroup); ++t, ++issued) {
              const uint32_t at = dy0 + s * kStage, row = t * kTokens;
              if (!(ok = barrier_wait(dy_empty + 8 * s, parity))) break;
              if (!PAIR || rank == 0) barrier_expect(dy_full + 8 * s, (PAIR ? 2 : 1) * kStage, elected);
#pragma unroll
              for (uint32_t q = 0; q < kBlockN / 64; ++q) {
                if (PAIR) copy_box_pair(at + q * kChunk, dy_map, n0 + 64 * (int)q, (int)row, first_full + 8 * s, elected);
                else copy_box(at + q * kChunk, dy_map, n0 + 64 * (int)q, (int)row, dy_full + 8 * s, elected);
              }
              if (++s == kStages) s = 0, parity ^= 1;
            }
          }
        }
      }
      if (!PAIR || rank == 0) await_copies(dy_full, issued, kStages);      // of a pair for both blocks, which end together
    } else if (warp == 3) {
      const uint32_t elected = elect();
      uint32_t s = 0, parity = 1, issued = 0;
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
        const int k0 = (int)(tile % p.lane_tiles * T::kK + (PAIR ? rank * kBlockK : 0));
        for (uint32_t i = first; i < last; ++i, ++issued) {
          if (!(ok = barrier_wait(taken + 8 * s, parity))) break;
          barrier_expect(coded + 8 * s, kCodes + kScales, elected);
          copy_box(codes0 + s * kCodes, &codes_map, k0, (int)(i * kTokens), coded + 8 * s, elected);
          copy_box(scales0 + s * kScales, &scales_map, k0 / 512 * 16, (int)(i * kTokens), coded + 8 * s, elected);
          if (++s == kSlots) s = 0, parity ^= 1;
        }
      }
      await_copies(coded, issued, kSlots);
    } else if (warp == 1 && (!PAIR || rank == 0)) {
      const uint32_t elected = elect();
      uint32_t q = 0;     // accumulators so far
      uint32_t sx = 0, px = 0, sdy = 0, pdy = 0;
      for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
        for (uint32_t i = first; ok && i < last; ++q) {
          const uint32_t buffer = q & 1, d = tmem + buffer * T::kN, begin = i, end = min(last, i + p.chain);
          if (!(ok = barrier_wait(drained + 8 * buffer, (q / 2 & 1) ^ 1))) break;
          tmem_fence_after();
          for (; ok && i < end; i += kGroup) {
            uint32_t sg = sx, pg = px;
#pragma unroll
            for (uint32_t turn = 0; turn < PLANES; ++turn) {
              sg = sx, pg = px;
              for (uint32_t t = i; t < min(end, i + kGroup); ++t) {
                if (turn == 0 && !(ok = barrier_wait(x_full + 8 * sg, pg))) break;
                if (PLANES > 1 && !(ok = barrier_wait(dy_full + 8 * sdy, pdy))) break;
                tmem_fence_after();
                const uint64_t x = swizzled_columns(x0 + sg * kStage, kChunk), dy = swizzled_columns(dy0 + (PLANES == 1 ? sg : sdy) * kStage, kChunk);
#pragma unroll
                for (uint32_t j = 0; j < kTokens / 16; ++j)
                  multiply<PAIR>(d, x + j * (2048 / 16), dy + j * (2048 / 16), t != begin || turn || j, elected);
                if (PLANES > 1) {
                  commit<PAIR>(dy_empty + 8 * sdy, elected);
                  if (++sdy == kStages) sdy = 0, pdy ^= 1;
                }
                if (turn == PLANES - 1) commit<PAIR>(x_empty + 8 * sg, elected);
                if (++sg == kStages) sg = 0, pg ^= 1;
              }
              if (!ok) break;
            }
            sx = sg, px = pg;
          }
          if (ok) commit<PAIR>(ready + 8 * buffer, elected);
        }
      }
    }
  } else if (warp < 12) {
    if (R::kTake > R::kLaunch) take_registers<R::kTake>();
    constexpr uint32_t kMine = T::kN / 2;
    const uint32_t group = warp % 4, half = (warp - 4) / 4 * kMine;   // the lanes a warp may read; its columns
    const uint32_t at = tmem + (group * 32 << 16) + half;
    const uint32_t first_drained = PAIR ? peer_address(drained, 0) : drained;
    float* part = reinterpret_cast<float*>(smem) + half * 128 + group * 32 + lane;   // [column][lane], once the stages are done with
    uint32_t q = 0;
    for (uint32_t tile = tile0; ok && tile < p.tiles; tile += tile_step) {
      const uint32_t k = tile % p.lane_tiles * T::kK + (PAIR ? rank * kBlockK : 0) + group * 32 + lane, n = tile / p.lane_tiles * T::kN + half;
      const uint32_t have = n < p.n ? min(kMine, p.n - n) : 0;
      G* to = static_cast<G*>(p.dw) + (uint64_t)n * p.lddw + k;
      const bool mine = k < p.k;
      if (last - first <= p.chain) {       // one accumulator: straight out
        const uint32_t buffer = q++ & 1;
        if (!(ok = barrier_wait(ready + 8 * buffer, (q - 1) / 2 & 1))) break;
        tmem_fence_after();
#pragma unroll 1
        for (uint32_t c = 0; c < have; c += 16) {
          uint32_t r[16];
          tmem_load16(at + buffer * T::kN + c, r);
          tmem_load_wait();
          if (!PAIR && p.split > 1) {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) part[(c + j) * 128] = __uint_as_float(r[j]);
          } else if (mine && c + 16 <= have) {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j, to += p.lddw) put_streaming(to, __uint_as_float(r[j]));
          } else if (mine) {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j, to += p.lddw)
              if (c + j < have) put_streaming(to, __uint_as_float(r[j]));
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) arrive<PAIR>(first_drained + 8 * buffer);
      } else if constexpr (GATHER) {
        float acc[kMine];
        for (uint32_t i = first; i < last; i += p.chain, ++q) {
          const uint32_t buffer = q & 1;
          if (!(ok = barrier_wait(ready + 8 * buffer, q / 2 & 1))) break;
          tmem_fence_after();
#pragma unroll
          for (uint32_t c = 0; c < kMine; c += 8) {
            uint32_t r[8];
            tmem_load8(at + buffer * T::kN + c, r);
            tmem_load_wait();
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) acc[c + j] = i == first ? __uint_as_float(r[j]) : acc[c + j] + __uint_as_float(r[j]);
          }
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) arrive<PAIR>(first_drained + 8 * buffer);
        }
        if (!PAIR && p.split > 1) {
#pragma unroll
          for (uint32_t c = 0; c < kMine; ++c) part[c * 128] = acc[c];
        } else if (mine && have == kMine) {
#pragma unroll
          for (uint32_t c = 0; c < kMine; ++c, to += p.lddw) put_streaming(to, acc[c]);
        } else if (mine) {
#pragma unroll
          for (uint32_t c = 0; c < kMine; ++c, to += p.lddw)
            if (c < have) put_streaming(to, acc[c]);
        }
      }
    }
  } else {
    if (R::kExpand < R::kLaunch) give_registers<R::kExpand>();
    // a thread expands two blocks of 32 values: tokens t and t + 32 of a stage, block b of the four
    const uint32_t mine = (warp - 12) / 4, t = warp % 4 * 8 + lane % 8, b = lane / 8, x = t % 8;
    const uint32_t from = codes0 + t * 128 + ((2 * b) ^ x) * 16, other = ((2 * b) ^ x) % 2 ? 0u - 16 : 16;   // a block's two 16-byte pieces
    const uint32_t to = x0 + (b / 2) * kChunk + t * 128, u0 = b % 2 * 4;
    const uint32_t first_full = PAIR ? peer_address(x_full, 0) : x_full;
    const uint32_t length = last - first, total = tile0 < p.tiles ? ((p.tiles - tile0 + tile_step - 1) / tile_step) * length : 0;
    uint32_t s = mine, sparity = 0, v = mine, vparity = 0;     // stage and slot, and which turn of theirs
    uint32_t tile = tile0, i = mine;
    for (uint32_t c = mine; c < total; c += kExpanders) {
      for (; i >= length; i -= length) tile += tile_step;
      const uint32_t scale_at = scales0 + t * 16 + (tile % p.lane_tiles * (T::kK / 32) + (PAIR ? rank * 4 : 0) + b) % 16;
      i += kExpanders;
      if (!(ok = barrier_wait(coded + 8 * v, vparity) && barrier_wait(x_empty + 8 * s, sparity ^ 1))) break;
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h) {
        const uint32_t row = h * 32 * 128;
        uint32_t q[8], e;
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(e) : "r"(scale_at + v * kScales + h * 32 * 16));
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "r"(from + v * kCodes + row));
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7]) : "r"(from + v * kCodes + row + other));
        const uint32_t scale = scale_pair(e);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};"
                       :: "r"(to + s * kStage + row + ((u0 + j) ^ x) * 16), "r"(scaled(__byte_perm(q[2 * j], 0, 0x4140), scale)),
                          "r"(scaled(__byte_perm(q[2 * j], 0, 0x4342), scale)), "r"(scaled(__byte_perm(q[2 * j + 1], 0, 0x4140), scale)),
                          "r"(scaled(__byte_perm(q[2 * j + 1], 0, 0x4342), scale)) : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        arrive<PAIR>(first_full + 8 * s);
        barrier_arrive(taken + 8 * v);
      }
      if ((s += kExpanders) >= kStages) s -= kStages, sparity ^= 1;
      if ((v += kExpanders) >= kSlots) v -= kSlots, vparity ^= 1;
    }
  }
  if (!ok) atomicAdd(&g_gave_up, 1u);
  __syncwarp();
  if (!PAIR && p.split > 1) {   // one tile to a cluster
    const uint32_t k0 = tile0 % p.lane_tiles * kBlockK, n0 = tile0 / p.lane_tiles * kBlockN;
    join_parts(x0, p.split, rank, min(kBlockN, p.n - n0), min(kBlockK, p.k - k0), static_cast<G*>(p.dw) + (uint64_t)n0 * p.lddw + k0, p.lddw);
  }
  tmem_fence_before();
  __syncthreads();
  if (PAIR) {      // neither block ends while the other may still use its memory
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 2) {
    tmem_fence_after();
    if (PAIR) tmem_free_pair(tmem, 2 * T::kN);
    else tmem_free(tmem, 2 * T::kN);
  }
}

// ------------------------------------------------------------------------------ dy that TMA can read

// Planes of bf16 with rows of `pitch` values (whole threads) and `rows` of them (whole stages, the last
// ones zero): dy itself, or the three parts of a float's significand.
template <typename G>
__global__ void __launch_bounds__(256) planes_kernel(Rows<G> dy, uint32_t tokens, uint32_t n, uint32_t pitch, uint64_t rows,
                                                     uint4* out) {
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t per_row = pitch / kValues;
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t row = i / per_row;
  if (row >= rows) return;
  const uint32_t c = (uint32_t)(i - row * per_row) * kValues;
  const int have = row < tokens && c < n ? (int)min((uint32_t)kValues, n - c) : 0;
  Values<G> v;
  v.template load<true>(dy, have ? row * dy.ld + c : 0, have);
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

template <typename G, bool PAIR, uint32_t PLANES, bool GATHER>
cudaError_t launch(const CUtensorMap* dy, const CUtensorMap& codes, const CUtensorMap& scales, Params p, cudaStream_t stream) {
  using T = Tile<PAIR>;
  static Device device;
  const Device::Facts* facts;
  const cudaError_t e = device.prepare(weight_grad_kernel<G, PAIR, PLANES, GATHER>, Groups<GATHER>::kThreads, kSmem, Groups<GATHER>::kLaunch, &facts);
  if (e != cudaSuccess) return e;
  Planes<PLANES> planes;
  std::copy(dy, dy + PLANES, planes.map);
  p.chain = GATHER ? (PLANES == 1 ? kChain : 2) : p.stages;
  p.lane_tiles = (p.k + T::kK - 1) / T::kK;
  const uint64_t tiles = (uint64_t)p.lane_tiles * ((p.n + T::kN - 1) / T::kN);
  if (tiles > 0x0FFFFFFFull) return cudaErrorInvalidConfiguration;
  p.tiles = (uint32_t)tiles;
  // A stage takes 0.29 us, joining 2.6 (512 x 512 outputs: 512 tokens 7.2 us by one block a tile, 8.2 by two; 4096
  // tokens 23.5 and 12.6 by four).
  p.split = PAIR ? 1 : pick_split(*facts, tiles, p.stages, (9 + PLANES - 1) / PLANES);
  const uint32_t together = PAIR ? 2 : p.split;
  const uint32_t blocks = p.split > 1 ? p.tiles * p.split : std::min(p.tiles, (uint32_t)facts->sms / together) * together;
  return launch_after(weight_grad_kernel<G, PAIR, PLANES, GATHER>, blocks, Groups<GATHER>::kThreads, kSmem, together, stream, planes, codes, scales, p);
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
    if (blocks > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    const cudaError_t e =
        dy.type == kF32 ? launch_after(planes_kernel<float>, (uint32_t)blocks, 256, 0, 1, stream, Rows<float>::of(dy.p, dy.rows, dy.cols, dy.ld, 0),
                                       (uint32_t)dy.rows, (uint32_t)dy.cols, (uint32_t)pitch, rows, static_cast<uint4*>(workspace))
                        : launch_after(planes_kernel<__nv_bfloat16>, (uint32_t)blocks, 256, 0, 1, stream,
                                       Rows<__nv_bfloat16>::of(dy.p, dy.rows, dy.cols, dy.ld, 0), (uint32_t)dy.rows, (uint32_t)dy.cols,
                                       (uint32_t)pitch, rows, static_cast<uint4*>(workspace));
    if (e != cudaSuccess) return e;
  }
  const uint64_t nb = (dw.cols + 31) / 32, scale_pitch = act8_scale_pitch(dw.cols);
  CUtensorMap dy_maps[3], codes_map, scales_map;
  cudaError_t e = cudaSuccess;
  for (uint64_t q = 0; e == cudaSuccess && q < planes; ++q)
    e = encode_rows(&dy_maps[q], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, static_cast<const uint8_t*>(from) + q * rows * pitch * 2, dy.cols, rows, pitch * 2, kTokens);
  if (e == cudaSuccess) e = encode_rows(&codes_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, saved.codes, nb * 32, dy.rows, nb * 32, kTokens);
  if (e == cudaSuccess) e = encode_plain(&scales_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, saved.scales, scale_pitch, dy.rows, scale_pitch, 16, kTokens);
  if (e != cudaSuccess) return e;
  Params p = {};
  p.dw = dw.p;
  p.lddw = dw.ld;
  p.n = (uint32_t)dw.rows;
  p.k = (uint32_t)dw.cols;
  p.stages = (uint32_t)((dy.rows + kTokens - 1) / kTokens);
  // Pairs once the tiles of single blocks no longer fit the SMs at once (4096 tokens: 144 tiles of 1536 x 1536 27.3 us
  // and 31.7 by pairs, 256 tiles of 2048 x 2048 47.5 and 33.2).
  const bool pair = ((dw.rows + 127) / 128) * ((dw.cols + 127) / 128) > kSms;
  const auto run = [&](auto type, auto gather) {
    using G = decltype(type);
    constexpr bool GATHER = decltype(gather)::value;
    if (planes == 1)
      return pair ? launch<G, true, 1, GATHER>(dy_maps, codes_map, scales_map, p, stream) : launch<G, false, 1, GATHER>(dy_maps, codes_map, scales_map, p, stream);
    return pair ? launch<G, true, 3, GATHER>(dy_maps, codes_map, scales_map, p, stream) : launch<G, false, 3, GATHER>(dy_maps, codes_map, scales_map, p, stream);
  };
  if (dw.type == kF32) return run(float(), std::true_type());
  return p.stages * planes > kLongest ? run(__nv_bfloat16(), std::true_type()) : run(__nv_bfloat16(), std::false_type());
}

cudaError_t act8_weight_grad_gave_up(uint32_t* count, cudaStream_t stream) { return read_count(g_gave_up, count, stream); }
cudaError_t act8_weight_grad_count(const uint32_t** at) { return count_address(g_gave_up, at); }

}  // namespace rudra
