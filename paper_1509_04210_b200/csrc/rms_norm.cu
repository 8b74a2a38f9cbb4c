// Root-mean-square norm with the residual's addition, forward and backward.
//
//   s = x + residual, rounded to the matrices' dtype;  rms = sqrt(mean(s^2) + eps);  y = s w / rms
//   ds = (w dy - s m / rms^2) / rms + dsum,  m = mean(w dy s);  dw = sum over the tokens of dy s / rms
//
// The norm is taken of the rounded s, so that the backward pass, which reads s, has the forward's values; statistics and
// sums are in 32 bits.  Both passes read and write each matrix once and multiply nothing: they are bound by HBM for
// many tokens, by launch latency for few.  Measured at 8192 x 4096 bf16 with a residual: forward to FP8 41 us = 5.7 TB/s, to bf16 49 us
// = 5.5 TB/s, backward 50 us = 5.4 TB/s; f32 69, 95 and 91 us = 6.3, 5.6 and 5.9 TB/s; one token 3 us, 37 x 1000 f32 backward 6.4 us.
// Rows that lie anyhow are held up by their values one by one: 4000 x 4111 bf16 35 us forward and 66 backward, 8192 x 1439 25 and 41, for 20
// and 15 us of memory.  Rows of more than 16 384 values have a block each and are read twice: 1000 x 20000 bf16 37 us forward and 71 backward,
// f32 59 and 119, for 25 and 50 us of memory; fewer of them than SMs leave the others idle (16 x 1 000 000 bf16 220 and 273 us for 20).
#include <algorithm>

#include "fp8.cuh"
#include "launch.cuh"
#include "learner.cuh"
#include "norm_rows.h"
#include "pairs.cuh"
#include "tensor.cuh"

namespace rudra {
namespace {

static_assert(kPiece == kValues && kMultiprocessors == kSms, "rows are given to threads and blocks by these");

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

// Where the threads of a row meet: its warps' sums, for this row and the next.
template <typename T> using Room = T[2][32];

__device__ __forceinline__ float exchanged(float v, int d) { return v + __shfl_xor_sync(0xFFFFFFFFu, v, d); }
__device__ __forceinline__ Pair exchanged(Pair v, int d) {
  return v + Pair(__shfl_xor_sync(0xFFFFFFFFu, v.lo(), d), __shfl_xor_sync(0xFFFFFFFFu, v.hi(), d));
}

// Sums over the `warps` warps of a row in a fixed order; every thread gets them.  The next row's go to the other half of the
// room, so that one barrier a row is enough.
template <typename T> __device__ __forceinline__ T row_sum(T v, uint32_t warps, uint32_t group, uint32_t parity, Room<T>& room) {
#pragma unroll
  for (int d = 16; d; d /= 2) v = exchanged(v, d);
  if (warps == 1) return v;
  const uint32_t lane = threadIdx.x % 32, span = 1u << (32 - __clz(warps - 1)), of = lane & (span - 1);
  if (lane == 0) room[parity][threadIdx.x / 32] = v;
  asm volatile("barrier.cta.sync %0, %1;" :: "r"(group + 1), "r"(warps * 32) : "memory");
  v = of < warps ? room[parity][group * warps + of] : T{};
#pragma unroll
  for (uint32_t d = 16; d; d /= 2)
    if (d < span) v = exchanged(v, (int)d);
  return v;
}

// sum / n from 1 / n, rounded about as a division would be, at a fraction of its instructions.
__device__ __forceinline__ float mean(float sum, float n, float one_nth) {
  const float q = sum * one_nth, off = fmaf(-q, n, sum);
  return fabsf(q) < 1e30f ? fmaf(off, one_nth, q) : q;      // beyond that `off` may be no number
}

// 1 / sqrt(m) as a float and what that is off by.
struct Root {
  float hi, lo;
  __device__ __forceinline__ explicit Root(float m) {
    hi = rsqrtf(m);
    const float p = hi * hi, off = fmaf(m, p, -1.f) + m * fmaf(hi, hi, -p);     // m hi^2 - 1
    lo = fabsf(off) < 1e-6f && m < 1e30f ? -0.5f * hi * off : 0.f;               // where nothing in it overflowed or was lost
  }
  __device__ __forceinline__ float value() const { return hi + lo; }
  // s * w / sqrt(m), rounded about once: two products round twice, and turn twice as many codes of an 8-bit output into their neighbours.
  __device__ __forceinline__ Pair scaled(Pair s, Pair w) const {
    const Pair h(hi), t = s * h, off = fma(s, Pair(lo), fma(s, h, Pair(-t.lo(), -t.hi())));
    return fma(t, w, off * w);
  }
  __device__ __forceinline__ float scaled(float s, float w) const {
    const float t = s * hi, off = fmaf(s, lo, fmaf(s, hi, -t));
    return fmaf(t, w, off * w);
  }
};

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
  float eps, columns, one_nth;   // cols as a float, and its inverse
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

// The same of a row that is held: y as pairs, of the columns that a Piece has from c on.  `bytes`: 512 of the warp's.
template <Lie LIE, typename G, typename W>
__device__ __forceinline__ void put_blocks(const Forward<G, W>& p, uint8_t* bytes, uint64_t row, uint32_t c, const Pair (&y)[kPairs]) {
  const uint32_t lane = threadIdx.x % 32, c0 = LIE == kSpread ? c - lane + lane * kValues : c;     // where the 16 codes that this lane writes begin
  if (p.codes) {
    uint4 w;
    uint32_t s;
    if constexpr (LIE == kSpread) {
      // 32 lanes hold four blocks side by side; their codes go through shared memory to leave as 16 bytes a lane
      s = 0;
      __syncwarp();
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const Pair u = y[2 * b], v = y[2 * b + 1];
        const uint32_t e = fp8_scale_byte(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(larger(larger(u.lo(), u.hi()), larger(v.lo(), v.hi())))));
        const float inv = inverse_scale(e);
        const uint32_t four = e == 255u ? 0u : e4m3_codes4(u.lo() * inv, u.hi() * inv, v.lo() * inv, v.hi() * inv);
#pragma unroll
        for (int i = 0; i < 4; ++i) bytes[(4 * b + i) * 32 + lane] = (uint8_t)(four >> 8 * i);
        if (lane / 8 == b) s = e;
      }
      __syncwarp();
      w = *reinterpret_cast<const uint4*>(bytes + lane * kValues);
    } else {
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) most = larger(larger(most, y[i].lo()), y[i].hi());
      s = fp8_scale_byte(fp8_block_max_bits(__float_as_uint(most)));
      const Pair inv(inverse_scale(s));
      uint32_t r[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const Pair u = y[2 * q] * inv, v = y[2 * q + 1] * inv;
        r[q] = e4m3_codes4(u.lo(), u.hi(), v.lo(), v.hi());
      }
      w = s == 255u ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(r[0], r[1], r[2], r[3]);
    }
    const uint32_t b = c0 / kFp8Block;
    if (b < p.nb) {
      p.codes[row * (p.nb * 8) + c0 / kValues] = w;
      if (c0 % kFp8Block == 0) put_fp8_scale(p.scales, row, b, p.nb, p.kt, s);
    }
  }
  if (p.kept) {
    uint4 w;
    uint32_t s;
    if constexpr (LIE == kSpread) {
      // the lanes hold a block at a time
      constexpr float kWhole = 12582912.f;
      s = 0;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kValues; ++i) {
        const float v = i % 2 ? y[i / 2].hi() : y[i / 2].lo();
        const uint32_t e = scale_byte(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v) & 0x7FFFFFFFu), 6);
        const float code = fminf(fmaxf(fmaf(v, inverse_scale(e), kWhole), kWhole - 127.f), kWhole + 127.f);
        bytes[i * 32 + lane] = e == 255u ? 0 : (uint8_t)__float_as_uint(code);
        if (lane / 2 == i) s = e;
      }
      __syncwarp();
      w = *reinterpret_cast<const uint4*>(bytes + lane * kValues);
    } else {
      Values<float> v;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) v.w[2 * i] = __float_as_uint(y[i].lo()), v.w[2 * i + 1] = __float_as_uint(y[i].hi());
      s = scale_byte(block_max_bits(v.max_bits()), 6);
      w = int8_codes(v, s);
    }
    const uint32_t b = c0 / 32;
    if (b < p.kept_blocks) {
      p.kept[row * (p.kept_blocks * 2) + c0 / kValues] = w;
      if (c0 % 32 == 0) p.kept_scales[row * p.kept_pitch + b] = (uint8_t)s;
    }
  }
}

// The columns of a row's piece k that thread t of T has: where they begin, and how many there are.
template <Lie LIE> __device__ __forceinline__ void place(uint32_t t, uint32_t T, uint32_t k, uint32_t cols, uint32_t& c, int& have) {
  const uint32_t at = k * T + t;
  c = LIE == kSpread ? at / 32 * 32 * kValues + at % 32 : at * kValues;
  have = c >= cols ? 0 : (int)min((uint32_t)kValues, LIE == kSpread ? (cols - c + 31) / 32 : cols - c);
}
// The column of value i of thread t.
template <Lie LIE> __device__ __forceinline__ uint32_t column_of(uint32_t t, uint32_t T, uint32_t i) {
  const uint32_t at = i / kValues * T + t;
  return LIE == kSpread ? at / 32 * 32 * kValues + i % kValues * 32 + at % 32 : at * kValues + i % kValues;
}

// What a group of warps does with a row that it has in registers; weight(k) gives its k-th piece of the weight.
template <Lie LIE, int PARTS, typename G, typename W, typename F>
__device__ __forceinline__ void norm_row(const Forward<G, W>& p, const Piece<G, LIE> (&s)[PARTS], F&& weight, uint64_t row, const uint32_t (&c)[PARTS], const int (&have)[PARTS],
                                         uint32_t warps, uint32_t group, uint32_t parity, Room<float>& room, uint8_t* bytes) {
  // f32 results are the very values that the 8-bit forms are made of; of bf16 ones two products in 32 bits leave nothing to see
  constexpr bool kExact = sizeof(G) == 4;
  Pair part(0.f);
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    if (p.sum) s[k].store(p.sum + row * p.ldsum + c[k], have[k]);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) part = fma(s[k].pair(i), s[k].pair(i), part);
  }
  const Root root(mean(row_sum(part.sum(), warps, group, parity, room), p.columns, p.one_nth) + p.eps);
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    const Piece<W, LIE> w = weight(k);
    if (p.y) {
      Piece<G, LIE> out;
      const Pair r(root.value());
#pragma unroll
      for (int i = 0; i < kPairs; ++i) out.set(i, kExact ? root.scaled(s[k].pair(i), w.pair(i)) : s[k].pair(i) * r * w.pair(i));
      out.store(p.y + row * p.ldy + c[k], have[k]);
    }
    if (p.codes || p.kept) {
      Pair v[kPairs];
#pragma unroll
      for (int i = 0; i < kPairs; ++i) v[i] = root.scaled(s[k].pair(i), w.pair(i));
      put_blocks<LIE>(p, bytes, row, c[k], v);
    }
  }
}

// Rows that are held in registers, a group of `warps` warps to each, 16 * PARTS values to a thread; a block's groups walk over
// the rows.
template <typename G, typename W, Lie LIE, int PARTS>
__global__ void __launch_bounds__(PARTS == 2 ? 512 : LIE == kSpread ? 1024 : 768) norm_kernel(const __grid_constant__ Forward<G, W> p, uint32_t rows, uint32_t warps) {
  static_assert(LIE != kSpread || PARTS == 1, "rows that lie anyhow are held with 16 values to a thread");
  __shared__ alignas(16) uint8_t bytes[LIE == kSpread ? 32 : 1][512];
  __shared__ Room<float> room;
  admit_next_kernel();
  const uint32_t warp = threadIdx.x / 32, group = warp / warps, groups = blockDim.x / 32 / warps, T = warps * 32, t = threadIdx.x - group * T;
  uint32_t c[PARTS];
  int have[PARTS];
#pragma unroll
  for (int k = 0; k < PARTS; ++k) place<LIE>(t, T, k, p.cols, c[k], have[k]);
  await_previous_kernel();
  uint32_t parity = 0;
  for (uint64_t row = blockIdx.x * groups + group; row < rows; row += (uint64_t)gridDim.x * groups, parity ^= 1) {
    Piece<G, LIE> s[PARTS];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      s[k].load(p.x.p + row * p.x.ld + c[k], have[k]);
      if (p.residual.p) {
        Piece<G, LIE> r;
        r.load(p.residual.p + row * p.residual.ld + c[k], have[k]);
        s[k].add(s[k], r);
      }
    }
    const auto weight = [&](int k) {
      Piece<W, LIE> w;
      w.load(p.w.p + c[k], have[k]);
      return w;
    };
    norm_row<LIE, PARTS>(p, s, weight, row, c, have, warps, group, parity, room, bytes[LIE == kSpread ? warp : 0]);
  }
}

// ------------------------------------------------------------------------------------------------
// Many rows whose memory bulk copies can read: a warp keeps a ring of slots filled, each with a row for every group, and the
// groups never wait for memory.  (8192 x 4096 bf16 to FP8 41 us = 5.7 TB/s; 50 with loads by the groups themselves, which take
// turns with their arithmetic.)

__device__ uint32_t g_gave_up;   // counts up

// The copying warp: slot by slot a row of each matrix for every group.  LANES: by a lane for each group (16384 x 512 without residual 7.7 us, and
// 8.8 by one lane); else by one for all, with addresses that are the same to the warp (8192 x 4096 to FP8 41.0 us, and 42.3 in a
// kernel that could do either).  `bars`: full barriers, then empty ones.
template <bool LANES, typename... P> __device__ __forceinline__ bool fill_ring(const Ring& ring, uint32_t ring0, uint32_t bars, uint64_t rows, const P&... matrices) {
  const uint32_t elected = elect(), lane = threadIdx.x % 32, full = bars, empty = bars + 8 * ring.slots;
  uint32_t s = 0, parity = 1, issued = 0;
  bool ok = true;
  for (uint64_t first = (uint64_t)blockIdx.x * ring.groups; first < rows; first += (uint64_t)gridDim.x * ring.groups, ++issued) {
    if (!(ok = barrier_wait(empty + 8 * s, parity))) break;
    const uint32_t n = (uint32_t)min((uint64_t)ring.groups, rows - first), bar = full + 8 * s, slot = ring0 + s * ring.slot();
    barrier_expect(bar, n * ring.matrices * ring.row, elected);
    uint32_t to = slot;
    if constexpr (LANES) {
      __syncwarp();
      to += lane * ring.matrices * ring.pitch;
      const auto copy = [&](const auto& m) {
        if (!m.p) return;
        copy_bulk(to, m.p + (first + (lane < n ? lane : 0)) * m.ld, ring.row, bar, lane < n);
        to += ring.pitch;
      };
      (copy(matrices), ...);
    } else {
      for (uint32_t g = 0; g < n; ++g) {
        const auto copy = [&](const auto& m) {
          if (!m.p) return;
          copy_bulk(to, m.p + (first + g) * m.ld, ring.row, bar, elected);
          to += ring.pitch;
        };
        (copy(matrices), ...);
      }
    }
    if (++s == ring.slots) s = 0, parity ^= 1;
  }
  await_copies(full, issued, ring.slots);
  return ok;
}
__device__ __forceinline__ void prepare_ring(const Ring& ring, uint32_t bars, uint32_t users) {
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < ring.slots; ++s) {
      barrier_init(bars + 8 * s, 1);
      barrier_init(bars + 8 * (ring.slots + s), users);
    }
    barrier_init_fence();
  }
  __syncthreads();
}
// The warp has what it wanted of the slot.
__device__ __forceinline__ void leave_slot(const Ring& ring, uint32_t bars, uint32_t s) {
  __syncwarp();
  if (threadIdx.x % 32 == 0) barrier_arrive(bars + 8 * (ring.slots + s));
}

// A wait that was given up leaves a group working on what the slot holds, so that its barriers are complete; the count tells.
template <typename G, typename W, Lie LIE, int PARTS>
__global__ void __launch_bounds__(kForwardWarps * 32 + 32) norm_staged_kernel(const __grid_constant__ Forward<G, W> p, uint32_t rows, uint32_t warps, const __grid_constant__ Ring ring) {
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ Room<float> room;
  __shared__ alignas(8) uint64_t barriers[2 * kMostSlots];
  const uint32_t bars = smem_address(barriers), warp = warp_index(), group = warp / warps, T = warps * 32, t = threadIdx.x - group * T;
  admit_next_kernel();
  prepare_ring(ring, bars, ring.groups * warps);
  await_previous_kernel();
  bool ok = true;
  if (warp == ring.groups * warps) {
    ok = fill_ring<PARTS == 1>(ring, smem_address(slots), bars, rows, p.x, p.residual);      // 16 values to a thread: short rows, many groups
  } else {
    uint32_t c[PARTS];
    int have[PARTS];
    Piece<W, LIE> w[PARTS];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      place<LIE>(t, T, k, p.cols, c[k], have[k]);
      w[k].load(p.w.p + c[k], have[k]);
    }
    uint32_t slot = 0, phase = 0, parity = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * ring.groups; first < rows; first += (uint64_t)gridDim.x * ring.groups, parity ^= 1) {
      if (ok) ok = barrier_wait(bars + 8 * slot, phase);
      const uint64_t row = first + group;
      if (row < rows) {
        const G* x = reinterpret_cast<const G*>(slots + slot * ring.slot() + group * ring.matrices * ring.pitch);
        Piece<G, LIE> s[PARTS];
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          s[k].fetch(x + c[k], have[k]);
          if (p.residual.p) {
            Piece<G, LIE> r;
            r.fetch(x + ring.pitch / sizeof(G) + c[k], have[k]);
            s[k].add(s[k], r);
          }
        }
        leave_slot(ring, bars, slot);
        norm_row<LIE, PARTS>(p, s, [&](int k) { return w[k]; }, row, c, have, warps, group, parity, room, nullptr);
      } else {
        leave_slot(ring, bars, slot);
      }
      if (++slot == ring.slots) slot = 0, phase ^= 1;
    }
  }
  if (!ok) atomicAdd(&g_gave_up, 1u);
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
  const Root root(mean(block_sum(total, room), p.columns, p.one_nth) + p.eps);     // its barriers: s is there for all to read
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
    for (int i = 0; i < kValues; ++i) y[i] = root.scaled(s.get(i), w.get(i));
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
  float eps, columns, one_nth;
  float2* stats;           // of a row: 1 / rms and m / rms^2
};

template <int PARTS> __device__ __forceinline__ float total_of(const Pair (&total)[PARTS][kPairs], int k, int i) {
  return i % 2 ? total[k][i / 2].hi() : total[k][i / 2].lo();
}
// The groups' sums for the weight added in order, to the first group's place in `sums`: value i of thread t at i * T + t.  All
// threads of the block; those of no group come with group = groups.
template <int PARTS>
__device__ __forceinline__ void join_groups(float* sums, const Pair (&total)[PARTS][kPairs], uint32_t group, uint32_t groups, uint32_t T, uint32_t t) {
  const uint32_t all = PARTS * kValues * T;
  if (group < groups)
#pragma unroll
    for (int k = 0; k < PARTS; ++k)
#pragma unroll
      for (int i = 0; i < kValues; ++i) sums[group * all + (k * kValues + i) * T + t] = total_of(total, k, i);
  __syncthreads();
  for (uint32_t j = threadIdx.x; j < all; j += blockDim.x) {
    float v = sums[j];
#pragma unroll 4
    for (uint32_t g = 1; g < groups; ++g) v += sums[g * all + j];
    sums[j] = v;
  }
  __syncthreads();
}
// A block's part to where the next kernel adds them.
template <int PARTS>
__device__ __forceinline__ void put_part(float* parts, const float* sums, const Pair (&total)[PARTS][kPairs], uint32_t groups, uint32_t T, uint32_t t, bool mine) {
  const uint32_t all = PARTS * kValues * T;
  float* const to = parts + (uint64_t)blockIdx.x * all;
  if (groups > 1) {
    for (uint32_t j = threadIdx.x; j < all; j += blockDim.x) to[j] = sums[j];
  } else if (mine) {
#pragma unroll
    for (int k = 0; k < PARTS; ++k)
#pragma unroll
      for (int i = 0; i < kValues; ++i) to[(k * kValues + i) * T + t] = total_of(total, k, i);
  }
}

__device__ __forceinline__ void put_weight(void* dw, GradType type, uint64_t column, float v) {
  if (type == kBF16) static_cast<__nv_bfloat16*>(dw)[column] = __float2bfloat16_rn(v);
  else static_cast<float*>(dw)[column] = v;
}

// Both gradients from rows that are held in registers, a group of `warps` warps to each, 16 * PARTS values to a thread.  A
// block's groups walk over the rows and add up what the rows give for the weight; at the end the groups' sums are added in order
// in shared memory and leave as one part, value i of thread t at i * T + t (T threads to a row).  CLUSTER: the blocks
// are one cluster, which adds the parts itself.
template <typename G, typename W, Lie LIE, int PARTS, bool CLUSTER, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS) norm_backward_kernel(const __grid_constant__ Backward<G, W> p, uint32_t warps, float* parts, void* dw, GradType dw_type) {
  constexpr bool kAhead = sizeof(G) == 2 && PARTS == 1 && LIE != kSpread;      // where registers do for two rows
  __shared__ Room<Pair> room;
  extern __shared__ float sums[];
  admit_next_kernel();
  const uint32_t warp = threadIdx.x / 32, group = warp / warps, groups = blockDim.x / 32 / warps, T = warps * 32, t = threadIdx.x - group * T;
  uint32_t c[PARTS];
  int have[PARTS];
  Piece<W, LIE> w[PARTS];
  Piece<G, LIE> s[PARTS], dy[PARTS], more[PARTS];
  uint64_t row = blockIdx.x * groups + group;
  const uint64_t step = (uint64_t)gridDim.x * groups;
  const G *from_s = p.s.p + row * p.s.ld, *from_dy = p.dy.p + row * p.dy.ld, *from_more = p.dsum.p + row * p.dsum.ld;     // of the row to be loaded next
  G* ds = p.ds + row * p.ldds;
#pragma unroll
  for (int k = 0; k < PARTS; ++k) place<LIE>(t, T, k, p.cols, c[k], have[k]);
  const auto load = [&](Piece<G, LIE> (&vs)[PARTS], Piece<G, LIE> (&vd)[PARTS], Piece<G, LIE> (&vm)[PARTS]) {
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      vs[k].load(from_s + c[k], have[k]);
      vd[k].load(from_dy + c[k], have[k]);
      if (p.dsum.p) vm[k].load(from_more + c[k], have[k]);
    }
    from_s += step * p.s.ld;
    from_dy += step * p.dy.ld;
    from_more += step * p.dsum.ld;
  };
  await_previous_kernel();
  Pair total[PARTS][kPairs];
#pragma unroll
  for (int k = 0; k < PARTS; ++k)
#pragma unroll
    for (int i = 0; i < kPairs; ++i) total[k][i] = Pair(0.f);
  if (row < p.rows) load(s, dy, more);
#pragma unroll
  for (int k = 0; k < PARTS; ++k) w[k].load(p.w.p + c[k], have[k]);
  for (uint32_t parity = 0; row < p.rows; row += step, parity ^= 1) {
    Piece<G, LIE> s1[PARTS], dy1[PARTS], more1[PARTS];
    if (kAhead && row + step < p.rows) load(s1, dy1, more1);
    Pair squares(0.f), inner(0.f);
#pragma unroll
    for (int k = 0; k < PARTS; ++k)
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const Pair a = s[k].pair(i);
        squares = fma(a, a, squares);
        inner = fma(dy[k].pair(i) * w[k].pair(i), a, inner);
      }
    const Pair both = row_sum(Pair(squares.sum(), inner.sum()), warps, group, parity, room);
    const float inv = Root(mean(both.lo(), p.columns, p.one_nth) + p.eps).value();
    const Pair root(inv), m(-(mean(both.hi(), p.columns, p.one_nth) * inv * inv * inv));
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      Piece<G, LIE> out;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const Pair a = s[k].pair(i), b = dy[k].pair(i) * root;
        total[k][i] = fma(a, b, total[k][i]);
        out.set(i, fma(b, w[k].pair(i), p.dsum.p ? fma(a, m, more[k].pair(i)) : a * m));
      }
      out.store(ds + c[k], have[k]);
    }
    ds += step * p.ldds;
    if (kAhead) {
#pragma unroll
      for (int k = 0; k < PARTS; ++k) s[k] = s1[k], dy[k] = dy1[k], more[k] = more1[k];
    } else if (row + step < p.rows) {
      load(s, dy, more);
    }
  }
  const uint32_t all = PARTS * kValues * T;
  if (groups > 1 || CLUSTER) join_groups<PARTS>(sums, total, group, groups, T, t);
  if (CLUSTER) {
    const uint32_t blocks = gridDim.x, rank = blocks > 1 ? cluster_rank() : 0;
    if (blocks > 1) {
      cluster_arrive();
      cluster_wait();
    }
    const uint32_t at = smem_address(sums);
    for (uint32_t j = rank * blockDim.x + threadIdx.x; j < all; j += blocks * blockDim.x) {
      float part[kMostCluster], v = 0.f;
#pragma unroll
      for (uint32_t b = 0; b < kMostCluster; ++b) part[b] = b >= blocks ? 0.f : blocks > 1 ? peer_value(at + 4 * j, b) : sums[j];
#pragma unroll
      for (uint32_t b = 0; b < kMostCluster; ++b) v += part[b];
      const uint32_t column = column_of<LIE>(j % T, T, j / T);
      if (column < p.cols) put_weight(dw, dw_type, column, v);
    }
    if (blocks > 1) {      // the sums stay until all have read them
      cluster_arrive();
      cluster_wait();
    }
    return;
  }
  put_part<PARTS>(parts, sums, total, groups, T, t, true);
}

template <typename G, typename W, Lie LIE, int PARTS>
__global__ void __launch_bounds__((PARTS == 1 ? kBackwardWarps : 16) * 32 + 32) norm_backward_staged_kernel(const __grid_constant__ Backward<G, W> p, uint32_t warps, float* parts, const __grid_constant__ Ring ring) {
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ Room<Pair> room;
  __shared__ alignas(8) uint64_t barriers[2 * kMostSlots];
  const uint32_t bars = smem_address(barriers), warp = warp_index(), group = warp / warps, T = warps * 32, t = threadIdx.x - group * T;
  admit_next_kernel();
  prepare_ring(ring, bars, ring.groups * warps);
  await_previous_kernel();
  bool ok = true;
  Pair total[PARTS][kPairs];
#pragma unroll
  for (int k = 0; k < PARTS; ++k)
#pragma unroll
    for (int i = 0; i < kPairs; ++i) total[k][i] = Pair(0.f);
  if (warp == ring.groups * warps) {
    ok = fill_ring<false>(ring, smem_address(slots), bars, p.rows, p.s, p.dy, p.dsum);
  } else {
    uint32_t c[PARTS];
    int have[PARTS];
    Piece<W, LIE> w[PARTS];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      place<LIE>(t, T, k, p.cols, c[k], have[k]);
      w[k].load(p.w.p + c[k], have[k]);
    }
    uint32_t slot = 0, phase = 0, parity = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * ring.groups; first < p.rows; first += (uint64_t)gridDim.x * ring.groups, parity ^= 1) {
      if (ok) ok = barrier_wait(bars + 8 * slot, phase);
      const uint64_t row = first + group;
      if (row < p.rows) {
        const G* from = reinterpret_cast<const G*>(slots + slot * ring.slot() + group * ring.matrices * ring.pitch);
        const uint32_t next = ring.pitch / sizeof(G);
        Pair squares(0.f), inner(0.f);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          Piece<G, LIE> s, dy;
          s.fetch(from + c[k], have[k]);
          dy.fetch(from + next + c[k], have[k]);
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            const Pair a = s.pair(i);
            squares = fma(a, a, squares);
            inner = fma(dy.pair(i) * w[k].pair(i), a, inner);
          }
        }
        const Pair both = row_sum(Pair(squares.sum(), inner.sum()), warps, group, parity, room);
        const float inv = Root(mean(both.lo(), p.columns, p.one_nth) + p.eps).value();
        const Pair root(inv), m(-(mean(both.hi(), p.columns, p.one_nth) * inv * inv * inv));
        asm volatile("" ::: "memory");      // both are read again: registers for them would cost 24 warps to an SM (63 us instead of 50)
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          Piece<G, LIE> s, dy, more, out;
          s.fetch(from + c[k], have[k]);
          dy.fetch(from + next + c[k], have[k]);
          if (p.dsum.p) more.fetch(from + 2 * next + c[k], have[k]);
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            const Pair a = s.pair(i), b = dy.pair(i) * root;
            total[k][i] = fma(a, b, total[k][i]);
            out.set(i, fma(b, w[k].pair(i), p.dsum.p ? fma(a, m, more.pair(i)) : a * m));
          }
          out.store(p.ds + row * p.ldds + c[k], have[k]);
        }
      }
      leave_slot(ring, bars, slot);
      if (++slot == ring.slots) slot = 0, phase ^= 1;
    }
  }
  if (!ok) atomicAdd(&g_gave_up, 1u);
  // The ring is done with: its copies have landed and been used, or the copying warp waited for them.
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(slots);
  const bool mine = warp < ring.groups * warps;
  if (ring.groups > 1) join_groups<PARTS>(sums, total, mine ? group : ring.groups, ring.groups, T, t);
  put_part<PARTS>(parts, sums, total, ring.groups, T, t, mine);
}

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

// The weight's gradient of a strip of 32 columns: eight warps take the tokens in turn.
template <typename G, typename W> __global__ void __launch_bounds__(256) norm_weight_kernel(const __grid_constant__ Backward<G, W> p, void* dw, GradType dw_type) {
  __shared__ float room[8][32];
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
  float total = 0.f;
  if (c < p.cols)
    for (uint64_t r = warp; r < p.rows; r += 8) total = fmaf((float)p.dy.p[r * p.dy.ld + c], (float)p.s.p[r * p.s.ld + c] * p.stats[r].x, total);
  room[warp][lane] = total;
  __syncthreads();
  if (warp == 0 && c < p.cols) {
    for (int i = 1; i < 8; ++i) total += room[i][lane];
    put_weight(dw, dw_type, c, total);
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

// dw: the blocks' parts added in order, by eight warps in turn.  A part has `length` values in the order of the T threads of a row.
template <typename D, Lie LIE> __global__ void __launch_bounds__(256) norm_join_kernel(const float* parts, uint32_t count, uint32_t length, uint32_t T, uint32_t cols, D* dw) {
  __shared__ float room[8][32];
  admit_next_kernel();
  await_previous_kernel();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, j = blockIdx.x * 32 + lane;
  float total = 0.f;
  if (j < length) {
#pragma unroll 4
    for (uint32_t i = warp; i < count; i += 8) total += parts[(uint64_t)i * length + j];
  }
  room[warp][lane] = total;
  __syncthreads();
  const uint32_t c = column_of<LIE>(j % T, T, j / T);
  if (warp == 0 && j < length && c < cols) {
    for (int k = 1; k < 8; ++k) total += room[k][lane];
    if constexpr (sizeof(D) == 4) dw[c] = total;
    else dw[c] = __float2bfloat16_rn(total);
  }
}

template <typename G, typename W, Lie LIE, int PARTS> cudaError_t run_staged(const Forward<G, W>& p, uint64_t rows, const Staged& a, cudaStream_t stream) {
  static Device device;
  const Device::Facts* facts;
  const cudaError_t e = device.prepare(norm_staged_kernel<G, W, LIE, PARTS>, a.threads(), kRing, 0, &facts);
  if (e != cudaSuccess) return e;
  return launch_overlapped(norm_staged_kernel<G, W, LIE, PARTS>, a.blocks, a.threads(), a.ring.slots * a.ring.slot(), 1, stream, p, (uint32_t)rows, a.warps, a.ring);
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
  p.one_nth = 1.f / p.columns;
  Access all = both(p.x.access, p.w.access);
  if (p.residual.p) all = both(all, p.residual.access);
  if (p.sum) all = both(all, access_of<G>(p.sum, p.ldsum));
  if (p.y) all = both(all, access_of<G>(p.y, p.ldy));
  const uint64_t padded = std::max(std::max<uint64_t>(cols, (uint64_t)p.nb * kFp8Block), (uint64_t)p.kept_blocks * 32);
  const bool any = all == kByElement;
  if (padded > kMostHeld)
    return launch_overlapped(any ? norm_long_kernel<G, W, true> : norm_long_kernel<G, W, false>, (uint32_t)rows, kMostThreads, 0, 1, stream, p);
  Lie lie = lie_of(n.x.p, n.x.ld, sizeof(G));
  lie = std::max(lie, lie_of(n.weight, 0, 1));
  if (p.residual.p) lie = std::max(lie, lie_of(n.residual.p, n.residual.ld, sizeof(G)));
  if (p.sum) lie = std::max(lie, lie_of(p.sum, p.ldsum, sizeof(G)));
  if (p.y) lie = std::max(lie, lie_of(p.y, p.ldy, sizeof(G)));
  if constexpr (sizeof(G) == 2) if (lie != kSpread) {
    const Staged st(rows, cols, sizeof(G), p.residual.p ? 2 : 1, padded, false);
    if (st.parts == 1) return lie == kBy32s ? run_staged<G, W, kBy32s, 1>(p, rows, st, stream) : run_staged<G, W, kBy16s, 1>(p, rows, st, stream);
    if (st.parts == 2) return lie == kBy32s ? run_staged<G, W, kBy32s, 2>(p, rows, st, stream) : run_staged<G, W, kBy16s, 2>(p, rows, st, stream);
  }
  const Split a = forward_split(rows, padded, lie == kSpread);
  const uint32_t parts = a.parts;
  const auto kernel = parts == 1 ? lie == kBy32s ? norm_kernel<G, W, kBy32s, 1> : lie == kBy16s ? norm_kernel<G, W, kBy16s, 1> : norm_kernel<G, W, kSpread, 1>
                                 : lie == kBy32s ? norm_kernel<G, W, kBy32s, 2> : norm_kernel<G, W, kBy16s, 2>;
  return launch_overlapped(kernel, a.blocks, a.threads, 0, 1, stream, p, (uint32_t)rows, a.warps);
}

template <typename G, typename W, Lie LIE, int PARTS>
cudaError_t run_staged_backward(const Backward<G, W>& p, const Staged& a, float* parts, cudaStream_t stream) {
  static Device device;
  const Device::Facts* facts;
  const cudaError_t e = device.prepare(norm_backward_staged_kernel<G, W, LIE, PARTS>, a.threads(), kRing, 0, &facts);
  if (e != cudaSuccess) return e;
  const uint32_t smem = std::max(a.ring.slots * a.ring.slot(), a.ring.groups > 1 ? a.ring.groups * a.length() * (uint32_t)sizeof(float) : 0u);
  return launch_overlapped(norm_backward_staged_kernel<G, W, LIE, PARTS>, a.blocks, a.threads(), smem, 1, stream, p, a.warps, parts, a.ring);
}

template <typename G, typename W, Lie LIE, int PARTS, bool CLUSTER, uint32_t THREADS = kMostThreads>
cudaError_t run_backward(const Backward<G, W>& p, const Split& a, float* parts, const NormBackward& n, cudaStream_t stream) {
  static Device device;
  const Device::Facts* facts;
  const cudaError_t e = device.prepare(norm_backward_kernel<G, W, LIE, PARTS, CLUSTER, THREADS>, a.threads, kMostSums * sizeof(float), 0, &facts);
  if (e != cudaSuccess) return e;
  const uint32_t groups = a.threads / 32 / a.warps, smem = CLUSTER || groups > 1 ? groups * a.length() * (uint32_t)sizeof(float) : 0;
  return launch_overlapped(norm_backward_kernel<G, W, LIE, PARTS, CLUSTER, THREADS>, a.blocks, a.threads, smem, CLUSTER ? a.blocks : 1, stream, p, a.warps, parts, n.dw, n.dw_type);
}
template <typename G, typename W, Lie LIE> cudaError_t pick_backward(const Backward<G, W>& p, const Split& a, float* parts, const NormBackward& n, cudaStream_t stream) {
  if (a.blocks <= kMostCluster) return a.parts == 2 ? run_backward<G, W, LIE, 2, true>(p, a, parts, n, stream) : run_backward<G, W, LIE, 1, true>(p, a, parts, n, stream);
  if constexpr (sizeof(G) == 2 && LIE == kSpread)
    if (a.threads > kMostThreads) return run_backward<G, W, LIE, 1, false, kWideThreads>(p, a, parts, n, stream);
  return a.parts == 2 ? run_backward<G, W, LIE, 2, false>(p, a, parts, n, stream) : run_backward<G, W, LIE, 1, false>(p, a, parts, n, stream);
}

template <Lie LIE> cudaError_t join(const NormBackward& n, const float* parts, uint32_t count, uint32_t length, uint32_t T, cudaStream_t stream) {
  const uint32_t strips = (length + 31) / 32, cols = (uint32_t)n.s.cols;
  if (n.dw_type == kBF16) return launch_overlapped(norm_join_kernel<__nv_bfloat16, LIE>, strips, 256, 0, 1, stream, parts, count, length, T, cols, static_cast<__nv_bfloat16*>(n.dw));
  return launch_overlapped(norm_join_kernel<float, LIE>, strips, 256, 0, 1, stream, parts, count, length, T, cols, static_cast<float*>(n.dw));
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
  p.one_nth = 1.f / p.columns;
  p.stats = static_cast<float2*>(workspace);
  Access all = both(both(p.dy.access, p.s.access), both(p.w.access, access_of<G>(p.ds, p.ldds)));
  if (p.dsum.p) all = both(all, p.dsum.access);
  const bool any = all == kByElement;
  if (cols <= kMostHeld) {
    float* parts = static_cast<float*>(workspace);
    Lie lie = std::max(std::max(lie_of(n.dy.p, n.dy.ld, sizeof(G)), lie_of(n.s.p, n.s.ld, sizeof(G))), std::max(lie_of(n.ds.p, n.ds.ld, sizeof(G)), lie_of(n.weight, 0, 1)));
    if (n.dsum.p) lie = std::max(lie, lie_of(n.dsum.p, n.dsum.ld, sizeof(G)));
    const Split a = backward_split(rows, cols, sizeof(G) == 2 && lie == kSpread);
    if constexpr (sizeof(G) == 2) if (lie != kSpread) {
      const Staged st(rows, cols, sizeof(G), p.dsum.p ? 3 : 2, cols, true);
      if (st.parts) {
        const cudaError_t e = st.parts == 1 ? lie == kBy32s ? run_staged_backward<G, W, kBy32s, 1>(p, st, parts, stream) : run_staged_backward<G, W, kBy16s, 1>(p, st, parts, stream)
                              : lie == kBy32s ? run_staged_backward<G, W, kBy32s, 2>(p, st, parts, stream) : run_staged_backward<G, W, kBy16s, 2>(p, st, parts, stream);
        return e != cudaSuccess ? e : join<kBy32s>(n, parts, st.blocks, st.length(), st.warps * 32, stream);
      }
    }
    const cudaError_t e = lie == kBy32s ? pick_backward<G, W, kBy32s>(p, a, parts, n, stream)
                          : lie == kBy16s ? pick_backward<G, W, kBy16s>(p, a, parts, n, stream) : pick_backward<G, W, kSpread>(p, a, parts, n, stream);
    if (e != cudaSuccess || a.blocks <= kMostCluster) return e;
    return lie == kSpread ? join<kSpread>(n, parts, a.blocks, a.length(), a.warps * 32, stream) : join<kBy32s>(n, parts, a.blocks, a.length(), a.warps * 32, stream);
  }
  cudaError_t e = launch_overlapped(any ? norm_stats_kernel<G, W, true> : norm_stats_kernel<G, W, false>, (uint32_t)rows, kMostThreads, 0, 1, stream, p);
  if (e == cudaSuccess) e = launch_overlapped(norm_weight_kernel<G, W>, (uint32_t)((cols + 31) / 32), 256, 0, 1, stream, p, n.dw, n.dw_type);
  // only now: it may be written over dy
  if (e == cudaSuccess) e = launch_overlapped(any ? norm_input_kernel<G, W, true> : norm_input_kernel<G, W, false>, (uint32_t)rows, kMostThreads, 0, 1, stream, p);
  return e;
}

}  // namespace

cudaError_t rms_norm_gave_up(uint32_t* count, cudaStream_t stream) { return read_count(g_gave_up, count, stream); }
cudaError_t rms_norm_count(const uint32_t** at) { return count_address(g_gave_up, at); }

cudaError_t launch_rms_norm(const NormForward& n, cudaStream_t stream) {
  if (n.x.type == kBF16) return n.weight_type == kBF16 ? forward<__nv_bfloat16, __nv_bfloat16>(n, stream) : forward<__nv_bfloat16, float>(n, stream);
  return n.weight_type == kBF16 ? forward<float, __nv_bfloat16>(n, stream) : forward<float, float>(n, stream);
}

uint64_t rms_norm_backward_workspace(uint64_t rows, uint64_t cols) {
  if (cols <= kMostHeld) {
    // enough however they lie: a part to an SM, of whole warps
    return backward_split(rows, cols, false).blocks <= kMostCluster ? 0 : kSms * ((cols + 1023) / 1024 * 1024) * sizeof(float);
  }
  return rows * sizeof(float2);      // statistics
}

cudaError_t launch_rms_norm_backward(const NormBackward& n, void* workspace, cudaStream_t stream) {
  if (n.s.type == kBF16) return n.weight_type == kBF16 ? backward<__nv_bfloat16, __nv_bfloat16>(n, workspace, stream) : backward<__nv_bfloat16, float>(n, workspace, stream);
  return n.weight_type == kBF16 ? backward<float, __nv_bfloat16>(n, workspace, stream) : backward<float, float>(n, workspace, stream);
}

}  // namespace rudra
