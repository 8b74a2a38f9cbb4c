// Blocks of 32 values with a shared power-of-two scale, as MX4 and ACT8 hold them: a thread works on
// 16 consecutive values of a row, two neighbouring lanes on one block.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "vec.cuh"

namespace rudra {
namespace {

constexpr int kValues = 16;   // of a row per thread

// How the rows of a matrix lie: every thread's values on a boundary of 32 bytes, of 16 (bf16 alone), or of an
// element.  A warp's 32-byte accesses are whole sectors; with 16 bytes every sector is asked for twice
// (4096 x 9216 bf16 values written: 21.7 us against 14.3).
enum Access : int { kByElement = 0, kBy16 = 1, kBy32 = 2 };

template <typename G> inline Access access_of(const void* p, uint64_t ld) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  if (a % 32 == 0 && ld * sizeof(G) % 32 == 0) return kBy32;
  return sizeof(G) == 2 && a % 16 == 0 && ld % 8 == 0 ? kBy16 : kByElement;
}
inline Access both(Access a, Access b) { return a < b ? a : b; }

// A matrix that is read: its rows, and where its memory ends.
template <typename G> struct Rows {
  const G* p;
  uint64_t ld;
  const G* end;
  Access access;
  // Rows from `row` on.
  static Rows of(const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t row) {
    if (!base) return Rows{nullptr, 0, nullptr, kByElement};
    const G* p = static_cast<const G*>(base);
    return Rows{p + row * ld, ld, p + (rows - 1) * ld + cols, access_of<G>(base, ld)};
  }
};

// A thread's values of a row.
template <typename G> struct Values {
  static constexpr int kWords = kValues * sizeof(G) / 4;
  uint32_t w[kWords];

  // FIRST: first to leave L2, for a matrix that is done with once it is read (quantization of 4096 x 9216 floats
  // 32.4 us without, 28.0 with it).
  template <bool FIRST> static __device__ __forceinline__ void load32(const uint32_t* q, uint32_t* r) {
    if (FIRST)
      asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(q) : "memory");
    else
      asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(q) : "memory");
  }

  // `have` values from element `at` of the matrix; the others are zero.  ANY: its rows may lie anyhow.
  template <bool ANY, bool FIRST = false> __device__ __forceinline__ void load(const Rows<G>& m, uint64_t at, int have) {
    const G* p = m.p + at;
    if (have == kValues && m.access == kBy32) {
#pragma unroll
      for (int i = 0; i < kWords; i += 8) load32<FIRST>(reinterpret_cast<const uint32_t*>(p) + i, w + i);
      return;
    }
    if (sizeof(G) == 2 && have == kValues && m.access == kBy16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "l"(reinterpret_cast<const uint32_t*>(p) + i) : "memory");
      return;
    }
    // Rows that lie anyhow: the 32-byte pieces around the values, as long as they are in the matrix's memory, moved
    // down by the values' distance from a boundary.  (Quantization of 4096 x 9216 floats in rows of 9219: 76.8 us by
    // element, 40.1 this way.)
    const uintptr_t from = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)31;
    const uintptr_t to = (reinterpret_cast<uintptr_t>(p) + kValues * sizeof(G) + 31) & ~(uintptr_t)31;
    if (ANY && have > 0 && from >= reinterpret_cast<uintptr_t>(m.p) && to <= reinterpret_cast<uintptr_t>(m.end)) {
      uint32_t r[kWords + 8];
      const uint32_t* q = reinterpret_cast<const uint32_t*>(from);
#pragma unroll
      for (int i = 0; i < kWords; i += 8) load32<false>(q + i, r + i);
      if (to - from > kWords * 4) {
        load32<false>(q + kWords, r + kWords);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[kWords + i] = 0;
      }
      const uint32_t words = (uint32_t)(reinterpret_cast<uintptr_t>(p) / 4) % 8;
#pragma unroll
      for (int i = 0; i < kWords + 4; ++i) r[i] = words & 4 ? r[i + 4] : r[i];
#pragma unroll
      for (int i = 0; i < kWords + 2; ++i) r[i] = words & 2 ? r[i + 2] : r[i];
#pragma unroll
      for (int i = 0; i < kWords + 1; ++i) r[i] = words & 1 ? r[i + 1] : r[i];
      const uint32_t half = sizeof(G) == 2 ? (uint32_t)(reinterpret_cast<uintptr_t>(p) / 2) % 2 * 16 : 0;
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = sizeof(G) == 2 ? __funnelshift_r(r[i], r[i + 1], half) : r[i];
      if (have < kValues) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
          if (sizeof(G) == 4) w[i] = i < have ? w[i] : 0u;
          else w[i] = 2 * i + 1 < have ? w[i] : 2 * i < have ? w[i] & 0xFFFFu : 0u;
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if (sizeof(G) == 4) w[i] = i < have ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
      else w[i] = (2 * i < have ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i] : 0u) |
                  (2 * i + 1 < have ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if (sizeof(G) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);   // bf16 is the upper half of a float
  }
  // Largest magnitude as the bits of a float: they order like the magnitudes, an infinity above every
  // number and NaN above both.
  __device__ __forceinline__ uint32_t max_bits() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if (sizeof(G) == 4) m = max(m, w[i] & 0x7FFFFFFFu);
      else m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
    }
    return sizeof(G) == 4 ? m : max(m << 16, m & 0xFFFF0000u);
  }
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Where the values of a warp meet when their rows lie anyhow.
struct alignas(16) Meeting {
  uint32_t words[32 * (kValues + 1)];
  uint64_t to[32];
  int have[32];
};

// Writes `have` of a thread's values at p, rows on boundaries of 16 or 32 bytes.
template <typename G> __device__ __forceinline__ void store_values(G* p, Access access, int have, const float (&x)[kValues]) {
  constexpr int kWords = kValues * sizeof(G) / 4;
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) w[i] = sizeof(G) == 4 ? __float_as_uint(x[i]) : pack_bf16(x[2 * i % kValues], x[(2 * i + 1) % kValues]);
  if (have == kValues && access == kBy32) {
#pragma unroll
    for (int i = 0; i < kWords; i += 8)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                   :: "l"(reinterpret_cast<uint32_t*>(p) + i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]),
                      "r"(w[i + 6]), "r"(w[i + 7]) : "memory");
  } else if (sizeof(G) == 2 && have == kValues && access == kBy16) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < kValues; ++i)
      if (i < have) {
        if constexpr (sizeof(G) == 4) p[i] = x[i];
        else p[i] = __float2bfloat16_rn(x[i]);
      }
  }
}

// The same to rows that lie anyhow; a whole warp calls it.  Expansion of 4096 x 9215 codes to bf16: 225 us with every lane writing
// its own elements, 36 with neighbouring lanes on neighbouring elements, 27 with runs of bf16 moved to 16-byte boundaries (f32
// gains nothing by that).
template <typename G> __device__ __forceinline__ void store_values_anyhow(Meeting& m, G* p, int have, const float (&x)[kValues]) {
  const int lane = threadIdx.x % 32;
  constexpr int kPitch = sizeof(G) == 4 ? kValues + 1 : kValues;   // of a lane's values
  const uint64_t to = reinterpret_cast<uint64_t>(p), next = __shfl_down_sync(0xFFFFFFFFu, to, 1);
  __syncwarp();
  if constexpr (sizeof(G) == 4) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) m.words[lane * kPitch + i] = __float_as_uint(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kValues; i += 8)
      *reinterpret_cast<uint4*>(m.words + (lane * kValues + i) / 2) =
          make_uint4(pack_bf16(x[i], x[i + 1]), pack_bf16(x[i + 2], x[i + 3]), pack_bf16(x[i + 4], x[i + 5]), pack_bf16(x[i + 6], x[i + 7]));
  }
  m.to[lane] = to;
  m.have[lane] = have;
  __syncwarp();
  const G* const values = reinterpret_cast<const G*>(m.words);
  if (sizeof(G) == 2 && __all_sync(0xFFFFFFFFu, lane == 31 || (have == kValues && next == to + kValues * sizeof(G)))) {
    // one run of elements: 16 bytes at a time on their boundaries, the words moved by the run's distance from one
    G* const base = reinterpret_cast<G*>(m.to[0]);
    const int total = 31 * kValues + m.have[31], head = min(total, (int)((16 - m.to[0] % 16) % 16 / 2));
    const int pieces = (total - head) / 8, tail = head + 8 * pieces;
    for (int j = lane; j < pieces; j += 32) {
      uint32_t r[8];
      *reinterpret_cast<uint4*>(r) = *reinterpret_cast<const uint4*>(m.words + 4 * j);
      *reinterpret_cast<uint4*>(r + 4) = *reinterpret_cast<const uint4*>(m.words + 4 * j + 4);
#pragma unroll
      for (int i = 0; i < 6; ++i) r[i] = head & 4 ? r[i + 2] : r[i];
#pragma unroll
      for (int i = 0; i < 5; ++i) r[i] = head & 2 ? r[i + 1] : r[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = __funnelshift_r(r[i], r[i + 1], head % 2 * 16);
      *reinterpret_cast<uint4*>(base + head + 8 * j) = make_uint4(r[0], r[1], r[2], r[3]);
    }
    const int e = lane < head ? lane : tail + lane - head;
    if (lane < head || e < total) base[e] = values[e];
    return;
  }
#pragma unroll 4
  for (int i = 0; i < kValues; ++i) {
    const int of = i * (32 / kValues) + lane / kValues, e = lane % kValues;
    if (e < m.have[of]) reinterpret_cast<G*>(m.to[of])[e] = values[of * kPitch + e];
  }
}

__device__ __forceinline__ uint32_t block_max_bits(uint32_t m) {   // over the two lanes of a block
  return max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
}

// Division of numbers below 2^31 by a fixed one below 2^31: the quotient is the high half of a product.
struct Divisor {
  uint32_t d, mul, shift;
  Divisor() = default;
  explicit Divisor(uint32_t by) : d(by), shift(0) {
    while ((1ull << shift) < by) ++shift;   // 2^(shift - 1) < by <= 2^shift: the rounded-up multiplier errs below one part in 2^31
    mul = (uint32_t)(((1ull << (31 + shift)) + by - 1) / by);
  }
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> (31 + shift)); }
};

// Scale byte s of a block for a format whose values reach 2^below * 2^(s - 127): 255 marks a block that
// holds an infinity or NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits, uint32_t below) {
  const uint32_t e = bits >> 23;
  return e == 255u ? 255u : e > below ? e - below : 0u;
}
// 2^(127 - s) for s <= 253, which is always a normal number; 0 for s = 255, whose codes are zero.
__device__ __forceinline__ float inverse_scale(uint32_t s) { return s == 255u ? 0.f : __uint_as_float((254u - s) << 23); }
// 2^(s - 127), NaN for s = 255.
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __uint_as_float(s == 255u ? 0x7FC00000u : s ? s << 23 : 0x00400000u);
}

// E2M1 codes of the thread's values, the first in the low bits: nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t e2m1_codes8(const float (&x)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(r) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return r;
}
template <typename V> __device__ __forceinline__ uint2 e2m1_codes(const V& v, uint32_t s) {
  const float inv = inverse_scale(s);
  float x[8];
  uint2 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = v.get(i) * inv;
  r.x = e2m1_codes8(x);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = v.get(8 + i) * inv;
  r.y = e2m1_codes8(x);
  return s == 255u ? make_uint2(0u, 0u) : r;
}

// The values E2M1 codes stand for under a scale.
__device__ __forceinline__ void e2m1_values(uint2 codes, float scale, float (&x)[kValues]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q ? codes.y : codes.x));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      x[8 * q + 2 * i] = f.x * scale;
      x[8 * q + 2 * i + 1] = f.y * scale;
    }
  }
}

// int8 codes of the thread's values: nearest, ties to even, at most 127 in magnitude.  Adding 1.5 * 2^23
// rounds to a whole number whose two's complement is the sum's low byte; values past 127 are cut off before,
// two bf16 at a time, or after.
template <typename G> __device__ __forceinline__ uint4 int8_codes(const Values<G>& v, uint32_t s) {
  constexpr float kWhole = 12582912.f;
  const float inv = inverse_scale(s);
  const uint32_t top = __float_as_uint(127.f * scale_value(s)) >> 16;   // exact in bf16
  const uint32_t high = top * 0x10001u, low = high | 0x80008000u;
  uint32_t r[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (sizeof(G) == 4) {
        b[i] = __float_as_uint(fminf(fmaxf(fmaf(v.get(4 * q + i), inv, kWhole), kWhole - 127.f), kWhole + 127.f));
      } else {
        const __nv_bfloat162 w = __hmax2(__hmin2(reinterpret_cast<const __nv_bfloat162&>(v.w[(4 * q + i) / 2]), reinterpret_cast<const __nv_bfloat162&>(high)),
                                         reinterpret_cast<const __nv_bfloat162&>(low));
        const uint32_t u = reinterpret_cast<const uint32_t&>(w);
        b[i] = __float_as_uint(fmaf(__uint_as_float(i % 2 ? u & 0xFFFF0000u : u << 16), inv, kWhole));
      }
    }
    r[q] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  }
  return s == 255u ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(r[0], r[1], r[2], r[3]);
}
// The values int8 codes stand for: a code plus 128, set into 2^23, is a float less 2^23 + 128.
__device__ __forceinline__ void int8_values(uint4 codes, float scale, float (&x)[kValues]) {
  const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t u = c[q] ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * q + i] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + i)) - 8388736.f) * scale;
  }
}

// Where the scale byte of (row r, block b) sits in an MX4 matrix with kt = ceil(blocks / 4).
__host__ __device__ __forceinline__ uint64_t mx4_scale_at(uint64_t r, uint64_t b, uint64_t kt) {
  return ((r / 128) * kt + b / 4) * 512 + (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4;
}

}  // namespace
}  // namespace rudra
