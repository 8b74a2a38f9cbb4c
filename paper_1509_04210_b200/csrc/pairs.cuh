// Pairs of floats, two to an instruction, and a thread's values of a row taken as pairs.
#pragma once
#include <cstdint>

#include "blocks.cuh"

namespace rudra {
namespace {

struct Pair {
  float2 v;
  Pair() = default;
  __device__ __forceinline__ Pair(float lo, float hi) : v(make_float2(lo, hi)) {}
  __device__ __forceinline__ explicit Pair(float both) : Pair(both, both) {}
  __device__ __forceinline__ explicit Pair(float2 both) : v(both) {}
  __device__ __forceinline__ float lo() const { return v.x; }
  __device__ __forceinline__ float hi() const { return v.y; }
  __device__ __forceinline__ float sum() const { return v.x + v.y; }
};
__device__ __forceinline__ Pair operator+(Pair a, Pair b) { return Pair(__fadd2_rn(a.v, b.v)); }
__device__ __forceinline__ Pair operator*(Pair a, Pair b) { return Pair(__fmul2_rn(a.v, b.v)); }
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) { return Pair(__ffma2_rn(a.v, b.v, c.v)); }

// The larger of two magnitudes; NaN if one is.
__device__ __forceinline__ float larger(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}

constexpr int kPairs = kValues / 2;

// How a thread's 16 values of a row lie: consecutive ones from a boundary of 32 or 16 bytes on; or every 32nd of the 512 that its
// warp has, which asks nothing of where a row begins: neighbouring lanes then read and write neighbouring values one by one.
// (Rows of 4111 bf16 values through shifted 32-byte pieces took five times as long as aligned ones.)
enum Lie : int { kBy32s, kBy16s, kSpread };

inline Lie lie_of(const void* p, uint64_t ld, uint64_t element) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p) | ld * element;
  return a % 32 == 0 ? kBy32s : a % 16 == 0 ? kBy16s : kSpread;
}

template <typename G, Lie LIE> struct Piece {
  static constexpr int kWords = Values<G>::kWords;
  Values<G> v;

  // `have` values from p on are in the row, the others zero.
  __device__ __forceinline__ void load(const G* p, int have) {
    if (LIE != kSpread && have == kValues) {
      if (LIE == kBy32s) {
#pragma unroll
        for (int i = 0; i < kWords; i += 8) Values<G>::template load32<false>(reinterpret_cast<const uint32_t*>(p) + i, v.w + i);
      } else {
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
          asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(v.w[i]), "=r"(v.w[i + 1]), "=r"(v.w[i + 2]), "=r"(v.w[i + 3]) : "l"(reinterpret_cast<const uint32_t*>(p) + i) : "memory");
      }
      return;
    }
    if (LIE == kSpread && have == kValues) gather<true>(p, have);
    else gather<false>(p, have);
  }
  // One by one; ALL: without asking for each whether it is there.
  template <bool ALL> __device__ __forceinline__ void gather(const G* p, int have) {
    constexpr int kStep = LIE == kSpread ? 32 : 1;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(G) == 4) {
        v.w[i] = ALL || i < have ? reinterpret_cast<const uint32_t*>(p)[kStep * i] : 0u;
      } else {
        const uint32_t lo = ALL || 2 * i < have ? reinterpret_cast<const uint16_t*>(p)[2 * kStep * i] : 0u;
        const uint32_t hi = ALL || 2 * i + 1 < have ? reinterpret_cast<const uint16_t*>(p)[2 * kStep * i + kStep] : 0u;
        v.w[i] = __byte_perm(lo, hi, 0x5410);
      }
    }
  }
  // The same out of shared memory, where a row begins on a boundary.
  __device__ __forceinline__ void fetch(const G* p, int have) {
    if (have == kValues) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 r = reinterpret_cast<const uint4*>(p)[i / 4];
        v.w[i] = r.x, v.w[i + 1] = r.y, v.w[i + 2] = r.z, v.w[i + 3] = r.w;
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(G) == 4) v.w[i] = i < have ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
      else v.w[i] = (2 * i < have ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i] : 0u) | (2 * i + 1 < have ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ Pair pair(int i) const { return Pair(v.get(2 * i), v.get(2 * i + 1)); }
  __device__ __forceinline__ void set(int i, Pair x) {
    if constexpr (sizeof(G) == 4) {
      v.w[2 * i] = __float_as_uint(x.lo());
      v.w[2 * i + 1] = __float_as_uint(x.hi());
    } else {
      v.w[i] = pack_bf16(x.lo(), x.hi());
    }
  }
  // a + b, rounded once.  (Two bf16 that a float does not hold the sum of lie so far apart that the sum rounds to the larger, so
  // this is also what rounding a float's sum gives.)
  __device__ __forceinline__ void add(const Piece& a, const Piece& b) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(G) == 4) v.w[i] = __float_as_uint(a.v.get(i) + b.v.get(i));
      else asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(v.w[i]) : "r"(a.v.w[i]), "r"(b.v.w[i]));
    }
  }
  __device__ __forceinline__ void store(G* p, int have) const {
    if (LIE != kSpread && have == kValues) {
      if (LIE == kBy32s) {
#pragma unroll
        for (int i = 0; i < kWords; i += 8)
          asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                       :: "l"(reinterpret_cast<uint32_t*>(p) + i), "r"(v.w[i]), "r"(v.w[i + 1]), "r"(v.w[i + 2]), "r"(v.w[i + 3]), "r"(v.w[i + 4]), "r"(v.w[i + 5]),
                          "r"(v.w[i + 6]), "r"(v.w[i + 7]) : "memory");
      } else {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(v.w[i], v.w[i + 1], v.w[i + 2], v.w[i + 3]);
      }
      return;
    }
    if (LIE == kSpread && have == kValues) scatter<true>(p, have);
    else scatter<false>(p, have);
  }
  template <bool ALL> __device__ __forceinline__ void scatter(G* p, int have) const {
    constexpr int kStep = LIE == kSpread ? 32 : 1;
#pragma unroll
    for (int i = 0; i < kValues; ++i)
      if (ALL || i < have) {
        if constexpr (sizeof(G) == 4) reinterpret_cast<uint32_t*>(p)[kStep * i] = v.w[i];
        else reinterpret_cast<uint16_t*>(p)[kStep * i] = (uint16_t)(v.w[i / 2] >> i % 2 * 16);
      }
  }
};

}  // namespace
}  // namespace rudra
