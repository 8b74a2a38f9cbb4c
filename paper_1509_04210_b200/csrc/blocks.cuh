// Blocks of 32 values with a shared power-of-two scale, as MX4 and ACT8 hold them: a thread works on
// 8 consecutive values of a row, four neighbouring lanes on one block.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "vec.cuh"

namespace rudra {
namespace {

// 8 values from p; `wide`: p sits on a boundary of the whole access and all 8 exist, else `have` do.
template <typename G> __device__ __forceinline__ void load8(const G* p, bool wide, int have, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float* p, bool wide, int have, float (&x)[8]) {
  if (wide) {
    asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(p));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < have ? p[i] : 0.f;
  }
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, bool wide, int have, float (&x)[8]) {
  if (wide) {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < have ? __bfloat162float(p[i]) : 0.f;
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <typename G> __device__ __forceinline__ void store8(G* p, bool wide, int have, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, bool wide, int have, const float (&x)[8]) {
  if (wide) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) p[i] = x[i];
  }
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, bool wide, int have, const float (&x)[8]) {
  if (wide) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) p[i] = __float2bfloat16_rn(x[i]);
  }
}

// Whether every 8-value unit of a matrix's rows sits on a boundary of its access (16 bytes bf16, 32 f32).
template <typename G> inline bool wide_rows(const void* p, uint64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % (8 * sizeof(G)) == 0 && ld % 8 == 0;
}

// Largest magnitude as the bits of a float: they order like the magnitudes, an infinity above every
// number and NaN above both.
__device__ __forceinline__ uint32_t max_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  return m;
}
__device__ __forceinline__ uint32_t block_max_bits(uint32_t m) {   // over the four lanes of a block
  m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  return max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
}

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

// 8 values to E2M1 codes, the first in the low bits: nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t e2m1_codes(const float (&x)[8], float inv) {
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(r)
      : "f"(x[0] * inv), "f"(x[1] * inv), "f"(x[2] * inv), "f"(x[3] * inv), "f"(x[4] * inv), "f"(x[5] * inv),
        "f"(x[6] * inv), "f"(x[7] * inv));
  return inv == 0.f ? 0u : r;
}

// 8 E2M1 codes to the values they stand for under a scale.
__device__ __forceinline__ void e2m1_values(uint32_t codes, float scale, float (&x)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    x[2 * i] = f.x * scale;
    x[2 * i + 1] = f.y * scale;
  }
}

// 8 values to int8 codes in two words: nearest, ties to even, at most 127 in magnitude.
__device__ __forceinline__ uint2 int8_codes(const float (&x)[8], float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = max(-127, min(127, __float2int_rn(x[i] * inv)));
    w[i / 4] |= (uint32_t)(c & 255) << (8 * (i % 4));
  }
  return inv == 0.f ? make_uint2(0u, 0u) : make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void int8_values(uint2 w, float scale, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = (float)(int8_t)(w.x >> (8 * i)) * scale;
    x[4 + i] = (float)(int8_t)(w.y >> (8 * i)) * scale;
  }
}

// Where the scale byte of (row r, block b) sits in an MX4 matrix with kt = ceil(blocks / 4).
__host__ __device__ __forceinline__ uint64_t mx4_scale_at(uint64_t r, uint64_t b, uint64_t kt) {
  return ((r / 128) * kt + b / 4) * 512 + (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4;
}

}  // namespace
}  // namespace rudra
