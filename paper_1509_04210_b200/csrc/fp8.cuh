// 8-bit floating point with a shared power-of-two scale for each block of 128 values: what the kernels that write and
// read the format have in common.  A thread works on 16 consecutive values of a row, eight neighbouring lanes on one
// block.
#pragma once
#include <cstdint>

#include "blocks.cuh"

namespace rudra {
namespace {

constexpr uint32_t kFp8Block = 128;

// Scale byte of a block whose largest magnitude has these bits: 2^(s - 127) is the smallest power of two (s >= 0) under
// which that is at most 448 = 1.75 * 2^8, so nothing saturates; a significand above 1.75 carries into the exponent.  255
// marks a block that holds an infinity or NaN.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t bits) {
  const uint32_t e = (bits + 0x1FFFFFu) >> 23;
  return bits >= 0x7F800000u ? 255u : e > 8u ? e - 8u : 0u;
}
__device__ __forceinline__ uint32_t fp8_block_max_bits(uint32_t m) {   // over the eight lanes of a block
  m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
  return max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
}

// E4M3 codes of four values, the first in the low bits: nearest, ties to even.
__device__ __forceinline__ uint32_t e4m3_codes4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
// Codes of a thread's values under scale byte s; `get(i)` gives value i.
template <typename V> __device__ __forceinline__ uint4 e4m3_codes(const V& get, uint32_t s) {
  const float inv = inverse_scale(s);
  uint32_t r[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) r[q] = e4m3_codes4(get(4 * q) * inv, get(4 * q + 1) * inv, get(4 * q + 2) * inv, get(4 * q + 3) * inv);
  return s == 255u ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(r[0], r[1], r[2], r[3]);
}

// The values E4M3 codes stand for under a scale.
__device__ __forceinline__ void e4m3_values(uint4 codes, float scale, float (&x)[kValues]) {
  const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t h[2];
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
        : "=r"(h[0]), "=r"(h[1]) : "r"(c[q]));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      x[4 * q + 2 * i] = f.x * scale;
      x[4 * q + 2 * i + 1] = f.y * scale;
    }
  }
}

// Writes the scale byte of (row, block b) of nb; with a row's last one the bytes up to a whole word, which are zero.
__device__ __forceinline__ void put_fp8_scale(uint8_t* scales, uint64_t row, uint32_t b, uint32_t nb, uint32_t kt, uint32_t s) {
  uint8_t* to = scales + mx4_scale_at(row, b, kt);
  *to = (uint8_t)s;
  if (b + 1 == nb)
    for (uint32_t i = b % 4 + 1; i < 4; ++i) *++to = 0;
}

}  // namespace
}  // namespace rudra
