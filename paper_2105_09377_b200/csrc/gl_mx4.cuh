// The 4-bit number format, shared by the kernel files: 32 E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) and an
// E8M0 scale 2^(e - 127) per block; e = 255 stands for NaN.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace {

// Scale exponent of a block whose largest magnitude has the bits `top`: floor(log2 top) - 2, so that the largest
// value falls in [4, 8) (above 6 it saturates).  A block that holds an Inf or a NaN becomes NaN as a whole.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t top) {
  const uint32_t b = top >> 23;   // subnormals have b = 0: below the smallest scale either way
  return b == 255u ? 255u : (b > 2u ? b - 2u : 0u);
}

// Eight values -> eight codes, value i in bits 4i..4i+3, rounded to nearest (ties to the even mantissa) after the
// exact multiplication with 2^(127 - e).
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], uint32_t e) {
  const float f = e == 255u ? 0.f : __uint_as_float((254u - e) << 23);
  uint32_t d;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(d)
      : "f"(v[0] * f), "f"(v[1] * f), "f"(v[2] * f), "f"(v[3] * f), "f"(v[4] * f), "f"(v[5] * f), "f"(v[6] * f), "f"(v[7] * f));
  return e == 255u ? 0u : d;
}

// 2^(e - 127) as fp32 (e = 0 is subnormal), NaN for e = 255.
__device__ __forceinline__ float mx4_scale(uint32_t e) {
  return e == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(max(e << 23, 0x00400000u));
}

// bf16x2 multiplication that keeps subnormals
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(0x80008000u));
  return d;
}
// Four pairs of codes -> four bf16 pairs times 2^-126.  `z` holds four codes in each 16-bit half; pair i is code i of the
// low half and code i of the high half.  The three magnitude bits of E2M1 are the low exponent bits and the top mantissa
// bit of a bf16 with bias 127 instead of 1, subnormals included, so moving the bits is the conversion.
__device__ __forceinline__ void mx4_pairs_moved(uint32_t z, uint32_t (&h)[4]) {
  h[0] = ((z << 12) & 0x80008000u) | ((z << 6) & 0x01C001C0u);
  h[1] = ((z << 8) & 0x80008000u) | ((z << 2) & 0x01C001C0u);
  h[2] = ((z << 4) & 0x80008000u) | ((z >> 2) & 0x01C001C0u);
  h[3] = (z & 0x80008000u) | ((z >> 6) & 0x01C001C0u);
}

// Eight codes of one block with scale exponent e -> eight bf16 values in their order (exact: two significant bits).
__device__ __forceinline__ void mx4_words_bf16(uint32_t z, uint32_t e, uint32_t (&w)[4]) {
  uint32_t h[4];
  mx4_pairs_moved(z, h);
  // 2^(e - 1) is a bf16 up to e = 128; larger scales in two steps
  const uint32_t f = (min(e, 128u) + 126u) * 0x00800080u;
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = mul_bf16x2(h[i], f);
  if (e > 128u) {
    const uint32_t f2 = (e == 255u ? 0x7FC0u : (e - 1u) << 7) * 0x00010001u;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = mul_bf16x2(h[i], f2);
  }
  w[0] = __byte_perm(h[0], h[1], 0x5410);
  w[1] = __byte_perm(h[2], h[3], 0x5410);
  w[2] = __byte_perm(h[0], h[1], 0x7632);
  w[3] = __byte_perm(h[2], h[3], 0x7632);
}

}  // namespace
