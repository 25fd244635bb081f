// mx4.cuh -- rows in microscaled 4-bit floating point (OCP MX, MXFP4): blocks of
// 32 values of e2m1 codes share a scale 2^(byte - 127).  A row of dim values is
// its blocks' codes (16 bytes each, the even value in a byte's low half), the
// blocks' scale bytes, and zeros up to a multiple of 16 bytes.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace agnes {

constexpr int kMxBlock = 32;

inline int64_t mx4_blocks(int64_t dim) { return (dim + kMxBlock - 1) / kMxBlock; }
inline int64_t mx4_row_bytes(int64_t dim) { return (mx4_blocks(dim) * 17 + 15) / 16 * 16; }

// 2^(byte - 127); 255 is NaN.  Byte 0 has no normal form.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}

// Eight codes from floats, each to nearest even, beyond 6 to 6; the first in the lowest
// bits.
__device__ __forceinline__ uint32_t mx4_codes8(const float (&f)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 q0, q1, q2, q3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 q0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 q1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 q2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 q3, %8, %7;\n\t"
      "mov.b32 %0, {q0, q1, q2, q3};\n\t}"
      : "=r"(r)
      : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  return r;
}

// The eight values of a word of codes, in order.
__device__ __forceinline__ void mx4_values(uint32_t codes, __half2 (&v)[4]) {
  uint32_t r[4];
  asm("{\n\t.reg .b8 q0, q1, q2, q3;\n\t"
      "mov.b32 {q0, q1, q2, q3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, q0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, q1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, q2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, q3;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = *(const __half2*)&r[i];
}

}  // namespace agnes
