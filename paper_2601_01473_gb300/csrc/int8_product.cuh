// int8_product.cuh -- what the products of 8-bit rows share: the checks of their arguments,
// and operands as sums of bfloat16 values.
#pragma once

#include "int8.cuh"
#include "tcgen05.cuh"

namespace agnes {

// The terms of a gradient lie below one another, and the TMA's coordinates are 32-bit.
constexpr int64_t kProductMaxRows = 1 << 29;

// A value of up to 16 significant bits as two bfloat16 ones, the first its leading eight
// bits; what is not finite is the first alone.
__device__ __forceinline__ void int8_split(float v, float& hi, float& lo) {
  hi = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  lo = fabsf(hi) <= 3.4e38f ? v - hi : 0.f;
}

// A row's scale, for the terms of its whole numbers.
struct Int8TermScale {
  float value;
  __nv_bfloat162 twice;
  bool brief;  // packed bfloat16 arithmetic makes the terms
  __device__ explicit Int8TermScale(float scale)
      : value(scale), twice(__float2bfloat162_rn(scale)) {
    // eight bits; and up to 2^121, 127 times it rounds to a finite bfloat16 value
    const uint32_t bits = __float_as_uint(scale);
    brief = (bits & 0xffffu) == 0 && (bits & 0x7fffffffu) <= 0x7c000000u;
  }
};

// Four whole numbers times a scale as pairs of bfloat16 terms that add up to it: exactly for a
// scale of eight bits, else to 2^-17 of it.
// Brief ones: hi the rounded products, lo what they leave.  A byte is its lower seven
// bits less 128 times its sign, and 128 + seven bits, 128 and 256 are bfloat16 bit patterns
// of the byte's parts.
// Others (a scale of more bits, that the quantiser did not write; a row with its type's largest
// number, whose products round past bfloat16's; one that stands for NaN), where the caller has not
// ruled them out (kBrief): in fp32, hi the leading eight bits and lo the next.
template <bool kBrief>
__device__ __forceinline__ void int8_terms4(uint32_t word, const Int8TermScale& scale, uint2& hi,
                                            uint2& lo) {
  uint32_t* h = &hi.x;
  uint32_t* l = &lo.x;
  if (!kBrief && !scale.brief) {
    float q[4], rest[4];
    int8_values4(word, q);
#pragma unroll
    for (int e = 0; e < 4; ++e) int8_split(q[e] * scale.value, q[e], rest[e]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __nv_bfloat162 top = __floats2bfloat162_rn(q[2 * i], q[2 * i + 1]);
      const __nv_bfloat162 left = __floats2bfloat162_rn(rest[2 * i], rest[2 * i + 1]);
      h[i] = *(const uint32_t*)&top;
      l[i] = *(const uint32_t*)&left;
    }
    return;
  }
  const uint32_t size = word & 0x7f7f7f7fu, sign = word & 0x80808080u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t pick = i ? 0x4342 : 0x4140;
    const uint32_t a = __byte_perm(size, 0x43434343u, pick);
    const uint32_t b = __byte_perm(sign, 0x43434343u, pick);
    const __nv_bfloat162 q = __hsub2(*(const __nv_bfloat162*)&a, *(const __nv_bfloat162*)&b);
    const __nv_bfloat162 top = __hmul2(q, scale.twice);
    const __nv_bfloat162 rest = __hfma2(q, scale.twice, __hneg2(top));
    h[i] = *(const uint32_t*)&top;
    l[i] = *(const uint32_t*)&rest;
  }
}

// How many such terms a gradient's type takes: all of its bits.
inline int grad_terms(int32_t dtype) {
  return dtype == AGNES_F32 ? 3 : dtype == AGNES_F16 ? 2 : 1;
}

// Whether the TMA can take a gradient as it is: bfloat16, 16-byte aligned rows.
inline bool takes_grad(const void* grad, int32_t dtype, int64_t stride) {
  return dtype == AGNES_BF16 && aligned_rows(grad, stride * 2, 16) && stride * 2 < (1ll << 40);
}

// rows x width values of dtype, stride apart, as grad_terms(dtype) bfloat16 matrices one
// after the other, their rows wpad apart (int8_linear.cu).
cudaError_t split_grad(const void* grad, int32_t dtype, int64_t stride, int64_t rows,
                       int64_t width, __nv_bfloat16* out, int64_t wpad, cudaStream_t st);

agnes_status product_check_sizes(const char* op, int64_t rows, int64_t width, int64_t dim);
agnes_status product_check_step(const char* op, const char* name, int64_t rows, int64_t cols,
                                int64_t stride);
agnes_status product_check_workspace(const char* op, const void* p, int64_t bytes, int64_t need,
                                     int device);
agnes_status check_direct(const char* op, int32_t grad_dtype, int32_t direct);

}  // namespace agnes
