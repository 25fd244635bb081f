// int8.cuh -- rows in 8 bits (include/agnes_ops.h): a row of dim values is its whole
// numbers q (a byte each), zeros, and its scale s in the last four of a multiple of 16
// bytes; it stands for q s.
//
// s is the row's largest magnitude / 127, rounded up to eight significant bits: a whole
// number times it has 15 bits, which are the sum of two bfloat16 values, so the tensor
// cores' products with a row's values are exact.  That costs the rounding 0.4% of a step
// at most (s is up to 2^-7 larger than it had to be, on average half that).  Rows that came
// another way may have any fp32 scale: the gradients' products keep 16 bits of their values.
#pragma once

#include "rows.cuh"

namespace agnes {

// Sums of whole products of up to 127^2 stay below 2^31.
constexpr int64_t kInt8MaxDim = 1 << 17;
constexpr int64_t kInt8MaxRows = 0x7fffffff - 255;

__host__ __device__ inline int64_t int8_row_bytes(int64_t dim) { return (dim + 4 + 15) / 16 * 16; }

// A stride in bytes between 8-bit rows of dim values (int8_rows.cu).
agnes_status int8_check_stride(const char* op, const char* name, int64_t rows, int64_t dim,
                               int64_t stride);

struct Int8Scale {
  float scale, inverse;
  bool fine;
};

// Of a row whose largest magnitude has the bits `top`.
__device__ __forceinline__ Int8Scale int8_scale(uint32_t top) {
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fffffffu), 0.f, false};
  const float most = __uint_as_float(top);
  if (most < 0x1p-100f) return {0.f, 0.f, true};
  const float s =
      __uint_as_float((__float_as_uint(__fdiv_rn(most, 127.f)) + 0xffffu) & 0xffff0000u);
  return {s, __frcp_rn(s), true};
}

// A value's whole number, in the low byte: adding 1.5 * 2^23 rounds to nearest even.
__device__ __forceinline__ uint32_t int8_code(float x, const Int8Scale& s) {
  return __float_as_uint(__fadd_rn(__fmul_rn(x, s.inverse), 12582912.f));
}
__device__ __forceinline__ uint32_t int8_codes4(const float* x, const Int8Scale& s) {
  const uint32_t low = __byte_perm(int8_code(x[0], s), int8_code(x[1], s), 0x0040);
  const uint32_t high = __byte_perm(int8_code(x[2], s), int8_code(x[3], s), 0x0040);
  return s.fine ? __byte_perm(low, high, 0x5410) : 0u;
}

// The four values of a word: xor 0x80 makes each byte q + 128, which the bytes of
// 2^23 + b hold as they are.
__device__ __forceinline__ void int8_values4(uint32_t word, float* q) {
  word ^= 0x80808080u;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    q[e] = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7540 + e)) - 8388736.f;
}

// Vector i of a thread's part of a row, to an 8-bit row at `to`; the group's threads write
// the row's zeros and scale besides.
template <int kVec, int kPer>
__device__ __forceinline__ void int8_store(const RowPart<kVec, kPer>& part, uint8_t* to, bool valid,
                                           int i, const float* v, const Int8Scale& s) {
  const int32_t c = part.col(i);
  if (!valid || c >= part.dim) return;
  if constexpr (kVec == 1) {
    to[c] = s.fine ? (uint8_t)int8_code(v[0], s) : 0;
  } else {
    static_assert(kVec == 8, "8 bytes a store");
    *(uint2*)(to + c) = make_uint2(int8_codes4(v, s), int8_codes4(v + 4, s));
  }
}
__device__ __forceinline__ void int8_store_end(uint8_t* to, int32_t dim, int lane, int lanes,
                                               bool valid, const Int8Scale& s) {
  if (!valid) return;
  const int32_t end = (int32_t)int8_row_bytes(dim) - 4;
  for (int32_t b = dim + lane; b < end; b += lanes) to[b] = 0;
  if (lane == 0) *(float*)(to + end) = s.scale;
}

// A thread's part of an 8-bit row as it lies in memory.
template <int kVec, int kPer>
struct Int8Regs {
  uint2 w[kPer];
  __device__ void load(const RowPart<kVec, kPer>& part, const uint8_t* row, bool valid) {
    static_assert(kVec == 8, "8 bytes a load");
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      w[i] = valid && part.has(i) ? *(const uint2*)(row + part.col(i)) : make_uint2(0, 0);
  }
  __device__ void get(int i, float* q) const {
    int8_values4(w[i].x, q);
    int8_values4(w[i].y, q + 4);
  }
};
template <int kPer>
struct Int8Regs<1, kPer> {
  int8_t q[kPer];
  __device__ void load(const RowPart<1, kPer>& part, const uint8_t* row, bool valid) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      q[i] = valid && part.has(i) ? (int8_t)row[part.col(i)] : (int8_t)0;
  }
  __device__ void get(int i, float* f) const { f[0] = (float)q[i]; }
};

}  // namespace agnes
