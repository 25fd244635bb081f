// mx4.cu -- rows to microscaled 4-bit floating point and back
// (include/agnes_ops.h; the format is in mx4.cuh).
//
// Bound by memory where the instructions leave it: a thread takes 16 values, so that
// two share a block of 32, whose largest magnitude takes one exchange.  Magnitudes are
// compared as bit patterns, which order as the numbers do and put what is not finite on
// top, two 16-bit ones at once.
#include <type_traits>

#include "mx4.cuh"
#include "ops_common.cuh"

namespace agnes {

namespace {

constexpr int kThreads = 256;
constexpr int kItems = kFlat / kThreads;  // groups of eight values per thread, to dequantise
constexpr int kQuantThreads = 512;
constexpr int kQuantItems = kFlat / kQuantThreads;  // groups of sixteen, to quantise

// Sixteen values of a row.
template <typename T>
struct Sixteen {
  static constexpr int kWords = 16 * sizeof(T) / 4;
  uint32_t w[kWords];
};

// From column col0 of a row on, zeros past its end; kWide: rows are 16-byte aligned
// and a whole number of eights.
template <typename T, bool kWide>
__device__ __forceinline__ void load16(const T* row, int32_t col0, int32_t dim, Sixteen<T>& x) {
  if constexpr (kWide) {
    constexpr int kN = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 16 / kN; ++h) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (col0 + h * kN < dim) v = __ldg((const uint4*)(row + col0 + h * kN));
      x.w[4 * h] = v.x;
      x.w[4 * h + 1] = v.y;
      x.w[4 * h + 2] = v.z;
      x.w[4 * h + 3] = v.w;
    }
  } else {
    T* e = (T*)x.w;
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = col0 + i < dim ? row[col0 + i] : from_f32<T>(0.f);
  }
}

// The largest magnitude, as the bits of a float.
__device__ __forceinline__ uint32_t top_of(const Sixteen<float>& x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, x.w[i] & 0x7fffffffu);
  return top;
}
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Sixteen<T>& x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = __vmaxu2(top, x.w[i] & 0x7fff7fffu);
  const uint16_t bits = (uint16_t)max(top & 0xffffu, top >> 16);
  return __float_as_uint(to_f32(*(const T*)&bits));
}

// Values 2 i and 2 i + 1.
__device__ __forceinline__ float2 two_of(const Sixteen<float>& x, int i) {
  return make_float2(__uint_as_float(x.w[2 * i]), __uint_as_float(x.w[2 * i + 1]));
}
__device__ __forceinline__ float2 two_of(const Sixteen<__half>& x, int i) {
  return __half22float2(*(const __half2*)&x.w[i]);
}
__device__ __forceinline__ float2 two_of(const Sixteen<__nv_bfloat16>& x, int i) {
  return make_float2(__uint_as_float(x.w[i] << 16), __uint_as_float(x.w[i] & 0xffff0000u));
}

// groups: 2 * blocks, groups of sixteen values per row.  kWords: a multiple of 8, so that
// eight lanes hold four whole blocks of a row and their scales are stored as a word
// (2M fp16 rows of 128 values, groups of eight: a byte each, and the padding by bytes,
// 233 us; by words 215; by groups of sixteen 96).
template <typename T, bool kWide, bool kWords>
__global__ void __launch_bounds__(kQuantThreads)
quantize_kernel(const T* __restrict__ x, int64_t rows, int64_t stride, int32_t dim, int32_t groups,
                uint32_t inv_groups, uint8_t* __restrict__ out, int64_t out_stride,
                int32_t row_bytes) {
  const FlatRows flat(blockIdx.x, groups, inv_groups);
  int64_t row[kQuantItems];
  uint32_t group[kQuantItems];
  Sixteen<T> v[kQuantItems];
#pragma unroll
  for (int u = 0; u < kQuantItems; ++u) {
    flat.at(threadIdx.x + u * kQuantThreads, &row[u], &group[u]);
    if (row[u] < rows) {
      load16<T, kWide>(x + row[u] * stride, (int32_t)group[u] * 16, dim, v[u]);
    } else {
#pragma unroll
      for (int i = 0; i < Sixteen<T>::kWords; ++i) v[u].w[i] = 0;
    }
  }
#pragma unroll
  for (int u = 0; u < kQuantItems; ++u) {
    uint32_t top = top_of(v[u]);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));  // a row has an even number
    const uint32_t exponent = top >> 23;  // floor(log2) + 127 of a normal magnitude
    const bool fine = exponent < 255;
    const uint32_t byte = !fine ? 255u : exponent > 2 ? exponent - 2 : 0u;
    // 1 / scale = 2^(127 - byte): a normal number, so the products are exact
    // where they are not far below the smallest step
    const float inv = fine ? __uint_as_float((254u - byte) << 23) : 0.f;
    uint32_t codes[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 t = two_of(v[u], 4 * h + i);
        f[2 * i] = t.x * inv;
        f[2 * i + 1] = t.y * inv;
      }
      codes[h] = fine ? mx4_codes8(f) : 0u;
    }
    uint32_t word = 0;
    if constexpr (kWords) {  // four blocks' scales, of eight lanes
      word = byte << (4 * (threadIdx.x & 6));
      word |= __shfl_xor_sync(0xffffffffu, word, 2);
      word |= __shfl_xor_sync(0xffffffffu, word, 4);
    }
    if (row[u] >= rows) continue;
    uint8_t* to = out + row[u] * out_stride;
    *(uint2*)(to + group[u] * 8) = make_uint2(codes[0], codes[1]);
    const int32_t blocks = groups >> 1;
    if constexpr (kWords) {
      if ((group[u] & 7) == 0) *(uint32_t*)(to + blocks * 16 + (group[u] >> 1)) = word;
      // the padding: three words at most, by the row's last lanes
      const uint32_t pad = blocks * 17 + (group[u] & 7) * 4;
      if (group[u] >= (uint32_t)groups - 8 && pad < (uint32_t)row_bytes)
        *(uint32_t*)(to + pad) = 0;
    } else {
      if ((group[u] & 1) == 0) to[blocks * 16 + (group[u] >> 1)] = (uint8_t)byte;
      if (group[u] == 0)
        for (int32_t b = blocks * 17; b < row_bytes; ++b) to[b] = 0;
    }
  }
}

template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t* __restrict__ x, int64_t rows, int64_t stride, int32_t dim,
                  int32_t groups, uint32_t inv_groups, T* __restrict__ out, int64_t out_stride) {
  const FlatRows flat(blockIdx.x, groups, inv_groups);
  const int32_t blocks = (dim + kMxBlock - 1) / kMxBlock;
  int64_t row[kItems];
  uint32_t group[kItems], codes[kItems], byte[kItems];
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    flat.at(threadIdx.x + u * kThreads, &row[u], &group[u]);
    codes[u] = byte[u] = 0;
    if (row[u] < rows) {
      const uint8_t* from = x + row[u] * stride;
      codes[u] = __ldg((const uint32_t*)from + group[u]);
      byte[u] = __ldg(from + (int64_t)blocks * 16 + (group[u] >> 2));
    }
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    if (row[u] >= rows) continue;
    const float scale = mx4_scale(byte[u]);
    __half2 h[4];
    mx4_values(codes[u], h);
    T y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(h[e]);
      y[2 * e] = from_f32<T>(f.x * scale);
      y[2 * e + 1] = from_f32<T>(f.y * scale);
    }
    T* to = out + row[u] * out_stride + (int64_t)group[u] * 8;
    if constexpr (kWide) {
      constexpr int kN = 16 / sizeof(T);
#pragma unroll
      for (int p = 0; p < 8 / kN; ++p) {
        Vec<T, kN> v;
#pragma unroll
        for (int e = 0; e < kN; ++e) v.v[e] = y[p * kN + e];
        ((Vec<T, kN>*)to)[p] = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((int32_t)group[u] * 8 + e < dim) to[e] = y[e];
    }
  }
}

// Values of rows that are not whole eights, to a contiguous output taken as one run:
// eight of it to a thread, from one row or from the end of one and the start of the next
// (dim of 8 or more).  A row's codes from any value on are two words, shifted.
// (Eight values of a row to a thread, stored one by one: 498,000 rows of 301 to fp16 392
// us, now 124.)
template <typename T>
__global__ void __launch_bounds__(kThreads)
dequantize_flat_kernel(const uint8_t* __restrict__ x, int64_t rows, int64_t stride, int32_t dim,
                       uint32_t inv_dim, T* __restrict__ out) {
  constexpr int kTurns = kFlatRun / (kThreads * 8);
  const FlatRun flat(blockIdx.x, dim, inv_dim);
  const int32_t blocks = (dim + kMxBlock - 1) / kMxBlock, words = blocks * 4;
  const int64_t total = rows * dim;
  uint32_t codes[kTurns];
  float s0[kTurns], s1[kTurns], s2[kTurns];
  int left[kTurns], same[kTurns];  // values of the first row, and of its first block
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    int64_t row;
    uint32_t col;
    flat.at((uint32_t)((u * kThreads + threadIdx.x) * 8), &row, &col);
    codes[u] = 0;
    s0[u] = s1[u] = s2[u] = 0.f;
    left[u] = (int)(dim - col);
    same[u] = (int)(kMxBlock - col % kMxBlock);
    if (row >= rows) continue;
    const uint8_t* from = x + row * stride;
    const uint8_t* scales = from + (int64_t)blocks * 16;
    const int w = (int)(col >> 3), b = (int)(col / kMxBlock);
    const uint32_t low = __ldg((const uint32_t*)from + w);
    const uint32_t high = __ldg((const uint32_t*)from + min(w + 1, words - 1));
    codes[u] = __funnelshift_r(low, high, 4 * (col & 7));
    s0[u] = mx4_scale(__ldg(scales + b));
    s1[u] = mx4_scale(__ldg(scales + min(b + 1, blocks - 1)));
    if (left[u] < 8) {
      uint32_t next = 0;
      if (row + 1 < rows) {
        next = __ldg((const uint32_t*)(from + stride));
        s2[u] = mx4_scale(__ldg(scales + stride));
      }
      codes[u] = (codes[u] & ((1u << (4 * left[u])) - 1u)) | next << (4 * left[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int64_t at = (int64_t)blockIdx.x * kFlatRun + (u * kThreads + threadIdx.x) * 8;
    __half2 h[4];
    mx4_values(codes[u], h);
    constexpr int kN = 16 / sizeof(T);
    Vec<T, kN> y[8 / kN];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = e & 1 ? __high2float(h[e >> 1]) : __low2float(h[e >> 1]);
      y[e / kN].v[e % kN] = from_f32<T>(f * (e >= left[u] ? s2[u] : e < same[u] ? s0[u] : s1[u]));
    }
    if (at + 8 <= total) {
#pragma unroll
      for (int p = 0; p < 8 / kN; ++p) ((Vec<T, kN>*)(out + at))[p] = y[p];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < total) out[at + e] = y[e / kN].v[e % kN];
    }
  }
}

constexpr int64_t kMaxDim = 1 << 26;  // 2^26 / 32 blocks of 17 bytes fit 32 bits
constexpr int64_t kMaxRows = 0x7fffffff - 255;

agnes_status check_rows(const char* op, int64_t rows, int64_t dim, int64_t stride,
                        int64_t packed_stride) {
  if (rows < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, dim %lld", op, (long long)rows, (long long)dim);
  if (rows > kMaxRows || dim > kMaxDim)
    return op_error(AGNES_ERANGE, "%s: rows %lld, dim %lld are too large", op, (long long)rows,
                    (long long)dim);
  if (rows > 1 && stride < dim)
    return op_error(AGNES_EINVAL, "%s: a stride of %lld is below dim %lld", op, (long long)stride,
                    (long long)dim);
  return mx4_check_stride(op, "packed", rows, dim, packed_stride);
}

// f(rows per call's groups, inverse, blocks) after the sizes' checks.
struct MxGrid {
  int32_t groups;
  uint32_t inv;
  int64_t ctas;
};

MxGrid mx_grid(int64_t rows, int64_t groups) {
  return {(int32_t)groups, flat_inverse(groups), ceil_div(rows * groups, kFlat)};
}

}  // namespace

agnes_status mx4_check_stride(const char* op, const char* name, int64_t rows, int64_t dim,
                              int64_t stride) {
  if (rows > 1 && (stride < mx4_row_bytes(dim) || stride % 16))
    return op_error(AGNES_EINVAL,
                    "%s: a stride of %lld bytes of %s is not a multiple of 16 of at least %lld", op,
                    (long long)stride, name, (long long)mx4_row_bytes(dim));
  return AGNES_OK;
}

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_mx4_row_bytes(int64_t dim, int64_t* bytes) {
  const char* op = "agnes_mx4_row_bytes";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_rows(op, 0, dim, dim, 0));
  *bytes = mx4_row_bytes(dim);
  return AGNES_OK;
}

agnes_status agnes_mx4_quantize(const void* x, int32_t dtype, int64_t stride, int64_t rows,
                                int64_t dim, void* out, int64_t out_stride, void* cuda_stream) {
  const char* op = "agnes_mx4_quantize";
  OP_TRY(check_rows(op, rows, dim, stride, out_stride));
  OP_TRY(op_float_type(op, "x", dtype));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "x", x, &device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "x", x, float_size(dtype)));
  OP_TRY(op_aligned(op, "out", out, 16));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const MxGrid g = mx_grid(rows, 2 * mx4_blocks(dim));
  if (g.ctas > 0x7fffffff) return op_error(AGNES_ERANGE, "%s: rows * dim is too large", op);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = with_float_type(dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    const bool wide =
        dim % 8 == 0 && aligned_rows(x, rows > 1 ? stride * (int64_t)sizeof(T) : 0, 16);
    const bool words = g.groups % 8 == 0;
    const auto kernel = wide ? (words ? quantize_kernel<T, true, true>
                                      : quantize_kernel<T, true, false>)
                             : (words ? quantize_kernel<T, false, true>
                                      : quantize_kernel<T, false, false>);
    kernel<<<(unsigned)g.ctas, kQuantThreads, 0, st>>>(
        (const T*)x, rows, stride, (int32_t)dim, g.groups, g.inv, (uint8_t*)out, out_stride,
        (int32_t)mx4_row_bytes(dim));
    return cudaGetLastError();
  });
  return op_launched(op, e);
}

agnes_status agnes_mx4_dequantize(const void* x, int64_t stride, int64_t rows, int64_t dim,
                                  void* out, int32_t dtype, int64_t out_stride,
                                  void* cuda_stream) {
  const char* op = "agnes_mx4_dequantize";
  OP_TRY(check_rows(op, rows, dim, out_stride, stride));
  OP_TRY(op_float_type(op, "out", dtype));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "x", x, &device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "x", x, 16));
  OP_TRY(op_aligned(op, "out", out, float_size(dtype)));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const MxGrid g = mx_grid(rows, ceil_div(dim, 8));
  if (g.ctas > 0x7fffffff) return op_error(AGNES_ERANGE, "%s: rows * dim is too large", op);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = with_float_type(dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    const bool wide =
        dim % 8 == 0 && aligned_rows(out, rows > 1 ? out_stride * (int64_t)sizeof(T) : 0, 16);
    if (!wide && dim >= 8 && (rows == 1 || out_stride == dim) && (uintptr_t)out % 16 == 0 &&
        ceil_div(rows * dim, kFlatRun) <= 0x7fffffff) {
      dequantize_flat_kernel<T><<<(unsigned)ceil_div(rows * dim, kFlatRun), kThreads, 0, st>>>(
          (const uint8_t*)x, rows, stride, (int32_t)dim, flat_inverse(dim), (T*)out);
      return cudaGetLastError();
    }
    (wide ? dequantize_kernel<T, true> : dequantize_kernel<T, false>)<<<(unsigned)g.ctas, kThreads,
                                                                        0, st>>>(
        (const uint8_t*)x, rows, stride, (int32_t)dim, g.groups, g.inv, (T*)out, out_stride);
    return cudaGetLastError();
  });
  return op_launched(op, e);
}

}  // extern "C"
