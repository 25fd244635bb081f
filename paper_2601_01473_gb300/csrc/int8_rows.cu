// int8_rows.cu -- rows to 8 bits and back, and nonlinearities whose input is kept in 8
// bits for their backward pass (include/agnes_ops.h; the format is in int8.cuh).
//
// Bound by memory: a group of threads holds a row in registers, so it is read once, for
// its largest magnitude, its whole numbers and its nonlinearity; rows of more than 8192
// values are read again, from L2 as far as it holds them.
#include "int8.cuh"

namespace agnes {

namespace {

constexpr int kElems = 8;  // values of a row to a thread at a time

struct KeepArgs {
  const void* x;
  int64_t stride, rows;
  int32_t dim;       // of a half where gated
  int32_t lanes, groups;
  int32_t f;         // AGNES_F_*, or -1: no nonlinearity
  bool gated;        // rows of 2 dim values
  bool out_rows8;
  void* out;         // may be null where f is -1
  int64_t out_stride;
  uint8_t* kept;     // may be null
  int64_t kept_stride;
};

// f(v), and its derivative where one is asked for.
template <bool kSlope>
__device__ __forceinline__ float nonlinear(int32_t f, float v, float* slope) {
  if (f == AGNES_F_RELU) {
    if (kSlope) *slope = v > 0.f ? 1.f : v <= 0.f ? 0.f : v;
    return v < 0.f ? 0.f : v;
  }
  if (f == AGNES_F_SILU) {
    const float p = __fdividef(1.f, 1.f + expf(-v));
    if (kSlope) *slope = p * fmaf(v, 1.f - p, 1.f);
    return v * p;
  }
  const float p = normcdff(v);
  if (kSlope) *slope = fmaf(v * 0.3989422804f, expf(-0.5f * v * v), p);  // 1 / sqrt(2 pi)
  return v * p;
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <typename T, int kVec, bool kLoop>
__global__ void __launch_bounds__(kRowLanesMax)
keep_kernel(const KeepArgs a) {
  constexpr int kPer = kElems / kVec;
  __shared__ RowScratch scratch;
  int turn = 0;
  const int group = threadIdx.x / a.lanes, lane = threadIdx.x - group * a.lanes;
  const int64_t row = (int64_t)blockIdx.x * a.groups + group;
  const bool valid = row < a.rows;
  const T* x = (const T*)a.x + row * a.stride;
  const int32_t chunk = a.lanes * kElems;
  float v[kElems], u[kElems], y[kElems];
  // columns c0 on of the row, and what is made of them
  const auto load = [&](int32_t c0) {
    const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
    part.load(x + c0, valid, v);
    if (a.gated) part.load(x + a.dim + c0, valid, u);
    if (a.f < 0) return;
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
      y[e] = nonlinear<false>(a.f, v[e], nullptr);
      if (a.gated) y[e] *= u[e];
    }
  };
  uint32_t top[3] = {0, 0, 0};
  const bool tops = a.kept || a.out_rows8;
  if (kLoop || tops || a.f >= 0) {
    for (int32_t c0 = 0; c0 < (kLoop ? a.dim : 1); c0 += chunk) {
      load(c0);
      if (!tops) break;
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        top[0] = max(top[0], magnitude(v[e]));
        if (a.gated) top[1] = max(top[1], magnitude(u[e]));
        if (a.out_rows8) top[2] = max(top[2], magnitude(y[e]));
      }
    }
  }
  Int8Scale s[3];
  if (tops) {
    group_reduce<MaxBits>(top, a.lanes, &scratch, turn);
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] = int8_scale(top[k]);
  }
  uint8_t* kept = a.kept + row * a.kept_stride;
  const int64_t half = int8_row_bytes(a.dim);
  uint8_t* out8 = (uint8_t*)a.out + row * a.out_stride;
  T* out = (T*)a.out + row * a.out_stride;
  for (int32_t c0 = 0; c0 < (kLoop ? a.dim : 1); c0 += chunk) {
    if (kLoop) load(c0);
    const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
    if (a.kept) {
      int8_store(part, kept + c0, valid, v, s[0]);
      if (a.gated) int8_store(part, kept + half + c0, valid, u, s[1]);
    }
    if (a.out_rows8)
      int8_store(part, out8 + c0, valid, y, s[2]);
    else if (a.f >= 0)
      part.store(out + c0, valid, y);
  }
  if (a.kept) {
    int8_store_end(kept, a.dim, lane, a.lanes, valid, s[0]);
    if (a.gated) int8_store_end(kept + half, a.dim, lane, a.lanes, valid, s[1]);
  }
  if (a.out_rows8) int8_store_end(out8, a.dim, lane, a.lanes, valid, s[2]);
}

struct BackArgs {
  const uint8_t* kept;
  int64_t kept_stride, rows;
  int32_t dim, lanes, groups;
  int32_t f;
  bool gated;
  const void* grad;  // null: the kept values themselves
  int64_t grad_stride;
  void* out;
  int64_t out_stride;
};

// The largest number of a type: a value past it is that (the row's scale was rounded up).
template <typename T>
__device__ __forceinline__ float most_of();
template <>
__device__ __forceinline__ float most_of<float>() {
  return 3.402823466e38f;
}
template <>
__device__ __forceinline__ float most_of<__half>() {
  return 65504.f;
}
template <>
__device__ __forceinline__ float most_of<__nv_bfloat16>() {
  return 3.3895313892515355e38f;
}

// What 8-bit rows stand for, or the nonlinearity's gradient at it.
template <typename TGrad, typename T, int kVec, bool kGrad>
__global__ void __launch_bounds__(kRowLanesMax)
back_kernel(const BackArgs a) {
  constexpr int kPer = kElems / kVec;
  const int group = threadIdx.x / a.lanes, lane = threadIdx.x - group * a.lanes;
  const int64_t row = (int64_t)blockIdx.x * a.groups + group;
  const bool valid = row < a.rows;
  if (!valid) return;
  const uint8_t* kept = a.kept + row * a.kept_stride;
  const int64_t half = int8_row_bytes(a.dim);
  const float s0 = *(const float*)(kept + half - 4);
  const float s1 = kGrad && a.gated ? *(const float*)(kept + 2 * half - 4) : 0.f;
  T* out = (T*)a.out + row * a.out_stride;
  const TGrad* grad = (const TGrad*)a.grad + row * a.grad_stride;
  for (int32_t c0 = 0; c0 < a.dim; c0 += a.lanes * kElems) {
    const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
    float v[kElems], u[kElems], d[kElems];
    int8_load(part, kept + c0, true, v);
    if constexpr (!kGrad) {
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const float most = most_of<T>(), y = v[e] * s0;
        v[e] = y > most ? most : y < -most ? -most : y;
      }
      part.store(out + c0, true, v);
    } else {
      if (a.gated) int8_load(part, kept + half + c0, true, u);
      part.load(grad + c0, true, d);
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        float slope;
        const float y = nonlinear<true>(a.f, v[e] * s0, &slope);
        v[e] = d[e] * slope;
        if (a.gated) {
          v[e] *= u[e] * s1;
          u[e] = d[e] * y;
        }
      }
      part.store(out + c0, true, v);
      if (a.gated) part.store(out + a.dim + c0, true, u);
    }
  }
}

// The elements of an access for rows of dim values that start at p and every stride after
// it: a vector needs each of its accesses aligned.
int vec_of(int64_t dim, bool aligned) { return aligned && dim % 8 == 0 ? 8 : 1; }

agnes_status check_sizes(const char* op, int64_t rows, int64_t dim) {
  if (rows < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, dim %lld", op, (long long)rows, (long long)dim);
  if (rows > kInt8MaxRows || dim > kInt8MaxDim)
    return op_error(AGNES_ERANGE, "%s: rows %lld, dim %lld are too large", op, (long long)rows,
                    (long long)dim);
  return AGNES_OK;
}

agnes_status check_step(const char* op, const char* name, int64_t rows, int64_t cols,
                        int64_t stride) {
  if (rows > 1 && stride < cols)
    return op_error(AGNES_EINVAL, "%s: a stride of %lld of %s is below %lld", op, (long long)stride,
                    name, (long long)cols);
  return AGNES_OK;
}

// `halves` 8-bit rows side by side.
agnes_status check_kept(const char* op, const char* name, int64_t rows, int64_t dim, int halves,
                        int64_t stride) {
  if (rows > 1 && (stride < halves * int8_row_bytes(dim) || stride % 16))
    return op_error(AGNES_EINVAL,
                    "%s: a stride of %lld bytes of %s is not a multiple of 16 of at least %lld", op,
                    (long long)stride, name, (long long)(halves * int8_row_bytes(dim)));
  return AGNES_OK;
}

template <typename T>
cudaError_t launch_keep(KeepArgs a, cudaStream_t st) {
  const int64_t next = a.rows > 1 ? 1 : 0;  // a single row has no next one
  const bool aligned =
      aligned_rows(a.x, next * a.stride * (int64_t)sizeof(T), 16) &&
      (a.f < 0 || a.out_rows8 || aligned_rows(a.out, next * a.out_stride * (int64_t)sizeof(T), 16));
  const RowShape shape = row_shape(a.dim, kElems);
  a.lanes = shape.lanes;
  a.groups = shape.groups;
  const bool loop = a.dim > a.lanes * kElems;
  const auto kernel = vec_of(a.dim, aligned) == 8
                          ? (loop ? keep_kernel<T, 8, true> : keep_kernel<T, 8, false>)
                          : (loop ? keep_kernel<T, 1, true> : keep_kernel<T, 1, false>);
  kernel<<<(unsigned)ceil_div(a.rows, a.groups), shape.threads(), 0, st>>>(a);
  return cudaGetLastError();
}

template <typename TGrad, typename T, bool kGrad>
cudaError_t launch_back(BackArgs a, cudaStream_t st) {
  const int64_t next = a.rows > 1 ? 1 : 0;
  const bool aligned =
      aligned_rows(a.out, next * a.out_stride * (int64_t)sizeof(T), 16) &&
      (!kGrad || aligned_rows(a.grad, next * a.grad_stride * (int64_t)sizeof(TGrad), 16));
  const RowShape shape = row_shape(a.dim, kElems);
  a.lanes = shape.lanes;
  a.groups = shape.groups;
  const auto kernel = vec_of(a.dim, aligned) == 8 ? back_kernel<TGrad, T, 8, kGrad>
                                                  : back_kernel<TGrad, T, 1, kGrad>;
  kernel<<<(unsigned)ceil_div(a.rows, a.groups), shape.threads(), 0, st>>>(a);
  return cudaGetLastError();
}

agnes_status check_f(const char* op, int32_t f, int32_t gated) {
  if (f != AGNES_F_RELU && f != AGNES_F_SILU && f != AGNES_F_GELU)
    return op_error(AGNES_EINVAL, "%s: an unknown nonlinearity (%d)", op, f);
  if (gated != 0 && gated != 1) return op_error(AGNES_EINVAL, "%s: gated is %d", op, gated);
  return AGNES_OK;
}

}  // namespace

agnes_status int8_check_stride(const char* op, const char* name, int64_t rows, int64_t dim,
                               int64_t stride) {
  return check_kept(op, name, rows, dim, 1, stride);
}

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_int8_row_bytes(int64_t dim, int64_t* bytes) {
  const char* op = "agnes_int8_row_bytes";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_sizes(op, 0, dim));
  *bytes = int8_row_bytes(dim);
  return AGNES_OK;
}

agnes_status agnes_int8_quantize(const void* x, int32_t dtype, int64_t stride, int64_t rows,
                                 int64_t dim, void* out, int64_t out_stride, void* cuda_stream) {
  const char* op = "agnes_int8_quantize";
  OP_TRY(check_sizes(op, rows, dim));
  OP_TRY(op_float_type(op, "x", dtype));
  OP_TRY(check_step(op, "x", rows, dim, stride));
  OP_TRY(check_kept(op, "out", rows, dim, 1, out_stride));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "x", x, &device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "x", x, float_size(dtype)));
  OP_TRY(op_aligned(op, "out", out, 16));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  KeepArgs a = {};
  a.x = x;
  a.stride = stride;
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.f = -1;
  a.kept = (uint8_t*)out;
  a.kept_stride = out_stride;
  return op_launched(op, with_float_type(dtype, [&](auto t) {
    return launch_keep<typename decltype(t)::type>(a, (cudaStream_t)cuda_stream);
  }));
}

agnes_status agnes_int8_dequantize(const void* x, int64_t stride, int64_t rows, int64_t dim,
                                   void* out, int32_t dtype, int64_t out_stride,
                                   void* cuda_stream) {
  const char* op = "agnes_int8_dequantize";
  OP_TRY(check_sizes(op, rows, dim));
  OP_TRY(op_float_type(op, "out", dtype));
  OP_TRY(check_step(op, "out", rows, dim, out_stride));
  OP_TRY(check_kept(op, "x", rows, dim, 1, stride));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "x", x, &device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "x", x, 16));
  OP_TRY(op_aligned(op, "out", out, float_size(dtype)));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  BackArgs a = {};
  a.kept = (const uint8_t*)x;
  a.kept_stride = stride;
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.out = out;
  a.out_stride = out_stride;
  return op_launched(op, with_float_type(dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    return launch_back<T, T, false>(a, (cudaStream_t)cuda_stream);
  }));
}

agnes_status agnes_activation(const void* x, int32_t dtype, int64_t stride, int64_t rows,
                              int64_t dim, int32_t f, int32_t gated, void* out, int32_t out_dtype,
                              int64_t out_stride, void* kept, int64_t kept_stride,
                              void* cuda_stream) {
  const char* op = "agnes_activation";
  OP_TRY(check_sizes(op, rows, dim));
  OP_TRY(op_float_type(op, "x", dtype));
  OP_TRY(check_f(op, f, gated));
  const int halves = gated ? 2 : 1;
  OP_TRY(check_step(op, "x", rows, halves * dim, stride));
  if (out_dtype == AGNES_INT8_ROWS) {
    OP_TRY(check_kept(op, "out", rows, dim, 1, out_stride));
  } else if (out_dtype != dtype) {
    return op_error(AGNES_EINVAL, "%s: out has another type than x", op);
  } else {
    OP_TRY(check_step(op, "out", rows, dim, out_stride));
  }
  if (kept) OP_TRY(check_kept(op, "kept", rows, dim, halves, kept_stride));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "x", x, &device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "x", x, float_size(dtype)));
  OP_TRY(op_aligned(op, "out", out, out_dtype == AGNES_INT8_ROWS ? 16 : float_size(dtype)));
  if (kept) {
    OP_TRY(op_on_device(op, "kept", kept, device));
    OP_TRY(op_aligned(op, "kept", kept, 16));
  }
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  KeepArgs a = {};
  a.x = x;
  a.stride = stride;
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.f = f;
  a.gated = gated != 0;
  a.out_rows8 = out_dtype == AGNES_INT8_ROWS;
  a.out = out;
  a.out_stride = out_stride;
  a.kept = (uint8_t*)kept;
  a.kept_stride = kept_stride;
  return op_launched(op, with_float_type(dtype, [&](auto t) {
    return launch_keep<typename decltype(t)::type>(a, (cudaStream_t)cuda_stream);
  }));
}

agnes_status agnes_activation_grad(const void* grad, int32_t grad_dtype, int64_t grad_stride,
                                   const void* kept, int64_t kept_stride, int64_t rows, int64_t dim,
                                   int32_t f, int32_t gated, void* out, int32_t out_dtype,
                                   int64_t out_stride, void* cuda_stream) {
  const char* op = "agnes_activation_grad";
  OP_TRY(check_sizes(op, rows, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(check_f(op, f, gated));
  const int halves = gated ? 2 : 1;
  OP_TRY(check_step(op, "grad", rows, dim, grad_stride));
  OP_TRY(check_step(op, "out", rows, halves * dim, out_stride));
  OP_TRY(check_kept(op, "kept", rows, dim, halves, kept_stride));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "kept", kept, &device));
  OP_TRY(op_on_device(op, "grad", grad, device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "kept", kept, 16));
  OP_TRY(op_aligned(op, "grad", grad, float_size(grad_dtype)));
  OP_TRY(op_aligned(op, "out", out, float_size(out_dtype)));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  BackArgs a = {};
  a.kept = (const uint8_t*)kept;
  a.kept_stride = kept_stride;
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.f = f;
  a.gated = gated != 0;
  a.grad = grad;
  a.grad_stride = grad_stride;
  a.out = out;
  a.out_stride = out_stride;
  return op_launched(op, with_float_type(grad_dtype, [&](auto t) {
    using TGrad = typename decltype(t)::type;
    return with_float_type(out_dtype, [&](auto o) {
      return launch_back<TGrad, typename decltype(o)::type, true>(a, (cudaStream_t)cuda_stream);
    });
  }));
}

}  // extern "C"
