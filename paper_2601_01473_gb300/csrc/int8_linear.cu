// int8_linear.cu -- 8-bit rows times 8-bit weights, and the gradients of that product
// (include/agnes_ops.h; the format is in int8.cuh).
//
//   out[r][j] = s_x[r] s_w[j] sum_i q_x[r][i] q_w[j][i] + bias[j]
//   dw[j][i]  = sum_r grad[r][j] s_x[r] q_x[r][i]
//   dx[r][i]  = sum_j grad[r][j] s_w[j] q_w[j][i]
//
// Few rows: the weights' bytes count, so a group of lanes takes a column's whole numbers,
// four products an instruction, for all rows.
// Otherwise tiles of 64 x 64 outputs, 4 x 4 to a thread, over slices of 16 staged in
// shared memory as fp32; sums of 4096 products in fp32, those in 64 bits.
#include "int8.cuh"

namespace agnes {

namespace {

// ---- few rows ------------------------------------------------------------------

constexpr int kFewThreads = 256;
constexpr int kFewCols = 2;  // of the output to a group of lanes at a time

struct LinearArgs {
  const uint8_t *x, *w;
  int64_t x_stride, w_stride;
  int64_t rows, width;
  int32_t dim, row_bytes;
  const float* bias;
  void* out;
  int64_t out_stride;
};

// The whole product of a sum and two scales: the smaller scale first, so that what is
// finite in the end does not overflow on the way.
__device__ __forceinline__ float scaled(float sum, float a, float b) {
  const bool less = a < b;  // a NaN is a factor either way
  return sum * (less ? a : b) * (less ? b : a);
}

template <typename TOut, int kRows>
__global__ void __launch_bounds__(kFewThreads)
linear_few_kernel(int lanes, const LinearArgs a) {
  const int lane = threadIdx.x % lanes;
  const int64_t groups = (int64_t)gridDim.x * (kFewThreads / lanes);
  const int chunks = (a.dim + 15) / 16;
  for (int64_t j0 = ((int64_t)blockIdx.x * (kFewThreads / lanes) + threadIdx.x / lanes) * kFewCols;
       // whole warps stay together for the exchange
       j0 - (threadIdx.x % 32) / lanes * kFewCols < a.width; j0 += groups * kFewCols) {
    int32_t sum[kRows * kFewCols];
#pragma unroll
    for (int k = 0; k < kRows * kFewCols; ++k) sum[k] = 0;
    for (int c = lane; c < chunks; c += lanes) {
      uint4 w[kFewCols];
#pragma unroll
      for (int k = 0; k < kFewCols; ++k)
        w[k] = j0 + k < a.width ? __ldg((const uint4*)(a.w + (j0 + k) * a.w_stride) + c)
                                : make_uint4(0, 0, 0, 0);
      uint4 keep = make_uint4(~0u, ~0u, ~0u, ~0u);
      if (c == chunks - 1) {  // the row's scale may be in its last 16 bytes
        const int left = a.dim - c * 16;
        const auto mask = [&](int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; };
        keep = make_uint4(mask(left), mask(left - 4), mask(left - 8), mask(left - 12));
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        if (r >= a.rows) break;
        uint4 x = __ldg((const uint4*)(a.x + r * a.x_stride) + c);
        x = make_uint4(x.x & keep.x, x.y & keep.y, x.z & keep.z, x.w & keep.w);
#pragma unroll
        for (int k = 0; k < kFewCols; ++k) {
          int32_t s = sum[r * kFewCols + k];
          s = __dp4a((int)x.x, (int)w[k].x, s);
          s = __dp4a((int)x.y, (int)w[k].y, s);
          s = __dp4a((int)x.z, (int)w[k].z, s);
          sum[r * kFewCols + k] = __dp4a((int)x.w, (int)w[k].w, s);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kRows * kFewCols; ++k)
      for (int d = lanes / 2; d > 0; d >>= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], d);
    if (lane) continue;
#pragma unroll
    for (int k = 0; k < kFewCols; ++k) {
      if (j0 + k >= a.width) break;
      const float sw = *(const float*)(a.w + (j0 + k) * a.w_stride + a.row_bytes - 4);
      const float b = a.bias ? __ldg(a.bias + j0 + k) : 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        if (r >= a.rows) break;
        const float sx = *(const float*)(a.x + r * a.x_stride + a.row_bytes - 4);
        ((TOut*)a.out)[r * a.out_stride + j0 + k] =
            from_f32<TOut>(scaled((float)sum[r * kFewCols + k], sx, sw) + b);
      }
    }
  }
}

// ---- tiles ----------------------------------------------------------------------

constexpr int kTile = 64, kSlice = 16, kChunk = 4096;

// out[m][n] = sum_k A(m, k) B(n, k), A and B functions of two indexes.
template <typename A, typename B, typename Out>
__device__ __forceinline__ void tile_product(int64_t M, int64_t N, int64_t K, A&& fa, B&& fb,
                                             Out&& out) {
  __shared__ float sa[kSlice][kTile + 4], sb[kSlice][kTile + 4];
  const int64_t m0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
  const int tm = threadIdx.x / 16 * 4, tn = threadIdx.x % 16 * 4;
  double total[4][4] = {};
  float sum[4][4] = {};
  for (int64_t k0 = 0; k0 < K; k0 += kSlice) {
    for (int i = threadIdx.x; i < kTile * kSlice; i += 256) {
      const int r = i / kSlice, k = i % kSlice;
      sa[k][r] = m0 + r < M && k0 + k < K ? fa(m0 + r, k0 + k) : 0.f;
      sb[k][r] = n0 + r < N && k0 + k < K ? fb(n0 + r, k0 + k) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSlice; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = fmaf(sa[k][tm + i], sb[k][tn + j], sum[i][j]);
    __syncthreads();
    if (k0 % kChunk == kChunk - kSlice || k0 + kSlice >= K) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          total[i][j] += sum[i][j];
          sum[i][j] = 0.f;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (m0 + tm + i < M && n0 + tn + j < N) out(m0 + tm + i, n0 + tn + j, total[i][j]);
}

template <typename TOut>
__global__ void __launch_bounds__(256) linear_kernel(const LinearArgs a) {
  const int end = a.row_bytes - 4;
  tile_product(
      a.rows, a.width, a.dim,
      [&](int64_t r, int64_t i) { return (float)(int8_t)a.x[r * a.x_stride + i]; },
      [&](int64_t j, int64_t i) { return (float)(int8_t)a.w[j * a.w_stride + i]; },
      [&](int64_t r, int64_t j, double v) {
        const float sx = *(const float*)(a.x + r * a.x_stride + end);
        const float sw = *(const float*)(a.w + j * a.w_stride + end);
        ((TOut*)a.out)[r * a.out_stride + j] =
            from_f32<TOut>(scaled((float)v, sx, sw) + (a.bias ? a.bias[j] : 0.f));
      });
}

struct GradArgs {
  const void* grad;
  int64_t grad_stride, rows, width;
  const uint8_t* q;  // x's rows, or w's
  int64_t q_stride;
  int32_t dim, row_bytes;
  void* out;
  int64_t out_stride;
  float* dbias;
};

template <typename TGrad, typename TOut>
__global__ void __launch_bounds__(256) grad_weight_kernel(const GradArgs a) {
  const int end = a.row_bytes - 4;
  tile_product(
      a.width, a.dim, a.rows,
      [&](int64_t j, int64_t r) {
        return to_f32(((const TGrad*)a.grad)[r * a.grad_stride + j]);
      },
      [&](int64_t i, int64_t r) {
        const uint8_t* row = a.q + r * a.q_stride;
        return (float)(int8_t)row[i] * *(const float*)(row + end);
      },
      [&](int64_t j, int64_t i, double v) {
        ((TOut*)a.out)[j * a.out_stride + i] = from_f32<TOut>((float)v);
      });
}

template <typename TGrad>
__global__ void __launch_bounds__(256) grad_bias_kernel(const GradArgs a) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (j >= a.width) return;
  double sum = 0;
  for (int64_t r = 0; r < a.rows; ++r) sum += to_f32(((const TGrad*)a.grad)[r * a.grad_stride + j]);
  a.dbias[j] = (float)sum;
}

template <typename TGrad, typename TOut>
__global__ void __launch_bounds__(256) grad_input_kernel(const GradArgs a) {
  const int end = a.row_bytes - 4;
  tile_product(
      a.rows, a.dim, a.width,
      [&](int64_t r, int64_t j) {
        return to_f32(((const TGrad*)a.grad)[r * a.grad_stride + j]);
      },
      [&](int64_t i, int64_t j) {
        const uint8_t* row = a.q + j * a.q_stride;
        return (float)(int8_t)row[i] * *(const float*)(row + end);
      },
      [&](int64_t r, int64_t i, double v) {
        ((TOut*)a.out)[r * a.out_stride + i] = from_f32<TOut>((float)v);
      });
}

template <typename TOut, int kRows>
cudaError_t launch_few(const LinearArgs& a, int device, cudaStream_t st) {
  int lanes = 1;
  while (lanes < 32 && lanes < (a.dim + 15) / 16) lanes *= 2;
  const int64_t ctas = ceil_div(a.width, kFewThreads / lanes * kFewCols);
  const int64_t most = 8 * (int64_t)op_num_sms(device);
  linear_few_kernel<TOut, kRows>
      <<<(unsigned)(ctas < most ? ctas : most), kFewThreads, 0, st>>>(lanes, a);
  return cudaGetLastError();
}

agnes_status check_sizes(const char* op, int64_t rows, int64_t width, int64_t dim) {
  if (rows < 0 || width < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, width %lld, dim %lld", op, (long long)rows,
                    (long long)width, (long long)dim);
  if (rows > kInt8MaxRows || width > kInt8MaxRows || dim > kInt8MaxDim)
    return op_error(AGNES_ERANGE, "%s: rows %lld, width %lld, dim %lld are too large", op,
                    (long long)rows, (long long)width, (long long)dim);
  return AGNES_OK;
}

agnes_status check_step(const char* op, const char* name, int64_t rows, int64_t cols,
                        int64_t stride) {
  if (rows > 1 && stride < cols)
    return op_error(AGNES_EINVAL, "%s: a stride of %lld of %s is below %lld", op, (long long)stride,
                    name, (long long)cols);
  return AGNES_OK;
}

agnes_status check_workspace(const char* op, const void* p, int64_t bytes, int64_t need,
                             int device) {
  if (need == 0) return AGNES_OK;
  OP_TRY(op_on_device(op, "workspace", p, device));
  OP_TRY(op_aligned(op, "workspace", p, 256));
  if (bytes < need)
    return op_error(AGNES_EINVAL, "%s: a workspace of %lld bytes, %lld are needed", op,
                    (long long)bytes, (long long)need);
  return AGNES_OK;
}

int64_t linear_workspace(int64_t, int64_t, int64_t) { return 0; }
int64_t grad_weight_workspace(int64_t, int64_t, int64_t, int32_t) { return 0; }
int64_t grad_input_workspace(int64_t, int64_t, int64_t, int32_t) { return 0; }

dim3 tile_grid(int64_t m, int64_t n) {
  return dim3((unsigned)ceil_div(m, kTile), (unsigned)ceil_div(n, kTile));
}

}  // namespace

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_int8_linear_workspace(int64_t rows, int64_t width, int64_t dim,
                                         int64_t* bytes) {
  const char* op = "agnes_int8_linear_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_sizes(op, rows, width, dim));
  *bytes = linear_workspace(rows, width, dim);
  return AGNES_OK;
}

agnes_status agnes_int8_linear(const void* x, int64_t x_stride, int64_t rows, const void* w,
                               int64_t w_stride, int64_t width, int64_t dim, const float* bias,
                               void* out, int32_t out_dtype, int64_t out_stride, void* workspace,
                               int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  const char* op = "agnes_int8_linear";
  OP_TRY(check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(int8_check_stride(op, "x", rows, dim, x_stride));
  OP_TRY(int8_check_stride(op, "w", width, dim, w_stride));
  OP_TRY(check_step(op, "out", rows, width, out_stride));
  if (rows == 0 || width == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "x", x, &device));
  OP_TRY(op_on_device(op, "w", w, device));
  OP_TRY(op_on_device(op, "out", out, device));
  OP_TRY(op_aligned(op, "x", x, 16));
  OP_TRY(op_aligned(op, "w", w, 16));
  OP_TRY(op_aligned(op, "out", out, float_size(out_dtype)));
  if (bias) {
    OP_TRY(op_on_device(op, "bias", bias, device));
    OP_TRY(op_aligned(op, "bias", bias, 4));
  }
  OP_TRY(op_status(op, status, device));
  OP_TRY(check_workspace(op, workspace, workspace_bytes, linear_workspace(rows, width, dim),
                         device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  LinearArgs a = {};
  a.rows = rows;
  a.width = width;
  a.dim = (int32_t)dim;
  a.row_bytes = (int32_t)int8_row_bytes(dim);
  a.bias = bias;
  a.out = out;
  a.x = (const uint8_t*)x;
  a.w = (const uint8_t*)w;
  // a single row has no next one: any stride will do
  a.x_stride = rows > 1 ? x_stride : a.row_bytes;
  a.w_stride = width > 1 ? w_stride : a.row_bytes;
  a.out_stride = rows > 1 ? out_stride : width;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return op_launched(op, with_float_type(out_dtype, [&](auto t) {
    using TOut = typename decltype(t)::type;
    if (rows == 1) return launch_few<TOut, 1>(a, device, st);
    if (rows == 2) return launch_few<TOut, 2>(a, device, st);
    if (rows <= 4) return launch_few<TOut, 4>(a, device, st);
    if (rows <= AGNES_INT8_FEW_ROWS) return launch_few<TOut, 8>(a, device, st);
    linear_kernel<TOut><<<tile_grid(rows, width), 256, 0, st>>>(a);
    return cudaGetLastError();
  }));
}

agnes_status agnes_int8_linear_grad_weight_workspace(int64_t rows, int64_t width, int64_t dim,
                                                     int32_t grad_dtype, int64_t* bytes) {
  const char* op = "agnes_int8_linear_grad_weight_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  *bytes = grad_weight_workspace(rows, width, dim, grad_dtype);
  return AGNES_OK;
}

agnes_status agnes_int8_linear_grad_weight(const void* grad, int32_t grad_dtype,
                                           int64_t grad_stride, int64_t rows, int64_t width,
                                           const void* x, int64_t x_stride, int64_t dim, void* out,
                                           int32_t out_dtype, int64_t out_stride, float* dbias,
                                           void* workspace, int64_t workspace_bytes,
                                           int32_t* status, void* cuda_stream) {
  const char* op = "agnes_int8_linear_grad_weight";
  OP_TRY(check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(check_step(op, "grad", rows, width, grad_stride));
  OP_TRY(int8_check_stride(op, "x", rows, dim, x_stride));
  OP_TRY(check_step(op, "out", width, dim, out_stride));
  if (width == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "out", out, &device));
  OP_TRY(op_aligned(op, "out", out, float_size(out_dtype)));
  if (dbias) {
    OP_TRY(op_on_device(op, "dbias", dbias, device));
    OP_TRY(op_aligned(op, "dbias", dbias, 4));
  }
  if (rows > 0) {
    OP_TRY(op_on_device(op, "grad", grad, device));
    OP_TRY(op_on_device(op, "x", x, device));
    OP_TRY(op_aligned(op, "grad", grad, float_size(grad_dtype)));
    OP_TRY(op_aligned(op, "x", x, 16));
  }
  OP_TRY(op_status(op, status, device));
  OP_TRY(check_workspace(op, workspace, workspace_bytes,
                         grad_weight_workspace(rows, width, dim, grad_dtype), device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  GradArgs a = {};
  a.grad = grad;
  a.rows = rows;
  a.width = width;
  a.q = (const uint8_t*)x;
  a.dim = (int32_t)dim;
  a.row_bytes = (int32_t)int8_row_bytes(dim);
  a.out = out;
  a.dbias = dbias;
  a.grad_stride = rows > 1 ? grad_stride : width;
  a.q_stride = rows > 1 ? x_stride : a.row_bytes;
  a.out_stride = width > 1 ? out_stride : dim;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return op_launched(op, with_float_type(grad_dtype, [&](auto t) {
    using TGrad = typename decltype(t)::type;
    if (dbias) grad_bias_kernel<TGrad><<<(unsigned)ceil_div(width, 256), 256, 0, st>>>(a);
    return with_float_type(out_dtype, [&](auto o) {
      using TOut = typename decltype(o)::type;
      grad_weight_kernel<TGrad, TOut><<<tile_grid(width, dim), 256, 0, st>>>(a);
      return cudaGetLastError();
    });
  }));
}

agnes_status agnes_int8_linear_grad_input_workspace(int64_t rows, int64_t width, int64_t dim,
                                                    int32_t grad_dtype, int64_t* bytes) {
  const char* op = "agnes_int8_linear_grad_input_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  *bytes = grad_input_workspace(rows, width, dim, grad_dtype);
  return AGNES_OK;
}

agnes_status agnes_int8_linear_grad_input(const void* grad, int32_t grad_dtype,
                                          int64_t grad_stride, int64_t rows, int64_t width,
                                          const void* w, int64_t w_stride, int64_t dim, void* out,
                                          int32_t out_dtype, int64_t out_stride, void* workspace,
                                          int64_t workspace_bytes, int32_t* status,
                                          void* cuda_stream) {
  const char* op = "agnes_int8_linear_grad_input";
  OP_TRY(check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(check_step(op, "grad", rows, width, grad_stride));
  OP_TRY(int8_check_stride(op, "w", width, dim, w_stride));
  OP_TRY(check_step(op, "out", rows, dim, out_stride));
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "out", out, &device));
  OP_TRY(op_aligned(op, "out", out, float_size(out_dtype)));
  if (width > 0) {
    OP_TRY(op_on_device(op, "grad", grad, device));
    OP_TRY(op_on_device(op, "w", w, device));
    OP_TRY(op_aligned(op, "grad", grad, float_size(grad_dtype)));
    OP_TRY(op_aligned(op, "w", w, 16));
  }
  OP_TRY(op_status(op, status, device));
  OP_TRY(check_workspace(op, workspace, workspace_bytes,
                         grad_input_workspace(rows, width, dim, grad_dtype), device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  GradArgs a = {};
  a.grad = grad;
  a.rows = rows;
  a.width = width;
  a.q = (const uint8_t*)w;
  a.dim = (int32_t)dim;
  a.row_bytes = (int32_t)int8_row_bytes(dim);
  a.out = out;
  a.grad_stride = rows > 1 ? grad_stride : width;
  a.q_stride = width > 1 ? w_stride : a.row_bytes;
  a.out_stride = rows > 1 ? out_stride : dim;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return op_launched(op, with_float_type(grad_dtype, [&](auto t) {
    using TGrad = typename decltype(t)::type;
    return with_float_type(out_dtype, [&](auto o) {
      using TOut = typename decltype(o)::type;
      grad_input_kernel<TGrad, TOut><<<tile_grid(rows, dim), 256, 0, st>>>(a);
      return cudaGetLastError();
    });
  }));
}

}  // extern "C"
