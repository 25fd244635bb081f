// ops_common.cuh -- what the operators of include/agnes_ops.h share: element
// types, vectors of elements, and the host's checks of arguments.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/agnes_ops.h"
#include "common.cuh"
#include "internal.h"

namespace agnes {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

// One rounding, to nearest even.
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) {
  return __float2half_rn(x);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}

// N elements that are loaded and stored as one access of N * sizeof(T) bytes.
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// A block of kFlat consecutive items of rows of `per_row` items each, row after
// row: where an item is.  Items are numbered from the block's first.
constexpr int kFlat = 1024;
struct FlatRows {
  int64_t row0;
  uint32_t col0, per_row, inv;

  // inv = ceil(2^32 / per_row), from the host (flat_inverse)
  __device__ FlatRows(int64_t block, int32_t per_row_, uint32_t inv_)
      : per_row((uint32_t)per_row_), inv(inv_) {
    const int64_t first = block * kFlat;
    row0 = first / per_row_;
    col0 = (uint32_t)(first - row0 * per_row_);
  }
  __device__ void at(uint32_t item, int64_t* row, uint32_t* col) const {
    const uint32_t q = col0 + item;  // < per_row + kFlat
    uint32_t r;
    if (per_row == 1)
      r = q;
    else if (per_row < kFlat)
      r = __umulhi(q, inv);  // q / per_row: exact, as q * per_row < 2^32
    else
      r = q >= per_row;
    *row = row0 + r;
    *col = q - r * per_row;
  }
};
// A CTA's share of a contiguous matrix taken as one run of elements: kFlatRun of them
// from element block * kFlatRun on; where element `first` + i of it is.
constexpr int kFlatRun = 8192;
struct FlatRun {
  int64_t row0;
  uint32_t col0, dim, inv;

  __device__ FlatRun(int64_t block, int32_t dim_, uint32_t inv_) : dim((uint32_t)dim_), inv(inv_) {
    const int64_t first = block * kFlatRun;
    row0 = first / dim_;
    col0 = (uint32_t)(first - row0 * dim_);
  }
  __device__ void at(uint32_t i, int64_t* row, uint32_t* col) const {
    const uint32_t q = col0 + i;  // < dim + kFlatRun
    // q / dim: exact, as q * dim < 2^32 where dim < kFlatRun
    const uint32_t r = dim == 1 ? q : dim < kFlatRun ? __umulhi(q, inv) : q >= dim;
    *row = row0 + r;
    *col = q - r * dim;
  }
};
inline uint32_t flat_inverse(int64_t per_row) {
  return (uint32_t)(((1ull << 32) + (uint64_t)per_row - 1) / (uint64_t)per_row);
}

// One of an operator's float types, as a type.
template <typename T>
struct TypeTag {
  using type = T;
};

// f(TypeTag<T>) for the type of an agnes_dtype code that has been checked.
template <typename F>
cudaError_t with_float_type(int32_t dtype, F&& f) {
  switch (dtype) {
    case AGNES_F32: return f(TypeTag<float>());
    case AGNES_F16: return f(TypeTag<__half>());
    default: return f(TypeTag<__nv_bfloat16>());
  }
}

template <typename F>
cudaError_t with_index_type(int32_t bits, F&& f) {
  return bits == 32 ? f(TypeTag<int32_t>()) : f(TypeTag<int64_t>());
}

inline bool is_float_type(int32_t dtype) {
  return dtype == AGNES_F32 || dtype == AGNES_F16 || dtype == AGNES_BF16;
}

inline int64_t float_size(int32_t dtype) { return dtype == AGNES_F32 ? 4 : 2; }

// Whether p and every stride bytes after it are multiples of `bytes`.
inline bool aligned_rows(const void* p, int64_t stride_bytes, int64_t bytes) {
  return (uintptr_t)p % (uintptr_t)bytes == 0 && stride_bytes % bytes == 0;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Launches a kernel in clusters of `cluster` CTAs, after its predecessor on the stream or `ahead` of
// that one's completion.
template <typename... Params, typename... Args>
cudaError_t launch_cluster(bool ahead, void (*kernel)(Params...), dim3 grid, unsigned threads,
                           size_t smem, unsigned cluster, cudaStream_t st, Args&&... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = cluster > 1 ? attr : attr + 1;
  cfg.numAttrs = (cluster > 1 ? 1 : 0) + (ahead ? 1 : 0);
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
// Launches a kernel whose predecessor on the stream is the kernel before it in the same
// call, ahead of that one's completion: its CTAs are set up meanwhile and wait in
// grid_dep_wait(), which has to be the kernel's first statement.
template <typename... Params, typename... Args>
cudaError_t launch_next_cluster(void (*kernel)(Params...), dim3 grid, unsigned threads,
                                size_t smem, unsigned cluster, cudaStream_t st, Args&&... args) {
  return launch_cluster(true, kernel, grid, threads, smem, cluster, st, args...);
}
template <typename... Params, typename... Args>
cudaError_t launch_next(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem,
                        cudaStream_t st, Args&&... args) {
  return launch_next_cluster(kernel, grid, threads, smem, 1, st, args...);
}

// Lets the next kernel's CTAs be set up from here on.
__device__ __forceinline__ void let_next_start() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// ---- argument checks (ops.cu); each records a message for
// agnes_last_error(NULL) when it fails ----------------------------------------

agnes_status op_error(agnes_status s, const char* fmt, ...);

// `p` is memory that the current or some other device can address as its own;
// *device receives which.
agnes_status op_device_of(const char* op, const char* name, const void* p, int* device);
// `p` lies in the memory of `device`.
agnes_status op_on_device(const char* op, const char* name, const void* p, int device);
agnes_status op_float_type(const char* op, const char* name, int32_t dtype);
agnes_status op_index_bits(const char* op, const char* name, int32_t bits);
// `p` is aligned to one element of `size` bytes.
agnes_status op_aligned(const char* op, const char* name, const void* p, int64_t size);
// The caller's status word, if there is one: on `device`, and aligned for an atomic.
agnes_status op_status(const char* op, const int32_t* status, int device);
// The launch's error, as a status.
agnes_status op_launched(const char* op, cudaError_t e);
// A stride in bytes between 4-bit rows of dim values (mx4.cu).
agnes_status mx4_check_stride(const char* op, const char* name, int64_t rows, int64_t dim,
                              int64_t stride);
// Multiprocessors of `device` (looked up once for each device).
int op_num_sms(int device);

// What a kernel needs set once on each device (its shared-memory limit) before its
// first launch there.
class OncePerDevice {
 public:
  template <typename F>
  cudaError_t run(int device, F&& f) {
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done_.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    const cudaError_t e = f();
    if (e == cudaSuccess && device < 64) done_.fetch_or(bit, std::memory_order_release);
    return e;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

#define OP_TRY(call)                          \
  do {                                        \
    const agnes_status op_s_ = (call);        \
    if (op_s_ != AGNES_OK) return op_s_;      \
  } while (0)

// Sets bits of the caller's status word, where there is one.
__device__ __forceinline__ void op_flag(int32_t* status, int32_t bits) {
  if (status) atomicOr(status, bits);
}

}  // namespace agnes
