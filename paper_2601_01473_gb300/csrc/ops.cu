// ops.cu -- the checks of arguments that the operators of include/agnes_ops.h
// share.
#include "ops_common.cuh"

#include <stdarg.h>
#include <stdio.h>

#include <atomic>

namespace agnes {

agnes_status op_error(agnes_status s, const char* fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  ctx_set_error(nullptr, "%s", text);
  return s;
}

agnes_status op_device_of(const char* op, const char* name, const void* p, int* device) {
  if (!p) return op_error(AGNES_EINVAL, "%s: %s is NULL", op, name);
  cudaPointerAttributes attr;
  const cudaError_t e = cudaPointerGetAttributes(&attr, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return op_error(AGNES_ECUDA, "%s: %s: %s", op, name, cudaGetErrorString(e));
  }
  if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged)
    return op_error(AGNES_EINVAL, "%s: %s is not device memory", op, name);
  *device = attr.device;
  return AGNES_OK;
}

agnes_status op_on_device(const char* op, const char* name, const void* p, int device) {
  int d = -1;
  OP_TRY(op_device_of(op, name, p, &d));
  if (d != device)
    return op_error(AGNES_EINVAL, "%s: %s is on device %d, the other arguments on %d", op, name, d,
                    device);
  return AGNES_OK;
}

agnes_status op_float_type(const char* op, const char* name, int32_t dtype) {
  if (!is_float_type(dtype))
    return op_error(AGNES_EINVAL, "%s: %s has an unknown type (%d)", op, name, dtype);
  return AGNES_OK;
}

agnes_status op_index_bits(const char* op, const char* name, int32_t bits) {
  if (bits != 32 && bits != 64)
    return op_error(AGNES_EINVAL, "%s: %s has %d bits, not 32 or 64", op, name, bits);
  return AGNES_OK;
}

agnes_status op_aligned(const char* op, const char* name, const void* p, int64_t size) {
  if ((uintptr_t)p % (uintptr_t)size)
    return op_error(AGNES_EINVAL, "%s: %s is not aligned to %lld bytes", op, name,
                    (long long)size);
  return AGNES_OK;
}

agnes_status op_status(const char* op, const int32_t* status, int device) {
  if (!status) return AGNES_OK;
  OP_TRY(op_on_device(op, "status", status, device));
  return op_aligned(op, "status", status, 4);
}

agnes_status op_launched(const char* op, cudaError_t e) {
  if (e == cudaSuccess) return AGNES_OK;
  return op_error(e == cudaErrorMemoryAllocation ? AGNES_ENOMEM : AGNES_ECUDA, "%s: %s", op,
                  cudaGetErrorString(e));
}

int op_num_sms(int device) {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  if (device >= 0 && device < kDevices) {
    const int n = known[device].load(std::memory_order_relaxed);
    if (n > 0) return n;
  }
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 1;
  }
  if (device >= 0 && device < kDevices) known[device].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace agnes
