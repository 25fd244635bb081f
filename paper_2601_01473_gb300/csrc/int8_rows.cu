// int8_rows.cu -- rows to 8 bits and back, and nonlinearities whose input is kept in 8
// bits for their backward pass (include/agnes_ops.h; the format is in int8.cuh).
//
// Bound by memory: a group of threads holds a row in registers, so it is read once, for
// its largest magnitude, its whole numbers and its nonlinearity; rows of more than 8192
// values are read again, from L2 as far as it holds them.
// 2M x 128 fp16 to 8 bits 145 us and back 124; gated silu of 65,536 x 1024 bfloat16 99 us kept
// in 8 bits and 86 back, 4.9 and 5.7 TB/s.  Rows that no vector divides are bound by instructions on
// single elements; gated ones to 8 bits spill 152 bytes a thread besides.
#include "int8.cuh"

namespace agnes {

namespace {

constexpr int kElems = 16;   // values of a row to a thread at a time
constexpr int kLanes = 512;  // threads to a row at most
constexpr int kBackLanes = 256;

struct KeepArgs {
  const void* x;
  int64_t stride, rows;
  int32_t dim;       // of a half where gated
  int32_t lanes, log_lanes, groups;
  int32_t f;         // AGNES_F_*
  void* out;
  int64_t out_stride;
  uint8_t* kept;     // may be null
  int64_t kept_stride;
  int32_t batches;              // of `groups` rows, to a CTA; one but where they are staged
  int32_t in_bytes, out_bytes;  // of the shared memory for what a CTA reads and writes
};

// The normal distribution function and its density at v, for results of 16 bits:
// Phi(-a) = exp(-a^2 / 2) t Q(t), t = 1 / (1 + 0.21 a), with Q of degree 8 fitted to the
// scaled complementary error function over 0 <= a <= 14, to 2^-24.6 of it (2^-26 of one).  The square's
// own rounding is put back into the exponential.  (normcdff and a second exponential: gelu of
// 131,072 x 1024 bf16 278 us forward and 537 backward.)
__device__ __forceinline__ void normal_fit(float v, float* phi, float* density) {
  const float a = fminf(fabsf(v), 16.f);
  const float t = __fdividef(1.f, fmaf(0.21f, a, 1.f));
  float q = -0.07165663f;
  q = fmaf(q, t, 0.28359011f);
  q = fmaf(q, t, -0.33025661f);
  q = fmaf(q, t, 0.34940478f);
  q = fmaf(q, t, -0.09392789f);
  q = fmaf(q, t, 0.12487392f);
  q = fmaf(q, t, 0.06919184f);
  q = fmaf(q, t, 0.0850689f);
  q = fmaf(q, t, 0.08371157f);
  const float square = a * a, rest = fmaf(a, a, -square);
  float e = __expf(-0.5f * square);
  e = fmaf(e, -0.5f * rest, e);
  const float tail = e * t * q;
  *phi = v < 0.f ? tail : 1.f - tail;
  *density = e * 0.3989422804f;  // 1 / sqrt(2 pi)
}

// silu by 1 / (1 + exp -v), which leaves fp32's range below kSiluNear: the result is zero there and
// not v exp v, 1e-36 and less, which fp16 and 8-bit rows have as zero anyway.
constexpr int32_t kNearSilu = 3;
constexpr float kSiluNear = -87.f;

// f(v), and its derivative where one is asked for; kFit: for results of 16 bits.
template <bool kSlope, bool kFit>
__device__ __forceinline__ float nonlinear(int32_t f, float v, float* slope) {
  if (f == AGNES_F_RELU) {
    if (kSlope) *slope = v > 0.f ? 1.f : v <= 0.f ? 0.f : v;
    return v < 0.f ? 0.f : v;
  }
  if (f == kNearSilu) {
    const float p = __fdividef(1.f, 1.f + (kFit ? __expf(-v) : expf(-v)));
    if (kSlope) *slope = p * fmaf(v, 1.f - p, 1.f);
    return v * p;
  }
  if (f == AGNES_F_SILU) {
    // p = 1 / (1 + exp -v) from exp -|v|, which stays in fp32's range, so v p does far below zero;
    // the slope p + v p (1 - p) by the product of both, as 1 - p would be a difference
    const float e = kFit ? __expf(-fabsf(v)) : expf(-fabsf(v));
    const float r = __fdividef(1.f, 1.f + e);
    const float up = v < 0.f ? e : 1.f;
    if constexpr (kSlope) {
      const float p = up * r;
      *slope = fmaf(v, e * r * r, p);
      return v * p;
    }
    return v * up * r;
  }
  float p, density;
  if constexpr (kFit) {
    normal_fit(v, &p, &density);
  } else {
    p = normcdff(v);
    if (kSlope) density = expf(-0.5f * v * v) * 0.3989422804f;
  }
  if (kSlope) *slope = fmaf(v, density, p);
  return v * p;
}

// f with the kind as a constant, chosen once for all of a thread's values.
// kNear: kNearSilu may be among them.
template <bool kNear, typename F>
__device__ __forceinline__ void with_kind(int32_t kind, F&& f) {
  if (kind == AGNES_F_RELU)
    f(std::integral_constant<int32_t, AGNES_F_RELU>());
  else if (kind == AGNES_F_SILU)
    f(std::integral_constant<int32_t, AGNES_F_SILU>());
  else if (kNear && kind == kNearSilu)
    f(std::integral_constant<int32_t, kNearSilu>());
  else
    f(std::integral_constant<int32_t, AGNES_F_GELU>());
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// What is made of a row: 8-bit rows alone, a nonlinearity, or a gated one.
enum { kRound, kPlain, kGated };

// kVec = 1: single elements, and without kLoop from and to shared memory (stage_in), where the
// matrices are contiguous.
template <typename T, int kMode, bool kOut8, int kVec, bool kLoop, bool kStaged>
__global__ void __launch_bounds__(kLanes, kVec == 1 && !kStaged ? 1 : 2)
keep_kernel(const KeepArgs a) {
  constexpr int kPer = kElems / kVec;
  constexpr bool kFit = sizeof(T) == 2;
  // 16-bit silu by the shorter form (65,536 x 1024 bf16, gated, 102 us and not 106): where small
  // results are zeros, or a thread's values are all nearer (their largest magnitude is known)
  constexpr bool kNear = kFit && (kOut8 || std::is_same<T, __half>::value), kAsk = kFit && !kNear;
  __shared__ RowScratch scratch;
  int turn = 0;
  const int group = threadIdx.x >> a.log_lanes, lane = threadIdx.x & (a.lanes - 1);
  const int32_t chunk = a.lanes * kElems;
  const bool keep = kMode == kRound || a.kept;
  // a CTA's rows: what it reads, its values and what it keeps
  extern __shared__ uint4 staged[];
  uint8_t* const in_stage = (uint8_t*)staged;
  uint8_t* const out_stage = in_stage + a.in_bytes;
  uint8_t* const kept_stage = out_stage + a.out_bytes;
  const int64_t row0 = (int64_t)blockIdx.x * a.groups * a.batches, left = a.rows - row0;
  const int rows = (int)(left < a.groups * a.batches ? left : a.groups * a.batches);
  const T* const x0 = (const T*)a.x + row0 * a.stride;
  T* const out0 = (T*)a.out + row0 * a.out_stride;
  uint8_t* const out8_0 = (uint8_t*)a.out + row0 * a.out_stride;
  if constexpr (kStaged) {
    stage_in(in_stage, x0, rows * a.stride * (int64_t)sizeof(T), a.x,
             (const T*)a.x + a.rows * a.stride);
    stage_wait();
  }
  for (int batch = 0; batch < (kStaged ? a.batches : 1); ++batch) {
    const int r = batch * a.groups + group;
    const bool valid = r < rows;
    const T* x = kStaged ? (const T*)(in_stage + stage_offset(x0)) + r * a.stride
                         : x0 + r * a.stride;
    T* to = kStaged ? (T*)(out_stage + stage_offset(out0)) + r * a.out_stride
                    : out0 + r * a.out_stride;
    uint8_t* to8 = (kStaged ? out_stage : out8_0) + r * a.out_stride;
    uint8_t* kept = (kStaged ? kept_stage : a.kept + row0 * a.kept_stride) + r * a.kept_stride;
    RowRegs<T, kVec, kPer> v, u;
    float y[kOut8 ? kElems : 1];
    uint32_t top[3] = {0, 0, 0};
    // The values are made of the row once: those of a type that is stored as it is go out at
    // once, those that are rounded to 8 bits wait for their largest magnitude.
    for (int32_t c0 = 0; c0 < (kLoop ? a.dim : 1); c0 += chunk) {
      const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
      v.load(part, x + c0, valid);
      if constexpr (kMode == kGated) u.load(part, x + a.dim + c0, valid);
      const uint32_t largest = keep || kAsk ? v.top() : 0;
      if (keep) {
        top[0] = max(top[0], largest);
        if constexpr (kMode == kGated) top[1] = max(top[1], u.top());
      }
      if constexpr (kMode != kRound) {
        const bool near = kNear || (kAsk && largest < __float_as_uint(-kSiluNear));
        with_kind<kFit>(a.f == AGNES_F_SILU && near ? kNearSilu : a.f, [&](auto kind) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            if (part.beyond(i)) break;
            float f[kVec];
            v.get(i, f);
            [[maybe_unused]] float g[kVec];
            if constexpr (kMode == kGated) u.get(i, g);
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              f[e] = nonlinear<false, kFit>(kind, f[e], nullptr);
              if constexpr (kMode == kGated) f[e] *= g[e];
              if constexpr (kOut8) {
                y[i * kVec + e] = f[e];
                top[2] = max(top[2], magnitude(f[e]));
              }
            }
            if constexpr (!kOut8) part.store_one(to + c0, valid, i, f);
          }
        });
      }
    }
    if (!keep && !kOut8) continue;
    v.pin();
    if constexpr (kMode == kGated) u.pin();
    Int8Scale s = {}, s_gate = {}, s_out = {};
    if constexpr (kMode == kRound) {
      uint32_t one[1] = {top[0]};
      group_reduce<MaxBits>(one, a.lanes, &scratch, turn);
      s = int8_scale(one[0]);
    } else {
      group_reduce<MaxBits>(top, a.lanes, &scratch, turn);
      s = int8_scale(top[0]);
      if constexpr (kMode == kGated) s_gate = int8_scale(top[1]);
      if constexpr (kOut8) s_out = int8_scale(top[2]);
    }
    const int64_t half = int8_row_bytes(a.dim);
    for (int32_t c0 = 0; c0 < (kLoop ? a.dim : 1); c0 += chunk) {
      const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
      if (kLoop) {
        v.load(part, x + c0, valid);
        if constexpr (kMode == kGated) u.load(part, x + a.dim + c0, valid);
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (part.beyond(i)) break;
        float f[kVec];
        v.get(i, f);
        [[maybe_unused]] float g[kVec];
        if constexpr (kMode == kGated) u.get(i, g);
        if (keep) {
          int8_store(part, kept + c0, valid, i, f, s);
          if constexpr (kMode == kGated) int8_store(part, kept + half + c0, valid, i, g, s_gate);
        }
        if constexpr (kOut8) {
          if (kLoop) {
            with_kind<kNear>(kNear && a.f == AGNES_F_SILU ? kNearSilu : a.f, [&](auto kind) {
#pragma unroll
              for (int e = 0; e < kVec; ++e) {
                f[e] = nonlinear<false, kFit>(kind, f[e], nullptr);
                if constexpr (kMode == kGated) f[e] *= g[e];
              }
            });
            int8_store(part, to8 + c0, valid, i, f, s_out);
          } else {
            int8_store(part, to8, valid, i, y + i * kVec, s_out);
          }
        }
      }
    }
    if (keep) {
      int8_store_end(kept, a.dim, lane, a.lanes, valid, s);
      if constexpr (kMode == kGated)
        int8_store_end(kept + half, a.dim, lane, a.lanes, valid, s_gate);
    }
    if constexpr (kOut8) int8_store_end(to8, a.dim, lane, a.lanes, valid, s_out);
  }
  if constexpr (kStaged) {
    __syncthreads();
    if (kMode != kRound && kOut8)
      stage_out(out_stage, out8_0, rows * a.out_stride);
    else if (kMode != kRound)
      stage_out(out_stage, out0, rows * a.out_stride * (int64_t)sizeof(T));
    if (keep) stage_out(kept_stage, a.kept + row0 * a.kept_stride, rows * a.kept_stride);
  }
}

struct BackArgs {
  const uint8_t* kept;
  int64_t kept_stride, rows;
  int32_t dim, lanes, log_lanes, groups;
  int32_t f;
  const void* grad;  // null: the kept values themselves
  int64_t grad_stride;
  void* out;
  int64_t out_stride;
  int32_t batches;                 // of `groups` rows, to a CTA; one but where they are staged
  int32_t kept_bytes, grad_bytes;  // of shared memory, where a CTA's rows are there
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

// A CTA's rows of the kept values, of the gradient and of the output in shared memory.
template <typename TGrad, typename T>
struct BackStage {
  const BackArgs& a;
  uint8_t* base;
  int64_t row0;
  int n;
  __device__ BackStage(const BackArgs& args, uint8_t* shared) : a(args), base(shared) {
    row0 = (int64_t)blockIdx.x * a.groups * a.batches;
    const int64_t left = a.rows - row0;
    n = (int)(left < a.groups * a.batches ? left : a.groups * a.batches);
  }
  __device__ uint8_t* kept() const { return base; }
  __device__ uint8_t* grad_base() const { return base + a.kept_bytes; }
  __device__ uint8_t* out_base() const { return grad_base() + a.grad_bytes; }
  __device__ const TGrad* grad_from() const { return (const TGrad*)a.grad + row0 * a.grad_stride; }
  __device__ T* out_to() const { return (T*)a.out + row0 * a.out_stride; }
  __device__ void load(bool with_grad) const {
    stage_in(kept(), a.kept + row0 * a.kept_stride, n * a.kept_stride, a.kept,
             a.kept + a.rows * a.kept_stride);
    if (with_grad)
      stage_in(grad_base(), grad_from(), n * a.grad_stride * (int64_t)sizeof(TGrad), a.grad,
               (const TGrad*)a.grad + a.rows * a.grad_stride);
    stage_wait();
  }
  __device__ const TGrad* grad() const {
    return (const TGrad*)(grad_base() + stage_offset(grad_from()));
  }
  __device__ T* out() const { return (T*)(out_base() + stage_offset(out_to())); }
  __device__ void store() const {
    __syncthreads();
    stage_out(out_base(), out_to(), n * a.out_stride * (int64_t)sizeof(T));
  }
};

// What 8-bit rows stand for.  kStaged: single elements (kVec = 1) through shared memory.
template <typename T, int kVec, bool kStaged>
__global__ void __launch_bounds__(kBackLanes, kVec == 1 ? 4 : 8)
values_kernel(const BackArgs a) {
  constexpr int kPer = kElems / kVec;
  extern __shared__ uint4 staged[];
  const int group = threadIdx.x >> a.log_lanes, lane = threadIdx.x & (a.lanes - 1);
  const BackStage<T, T> stage(a, (uint8_t*)staged);
  if constexpr (kStaged) stage.load(false);
  for (int batch = 0; batch < (kStaged ? a.batches : 1); ++batch) {
    const int r = batch * a.groups + group;
    if (r >= stage.n) break;
    const uint8_t* kept =
        kStaged ? stage.kept() + r * a.kept_stride : a.kept + (stage.row0 + r) * a.kept_stride;
    T* out = kStaged ? stage.out() + r * a.out_stride : stage.out_to() + r * a.out_stride;
    const float scale = *(const float*)(kept + int8_row_bytes(a.dim) - 4);
    for (int32_t c0 = 0; c0 < a.dim; c0 += a.lanes * kElems) {
      const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
      Int8Regs<kVec, kPer> v;
      v.load(part, kept + c0, true);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (part.beyond(i)) break;
        float f[kVec];
        v.get(i, f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float most = most_of<T>(), y = f[e] * scale;
          f[e] = y > most ? most : y < -most ? -most : y;
        }
        part.store_one(out + c0, true, i, f);
      }
    }
  }
  if constexpr (kStaged) stage.store();
}

// The nonlinearity's gradient at them.
template <typename TGrad, typename T, bool kGate, int kVec, bool kStaged>
__global__ void __launch_bounds__(kBackLanes, kVec == 1 ? 2 : 4)
back_kernel(const BackArgs a) {
  constexpr int kPer = kElems / kVec;
  constexpr bool kFit = sizeof(T) == 2;
  extern __shared__ uint4 staged[];
  const int group = threadIdx.x >> a.log_lanes, lane = threadIdx.x & (a.lanes - 1);
  const BackStage<TGrad, T> stage(a, (uint8_t*)staged);
  if constexpr (kStaged) stage.load(true);
  for (int batch = 0; batch < (kStaged ? a.batches : 1); ++batch) {
    const int r = batch * a.groups + group;
    if (r >= stage.n) break;
    const uint8_t* kept =
        kStaged ? stage.kept() + r * a.kept_stride : a.kept + (stage.row0 + r) * a.kept_stride;
    T* out = kStaged ? stage.out() + r * a.out_stride : stage.out_to() + r * a.out_stride;
    const TGrad* grad = (kStaged ? stage.grad() : stage.grad_from()) + r * a.grad_stride;
    const int64_t half = int8_row_bytes(a.dim);
    const float s0 = *(const float*)(kept + half - 4);
    const float s1 = kGate ? *(const float*)(kept + 2 * half - 4) : 0.f;
    for (int32_t c0 = 0; c0 < a.dim; c0 += a.lanes * kElems) {
      const RowPart<kVec, kPer> part = {a.lanes, lane, a.dim - c0};
      Int8Regs<kVec, kPer> v, u;
      RowRegs<TGrad, kVec, kPer> d;
      v.load(part, kept + c0, true);
      if constexpr (kGate) u.load(part, kept + half + c0, true);
      d.load(part, grad + c0, true);
      with_kind<false>(a.f, [&](auto kind) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (part.beyond(i)) break;
          float f[kVec], h[kVec];
          v.get(i, f);
          d.get(i, h);
          [[maybe_unused]] float g[kVec];
          if constexpr (kGate) u.get(i, g);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            float slope;
            const float y = nonlinear<true, kFit>(kind, f[e] * s0, &slope);
            f[e] = h[e] * slope;
            if constexpr (kGate) {
              f[e] *= g[e] * s1;
              g[e] = h[e] * y;
            }
          }
          part.store_one(out + c0, true, i, f);
          if constexpr (kGate) part.store_one(out + a.dim + c0, true, i, g);
        }
      });
    }
  }
  if constexpr (kStaged) stage.store();
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

template <typename T, int kMode, bool kOut8>
cudaError_t launch_keep(KeepArgs a, int device, cudaStream_t st) {
  const int64_t next = a.rows > 1 ? 1 : 0;  // a single row has no next one
  const bool aligned =
      aligned_rows(a.x, next * a.stride * (int64_t)sizeof(T), 16) &&
      (kMode == kRound || kOut8 ||
       aligned_rows(a.out, next * a.out_stride * (int64_t)sizeof(T), 16));
  const RowShape shape = row_shape(a.dim, kElems, kLanes);
  a.lanes = shape.lanes;
  a.log_lanes = shape.log_lanes;
  a.groups = shape.groups;
  const bool loop = a.dim > a.lanes * kElems, wide = vec_of(a.dim, aligned) == 8;
  const int64_t cols = kMode == kGated ? 2 * (int64_t)a.dim : a.dim;
  const int64_t kept_row = int8_row_bytes(a.dim) * (kMode == kGated ? 2 : 1);
  const bool staged = !wide && !loop && (!next || a.stride == cols) &&
                      (kMode == kRound || !next ||
                       a.out_stride == (kOut8 ? int8_row_bytes(a.dim) : a.dim)) &&
                      (!a.kept || !next || a.kept_stride == kept_row);
  size_t smem = 0;
  a.batches = 1;
  if (staged) {
    if (!next) {
      a.stride = cols;
      a.out_stride = kOut8 ? int8_row_bytes(a.dim) : a.dim;
      a.kept_stride = kept_row;
    }
    const int64_t out_row =
        kMode == kRound ? 0 : a.out_stride * (kOut8 ? 1 : (int64_t)sizeof(T));
    const int64_t row = cols * (int64_t)sizeof(T) + out_row + (a.kept ? kept_row : 0);
    a.batches = stage_batches(a.rows, a.groups, row, op_num_sms(device));
    const int64_t rows = a.groups * (int64_t)a.batches;
    a.in_bytes = (int32_t)staged_bytes(rows * cols * (int64_t)sizeof(T));
    a.out_bytes = kMode == kRound ? 0 : (int32_t)staged_bytes(rows * out_row);
    smem = (size_t)a.in_bytes + a.out_bytes + (a.kept ? rows * kept_row : 0);
  }
  const auto kernel = wide     ? (loop ? keep_kernel<T, kMode, kOut8, 8, true, false>
                                       : keep_kernel<T, kMode, kOut8, 8, false, false>)
                      : staged ? keep_kernel<T, kMode, kOut8, 1, false, true>
                      : loop   ? keep_kernel<T, kMode, kOut8, 1, true, false>
                               : keep_kernel<T, kMode, kOut8, 1, false, false>;
  if (smem + sizeof(RowScratch) > 48 * 1024) {
    static OncePerDevice once;
    const cudaError_t e = once.run(device, [&] {
      return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
    });
    if (e != cudaSuccess) return e;
  }
  kernel<<<(unsigned)ceil_div(a.rows, a.groups * a.batches), shape.threads(), smem, st>>>(a);
  return cudaGetLastError();
}

// kernels[0] for vectors, [1] for single elements, [2] for those through shared memory
using BackKernel = void (*)(BackArgs);
cudaError_t launch_back(const BackKernel (&kernels)[3], BackArgs a, int halves, int64_t grad_size,
                        int64_t size, int device, cudaStream_t st) {
  const int64_t next = a.rows > 1 ? 1 : 0;
  const bool aligned = aligned_rows(a.out, next * a.out_stride * size, 16) &&
                       (!a.grad || aligned_rows(a.grad, next * a.grad_stride * grad_size, 16));
  const RowShape shape = row_shape(a.dim, kElems, kBackLanes);
  a.lanes = shape.lanes;
  a.log_lanes = shape.log_lanes;
  a.groups = shape.groups;
  const int64_t kept_row = halves * int8_row_bytes(a.dim);
  const bool staged = a.dim <= a.lanes * kElems &&
                      (!next || (a.kept_stride == kept_row && a.out_stride == halves * a.dim &&
                                 (!a.grad || a.grad_stride == a.dim)));
  const int which = vec_of(a.dim, aligned) == 8 ? 0 : staged ? 2 : 1;
  size_t smem = 0;
  a.batches = 1;
  if (which == 2) {
    a.kept_stride = kept_row;
    a.out_stride = halves * a.dim;
    a.grad_stride = a.dim;
    const int64_t out_row = halves * a.dim * size, grad_row = a.grad ? a.dim * grad_size : 0;
    a.batches = stage_batches(a.rows, a.groups, kept_row + out_row + grad_row, op_num_sms(device));
    const int64_t rows = a.groups * (int64_t)a.batches;
    a.kept_bytes = (int32_t)staged_bytes(rows * kept_row);
    a.grad_bytes = a.grad ? (int32_t)staged_bytes(rows * grad_row) : 0;
    smem = (size_t)a.kept_bytes + a.grad_bytes + staged_bytes(rows * out_row);
    if (smem > 48 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(
          kernels[which], cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024);
      if (e != cudaSuccess) return e;
    }
  }
  kernels[which]<<<(unsigned)ceil_div(a.rows, a.groups * a.batches), shape.threads(), smem, st>>>(a);
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
  a.kept = (uint8_t*)out;
  a.kept_stride = out_stride;
  return op_launched(op, with_float_type(dtype, [&](auto t) {
    return launch_keep<typename decltype(t)::type, kRound, false>(a, device, (cudaStream_t)cuda_stream);
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
    const BackKernel kernels[3] = {values_kernel<T, 8, false>, values_kernel<T, 1, false>,
                                   values_kernel<T, 1, true>};
    return launch_back(kernels, a, 1, 0, sizeof(T), device, (cudaStream_t)cuda_stream);
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
  a.out = out;
  a.out_stride = out_stride;
  a.kept = (uint8_t*)kept;
  a.kept_stride = kept_stride;
  return op_launched(op, with_float_type(dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (out_dtype == AGNES_INT8_ROWS)
      return gated ? launch_keep<T, kGated, true>(a, device, st) : launch_keep<T, kPlain, true>(a, device, st);
    return gated ? launch_keep<T, kGated, false>(a, device, st) : launch_keep<T, kPlain, false>(a, device, st);
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
  a.grad = grad;
  a.grad_stride = grad_stride;
  a.out = out;
  a.out_stride = out_stride;
  return op_launched(op, with_float_type(grad_dtype, [&](auto t) {
    using TGrad = typename decltype(t)::type;
    return with_float_type(out_dtype, [&](auto o) {
      using T = typename decltype(o)::type;
      const BackKernel kernels[2][3] = {
          {back_kernel<TGrad, T, false, 8, false>, back_kernel<TGrad, T, false, 1, false>,
           back_kernel<TGrad, T, false, 1, true>},
          {back_kernel<TGrad, T, true, 8, false>, back_kernel<TGrad, T, true, 1, false>,
           back_kernel<TGrad, T, true, 1, true>}};
      return launch_back(kernels[gated], a, halves, sizeof(TGrad), sizeof(T), device,
                         (cudaStream_t)cuda_stream);
    });
  }));
}

}  // extern "C"
