// distill.cu -- the loss of a student's logits against a teacher's top logits,
// and its gradient (include/agnes_ops.h).  Of a row x of logits, with the
// teacher's entries (index_k, t_k):
//
//   p = softmax(t / T)    q = softmax(x / T)    loss = T^2 sum_k p_k (ln p_k - ln q_{index_k})
//   d loss / d x_v = T (q_v sum_k p_k - sum_{k: index_k = v} p_k)
//
// One pass over the row keeps a running maximum M and sum S of exp((x - M) / T).
// A cluster of CTAs shares a row, each a slice of it, and joins (M, S) through
// distributed shared memory; a step that also wants the gradient keeps its slice
// in shared memory, so that the logits are read from memory once.  The gradient
// is written as if the teacher had no entry, and then the few entries' classes
// once more.
#include <cooperative_groups.h>

#include "ops_common.cuh"

namespace cg = cooperative_groups;

namespace agnes {

namespace {

constexpr int kMaxTop = AGNES_DISTILL_MAX_TOP;
constexpr int kMaxReaders = 512;
constexpr int kMaxThreads = kMaxReaders + 32;
constexpr int kMaxCluster = 8;
constexpr float kNegInf = -__builtin_huge_valf();

enum Mode { kLoss, kGrad, kStep };

struct DistillArgs {
  const void* logits;
  int64_t stride;
  int32_t classes;
  int32_t slice;  // classes per CTA, a multiple of 64
  const void* teacher;
  int32_t teacher_dtype;
  const void* index;
  int32_t index_bits;
  int32_t top;
  float temperature;
  float c;        // log2(e) / T
  float* loss;    // R
  float2* stats;  // R: (M, S); written by kLoss, read by kGrad
  const float* weight;  // R, or null: 1
  float weight_scale;
  void* out;
  int64_t out_stride;
  bool keep;  // the slice stays in shared memory
  int32_t* status;
};

__device__ __forceinline__ float load_teacher(const DistillArgs& a, int64_t i) {
  if (a.teacher_dtype == AGNES_F32) return __ldg((const float*)a.teacher + i);
  if (a.teacher_dtype == AGNES_F16) return __half2float(__ldg((const __half*)a.teacher + i));
  return __bfloat162float(__ldg((const __nv_bfloat16*)a.teacher + i));
}

__device__ __forceinline__ float exp2_fast(float x) {  // 2 ulp; 0 below 2^-126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A running maximum and the sum of 2^((x - max) c).
struct MaxSum {
  float m, s;
};

// x - m for m that may be -inf (then every x is): -inf, not NaN.
__device__ __forceinline__ float above(float m) { return m == kNegInf ? 0.f : m; }

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.m, b.m), z = above(m);
  return {m, a.s * exp2_fast((a.m - z) * c) + b.s * exp2_fast((b.m - z) * c)};
}

// The join over a warp's lanes: the largest maximum first, so that a lane's sum is
// scaled once.
__device__ __forceinline__ MaxSum warp_join(MaxSum x, float c) {
  float m = x.m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  return {m, warp_sum(x.s * exp2_fast((x.m - above(m)) * c))};
}

// Pairs of floats, for the packed instructions (each half rounded as by a single one).
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t p) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
  return f;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Two elements of a vector as a pair of floats.
__device__ __forceinline__ uint64_t pair_of(const float* v) { return pack2(v[0], v[1]); }
__device__ __forceinline__ uint64_t pair_of(const __half* v) {
  const float2 f = __half22float2(*(const __half2*)v);
  return pack2(f.x, f.y);
}
__device__ __forceinline__ uint64_t pair_of(const __nv_bfloat16* v) {
  const float2 f = __bfloat1622float2(*(const __nv_bfloat162*)v);
  return pack2(f.x, f.y);
}
__device__ __forceinline__ void put_pair(float* to, float2 f) {
  to[0] = f.x;
  to[1] = f.y;
}
__device__ __forceinline__ void put_pair(__half* to, float2 f) {
  *(__half2*)to = __float22half2_rn(f);
}
__device__ __forceinline__ void put_pair(__nv_bfloat16* to, float2 f) {
  *(__nv_bfloat162*)to = __float22bfloat162_rn(f);
}

// The largest of a vector's elements; a NaN is not looked at.
__device__ __forceinline__ float largest(const Vec<float, 4>& x) {
  return fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3]));
}
__device__ __forceinline__ float largest(const Vec<__half, 8>& x) {
  const __half2* h = (const __half2*)x.v;
  const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float largest(const Vec<__nv_bfloat16, 8>& x) {
  const __nv_bfloat162* h = (const __nv_bfloat162*)x.v;
  const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(__low2float(m), __high2float(m));
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
  return x;
}

// A thread's running maximum, and the sum as a pair.
struct Running {
  float m;
  uint64_t s;

  __device__ void raise(float top, float c) {  // a larger maximum
    if (top > m) {
      const float scale = exp2_fast((m - top) * c);
      s = mul2(s, pack2(scale, scale));
      m = top;
    }
  }
  template <typename T, int kN>
  __device__ void take(const Vec<T, kN>& x, float c) {
    raise(largest(x), c);
    const float z = -above(m);
    const uint64_t z2 = pack2(z, z), c2 = pack2(c, c);
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
      const float2 f = unpack2(mul2(add2(pair_of(x.v + e), z2), c2));
      s = add2(s, pack2(exp2_fast(f.x), exp2_fast(f.y)));
    }
  }
  __device__ void take_one(float f, float c) {
    raise(f, c);
    s = add2(s, pack2(exp2_fast((f - above(m)) * c), 0.f));
  }
  __device__ MaxSum sum() const {
    const float2 f = unpack2(s);
    return {m, f.x + f.y};
  }
};

struct alignas(16) DistillSmem {  // the kept slice follows it, in 16-byte vectors
  float p[kMaxTop];
  int32_t index[kMaxTop];  // -1: absent
  float x[kMaxTop];        // the student's logit at index
  MaxSum part[32];         // the readers' warps'
  MaxSum joined;           // this CTA's
  float mass;              // sum of p: 1, or 0 without a teacher entry
};
static_assert(sizeof(DistillSmem) % 16 == 0, "what follows is 16-byte aligned");

// A warp: the teacher's distribution of the row.
__device__ __forceinline__ void teacher_row(const DistillArgs& a, int64_t row, float c,
                                            DistillSmem& s) {
  const int lane = lane_id();
  float top = kNegInf;
  bool bad = false;
  for (int k = lane; k < a.top; k += 32) {
    const int64_t i = row * a.top + k;
    const int64_t v = a.index_bits == 32 ? (int64_t)__ldg((const int32_t*)a.index + i)
                                         : __ldg((const int64_t*)a.index + i);
    const bool in = v >= 0 && v < a.classes;
    bad |= v >= a.classes;
    s.index[k] = in ? (int32_t)v : -1;
    const float t = in ? load_teacher(a, i) : kNegInf;
    s.p[k] = t;
    top = fmaxf(top, t);
  }
  if (bad) op_flag(a.status, AGNES_OP_BAD_INDEX);
  top = warp_max(top);
  const float z = above(top);
  float sum = 0.f;
  for (int k = lane; k < a.top; k += 32) {
    const float e = s.index[k] < 0 ? 0.f : exp2_fast((s.p[k] - z) * c);
    s.p[k] = e;
    sum += e;
  }
  sum = warp_sum(sum);
  // without an entry, or with -inf alone, there is nothing to divide by
  const bool some = !(sum == 0.f);
  const float inv = some ? 1.f / sum : 0.f;
  for (int k = lane; k < a.top; k += 32) s.p[k] *= inv;
  if (lane == 0) s.mass = some ? sum * inv : 0.f;
}

// A warp: the row's loss.
__device__ __forceinline__ float row_loss(const DistillArgs& a, const DistillSmem& s, MaxSum q) {
  const float inv_t = 1.f / a.temperature, log_s = logf(q.s);
  float sum = 0.f;
  for (int k = lane_id(); k < a.top; k += 32) {
    const float p = s.p[k];
    if (p != 0.f && s.index[k] >= 0)
      sum += p * (logf(p) - ((s.x[k] - q.m) * inv_t - log_s));
  }
  return warp_sum(sum) * a.temperature * a.temperature;
}

// The vectors of a slice: `head` elements up to the first 16-byte boundary, then
// `body` whole vectors, then the rest.
template <typename T>
struct Cut {
  static constexpr int kN = 16 / sizeof(T);
  int32_t shift;  // of the slice's first element past a 16-byte boundary, in elements
  int32_t head, body, n;
  __device__ Cut(const T* p, int32_t count) : n(count) {
    shift = (int32_t)(((uintptr_t)p / sizeof(T)) % kN);
    head = min(n, (kN - shift) % kN);
    body = (n - head) / kN;
  }
  __device__ int32_t tail0() const { return head + body * kN; }
};

template <typename T>
__device__ __forceinline__ MaxSum read_slice(const T* x, const Cut<T>& cut, T* kept,
                                             bool keep, int tid, int threads, float c) {
  constexpr int kN = Cut<T>::kN, kAhead = 4;
  Running r = {kNegInf, pack2(0.f, 0.f)};
  const Vec<T, kN>* body = (const Vec<T, kN>*)(x + cut.head);
  Vec<T, kN>* kept_body = (Vec<T, kN>*)(kept + cut.shift + cut.head);
  int32_t j = tid;
  for (; j + (kAhead - 1) * threads < cut.body; j += kAhead * threads) {
    Vec<T, kN> v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = body[j + u * threads];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (keep) kept_body[j + u * threads] = v[u];
      r.take(v[u], c);
    }
  }
  for (; j < cut.body; j += threads) {
    const Vec<T, kN> v = body[j];
    if (keep) kept_body[j] = v;
    r.take(v, c);
  }
  const auto one = [&](int32_t i) {
    const T v = x[i];
    if (keep) kept[cut.shift + i] = v;
    r.take_one(to_f32(v), c);
  };
  if (tid < cut.head) one(tid);
  if (tid < cut.n - cut.tail0()) one(cut.tail0() + tid);
  return r.sum();
}

// out = factor * 2^((x - m) c) for the slice, from shared memory or from x.
template <typename T, typename TOut>
__device__ __forceinline__ void write_slice(const T* x, const Cut<T>& cut, const T* kept, bool keep,
                                            TOut* out, float m, float factor, float c, bool zero) {
  constexpr int kN = Cut<T>::kN;
  constexpr int kOutBytes = kN * sizeof(TOut), kPart = kOutBytes > 16 ? 16 : kOutBytes;
  constexpr int kPartN = kPart / (int)sizeof(TOut);
  const int tid = threadIdx.x, threads = blockDim.x;
  const auto value = [&](T v) {
    return from_f32<TOut>(zero ? 0.f : factor * exp2_fast((to_f32(v) - m) * c));
  };
  if (zero || (uintptr_t)(out + cut.head) % kPart != 0) {
    for (int32_t i = tid; i < cut.n; i += threads)
      out[i] = value(keep ? kept[cut.shift + i] : x[i]);
    return;
  }
  const Vec<T, kN>* body =
      (const Vec<T, kN>*)(keep ? kept + cut.shift + cut.head : x + cut.head);
#pragma unroll 2
  for (int32_t j = tid; j < cut.body; j += threads) {
    const Vec<T, kN> v = body[j];
#pragma unroll
    for (int h = 0; h < kN / kPartN; ++h) {
      Vec<TOut, kPartN> y;
#pragma unroll
      for (int e = 0; e < kPartN; e += 2) {
        const float2 f =
            unpack2(mul2(add2(pair_of(v.v + h * kPartN + e), pack2(-m, -m)), pack2(c, c)));
        put_pair(y.v + e, unpack2(mul2(pack2(exp2_fast(f.x), exp2_fast(f.y)),
                                       pack2(factor, factor))));
      }
      *(Vec<TOut, kPartN>*)(out + cut.head + j * kN + h * kPartN) = y;
    }
  }
  const auto one = [&](int32_t i) { out[i] = value(keep ? kept[cut.shift + i] : x[i]); };
  if (tid < cut.head) one(tid);
  if (tid < cut.n - cut.tail0()) one(cut.tail0() + tid);
}

// grid: (CTAs per row, rows); kLoss and kStep: a row's CTAs are a cluster.
template <typename T, typename TOut, int kMode>
__global__ void __launch_bounds__(kMaxThreads) distill_kernel(DistillArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  DistillSmem& s = *(DistillSmem*)smem;
  T* kept = (T*)(smem + sizeof(DistillSmem));
  const int64_t row = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
  const int rank = blockIdx.x, ranks = gridDim.x;
  const int tid = threadIdx.x;
  const float c = a.c;
  const T* x_row = (const T*)a.logits + row * a.stride;
  const int32_t v0 = min(a.classes, rank * a.slice);
  const int32_t n = min(a.classes, v0 + a.slice) - v0;
  const Cut<T> cut(x_row + v0, n);
  // the last warp reads the teacher's entries, the others the slice
  const int readers = (int)blockDim.x - 32;
  MaxSum q = {kNegInf, 0.f};
  if (tid >= readers) {
    teacher_row(a, row, c, s);
    // of all classes for the loss, else of this slice's: others' may be overwritten
    const bool all = kMode != kGrad && rank == 0;
    for (int k = tid - readers; k < a.top; k += 32) {
      const int32_t v = s.index[k];
      s.x[k] = v >= 0 && (all || (v >= v0 && v < v0 + n)) ? to_f32(x_row[v]) : 0.f;
    }
  } else if (kMode != kGrad) {
    q = warp_join(read_slice<T>(x_row + v0, cut, kept, a.keep, tid, readers, c), c);
    if (lane_id() == 0) s.part[tid >> 5] = q;
  }
  __syncthreads();
  if (kMode == kGrad) {
    const float2 st = a.stats[row];
    q = {st.x, st.y};
  } else {
    q = {kNegInf, 0.f};
    if (lane_id() < readers >> 5) q = s.part[lane_id()];
    q = warp_join(q, c);
    if (ranks > 1) {
      cg::cluster_group cluster = cg::this_cluster();
      if (tid == 0) s.joined = q;
      cluster.sync();
      q = *cluster.map_shared_rank(&s.joined, 0);
      for (int r = 1; r < ranks; ++r) q = join(q, *cluster.map_shared_rank(&s.joined, r), c);
    }
    if (rank == 0 && tid < 32) {
      const bool some = s.mass != 0.f && q.s != 0.f;  // s = 0: every logit is -inf
      const float loss = some ? row_loss(a, s, q) : 0.f;
      if (tid == 0) {
        a.loss[row] = loss;
        if (kMode == kLoss) a.stats[row] = make_float2(q.m, q.s);
      }
    }
  }
  if (kMode != kLoss) {
    const float coef = (a.weight ? a.weight[row] : 1.f) * a.weight_scale * a.temperature;
    const bool zero = s.mass == 0.f || q.s == 0.f;
    TOut* out = (TOut*)a.out + row * a.out_stride + v0;
    const float inv = 1.f / q.s, factor = coef * s.mass * inv;
    const bool keep = kMode == kStep && a.keep;
    write_slice<T, TOut>(x_row + v0, cut, kept, keep, out, q.m, factor, c, zero);
    __syncthreads();
    for (int k = tid; k < a.top && !zero; k += blockDim.x) {
      const int32_t v = s.index[k] - v0;
      if (s.index[k] < 0 || v < 0 || v >= n) continue;
      // the class's whole mass, by the first of the entries that name it
      float p = 0.f;
      bool first = true;
      for (int j = 0; j < a.top; ++j) {
        if (s.index[j] != v + v0) continue;
        p += s.p[j];
        first &= j >= k;
      }
      if (first)
        out[v] = from_f32<TOut>(coef * (s.mass * inv * exp2_fast((s.x[k] - q.m) * c) - p));
    }
  }
  if (kMode != kGrad && ranks > 1) cg::this_cluster().sync();  // the others have read s.joined
}

// ---- host ------------------------------------------------------------------

constexpr size_t kMaxKeep = 200 * 1024;  // of a slice in shared memory

struct Shape {
  int threads, ranks;
  int32_t slice;
  bool keep;
  size_t smem;
};

Shape distill_shape(int64_t rows, int64_t classes, int64_t size, int mode, int num_sms) {
  Shape s = {};
  const auto slice_of = [&](int64_t ranks) { return ceil_div(ceil_div(classes, ranks), 64) * 64; };
  int64_t ranks = 1;
  if (mode == kGrad) {
    while (slice_of(ranks) * size > 64 * 1024 ||
           (rows * ranks < 4 * num_sms && slice_of(ranks) > 4096))
      ranks *= 2;
  } else {
    // until the slice fits twice in an SM's shared memory, and every SM has work
    while (ranks < kMaxCluster && (slice_of(ranks) * size > 100 * 1024 ||
                                   (rows * ranks < 2 * num_sms && slice_of(ranks) > 4096)))
      ranks *= 2;
  }
  s.ranks = (int)ranks;
  s.slice = (int32_t)slice_of(ranks);
  s.threads = 32 + (s.slice <= 2048 ? 128 : s.slice <= 8192 ? 256 : kMaxReaders);
  const size_t kept = (size_t)(s.slice * size + 32);
  s.keep = mode == kStep && kept <= kMaxKeep;
  s.smem = sizeof(DistillSmem) + (s.keep ? kept : 0);
  return s;
}

template <typename T, typename TOut, int kMode>
cudaError_t launch_distill(DistillArgs a, int64_t rows, int device, cudaStream_t st) {
  const Shape s = distill_shape(rows, a.classes, sizeof(T), kMode, op_num_sms(device));
  a.slice = s.slice;
  a.keep = s.keep;
  const auto kernel = distill_kernel<T, TOut, kMode>;
  static OncePerDevice once;
  cudaError_t e = once.run(device, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)(sizeof(DistillSmem) + (kMode == kStep ? kMaxKeep : 0)));
  });
  if (e != cudaSuccess) return e;
  // rows over two grid dimensions of 65,535 at most; an exact cover, row by row
  for (int64_t r0 = 0; r0 < rows;) {
    const int64_t left = rows - r0;
    const int64_t y = left < 65535 ? left : 65535, z = left / y < 65535 ? left / y : 65535;
    DistillArgs b = a;
    b.logits = (const T*)a.logits + r0 * a.stride;
    const int64_t entries = r0 * a.top;
    b.teacher = (const uint8_t*)a.teacher + entries * float_size(a.teacher_dtype);
    b.index = (const uint8_t*)a.index + entries * (a.index_bits / 8);
    if (a.loss) b.loss = a.loss + r0;
    if (a.stats) b.stats = a.stats + r0;
    if (a.weight) b.weight = a.weight + r0;
    if (a.out) b.out = (TOut*)a.out + r0 * a.out_stride;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)s.ranks, (unsigned)y, (unsigned)z);
    cfg.blockDim = dim3((unsigned)s.threads);
    cfg.dynamicSmemBytes = s.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kMode == kGrad ? 1 : (unsigned)s.ranks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, b);
    if (e != cudaSuccess) return e;
    r0 += y * z;
  }
  return cudaGetLastError();
}

struct DistillCall {
  const char* op;
  int mode;
  const void* logits;
  int32_t logits_dtype;
  int64_t logits_stride, rows, classes;
  const void* teacher;
  int32_t teacher_dtype;
  const void* index;
  int32_t index_bits;
  int64_t top;
  float temperature;
  float* loss;
  float* stats;
  const float* weight;
  float weight_scale;
  void* out;
  int32_t out_dtype;
  int64_t out_stride;
  int32_t* status;
  cudaStream_t st;
};

agnes_status distill(const DistillCall& c) {
  const char* op = c.op;
  const bool wants_loss = c.mode != kGrad, wants_grad = c.mode != kLoss;
  if (c.rows < 0 || c.classes < 1 || c.top < 0)
    return op_error(AGNES_EINVAL, "%s: rows %lld, classes %lld, top %lld", op, (long long)c.rows,
                    (long long)c.classes, (long long)c.top);
  if (c.rows > 0x7fffffff || c.classes > AGNES_DISTILL_MAX_CLASSES || c.top > kMaxTop)
    return op_error(AGNES_ERANGE, "%s: rows %lld, classes %lld, top %lld are too large", op,
                    (long long)c.rows, (long long)c.classes, (long long)c.top);
  if (!(c.temperature > 0.f) || c.temperature > 1e30f || c.temperature < 1e-30f)
    return op_error(AGNES_EINVAL, "%s: a temperature of %g", op, (double)c.temperature);
  OP_TRY(op_float_type(op, "logits", c.logits_dtype));
  OP_TRY(op_float_type(op, "teacher", c.teacher_dtype));
  OP_TRY(op_index_bits(op, "index", c.index_bits));
  if (wants_grad) OP_TRY(op_float_type(op, "out", c.out_dtype));
  if (c.rows > 1 && (c.logits_stride < c.classes || (wants_grad && c.out_stride < c.classes)))
    return op_error(AGNES_EINVAL, "%s: a row stride is below classes %lld", op,
                    (long long)c.classes);
  if (c.rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "logits", c.logits, &device));
  OP_TRY(op_aligned(op, "logits", c.logits, float_size(c.logits_dtype)));
  if (c.top > 0) {
    OP_TRY(op_on_device(op, "teacher", c.teacher, device));
    OP_TRY(op_aligned(op, "teacher", c.teacher, float_size(c.teacher_dtype)));
    OP_TRY(op_on_device(op, "index", c.index, device));
    OP_TRY(op_aligned(op, "index", c.index, c.index_bits / 8));
  }
  if (wants_loss) {
    OP_TRY(op_on_device(op, "loss", c.loss, device));
    OP_TRY(op_aligned(op, "loss", c.loss, 4));
  }
  if (c.mode != kStep) {
    OP_TRY(op_on_device(op, "stats", c.stats, device));
    OP_TRY(op_aligned(op, "stats", c.stats, 8));
  }
  if (wants_grad) {
    OP_TRY(op_on_device(op, "out", c.out, device));
    OP_TRY(op_aligned(op, "out", c.out, float_size(c.out_dtype)));
    if (c.weight) {
      OP_TRY(op_on_device(op, "weight", c.weight, device));
      OP_TRY(op_aligned(op, "weight", c.weight, 4));
    }
    if (c.out == c.logits && (c.out_dtype != c.logits_dtype ||
                              (c.rows > 1 && c.out_stride != c.logits_stride)))
      return op_error(AGNES_EINVAL, "%s: out in place of logits has another type or stride", op);
  }
  if (c.status) OP_TRY(op_on_device(op, "status", c.status, device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  DistillArgs a = {};
  a.logits = c.logits;
  a.stride = c.logits_stride;
  a.classes = (int32_t)c.classes;
  a.teacher = c.teacher;
  a.teacher_dtype = c.teacher_dtype;
  a.index = c.index;
  a.index_bits = c.index_bits;
  a.top = (int32_t)c.top;
  a.temperature = c.temperature;
  a.c = (float)(1.4426950408889634 / (double)c.temperature);
  a.loss = c.loss;
  a.stats = (float2*)c.stats;
  a.weight = c.weight;
  a.weight_scale = c.weight_scale;
  a.out = c.out;
  a.out_stride = c.out_stride;
  a.status = c.status;
  const cudaError_t e = with_float_type(c.logits_dtype, [&](auto tin) {
    using T = typename decltype(tin)::type;
    if (c.mode == kLoss) return launch_distill<T, T, kLoss>(a, c.rows, device, c.st);
    return with_float_type(c.out_dtype, [&](auto tout) {
      using TOut = typename decltype(tout)::type;
      if (c.mode == kGrad) return launch_distill<T, TOut, kGrad>(a, c.rows, device, c.st);
      return launch_distill<T, TOut, kStep>(a, c.rows, device, c.st);
    });
  });
  return op_launched(op, e);
}

}  // namespace

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_distill_loss(const void* logits, int32_t logits_dtype, int64_t logits_stride,
                                int64_t rows, int64_t classes, const void* teacher,
                                int32_t teacher_dtype, const void* index, int32_t index_bits,
                                int64_t top, float temperature, float* loss, float* stats,
                                int32_t* status, void* cuda_stream) {
  return distill({"agnes_distill_loss", kLoss, logits, logits_dtype, logits_stride, rows, classes,
                  teacher, teacher_dtype, index, index_bits, top, temperature, loss, stats, nullptr,
                  1.f, nullptr, 0, 0, status, (cudaStream_t)cuda_stream});
}

agnes_status agnes_distill_grad(const void* logits, int32_t logits_dtype, int64_t logits_stride,
                                int64_t rows, int64_t classes, const void* teacher,
                                int32_t teacher_dtype, const void* index, int32_t index_bits,
                                int64_t top, float temperature, const float* stats,
                                const float* weight, float weight_scale, void* out,
                                int32_t out_dtype, int64_t out_stride, int32_t* status,
                                void* cuda_stream) {
  return distill({"agnes_distill_grad", kGrad, logits, logits_dtype, logits_stride, rows, classes,
                  teacher, teacher_dtype, index, index_bits, top, temperature, nullptr,
                  (float*)stats, weight, weight_scale, out, out_dtype, out_stride, status,
                  (cudaStream_t)cuda_stream});
}

agnes_status agnes_distill_loss_grad(const void* logits, int32_t logits_dtype,
                                     int64_t logits_stride, int64_t rows, int64_t classes,
                                     const void* teacher, int32_t teacher_dtype, const void* index,
                                     int32_t index_bits, int64_t top, float temperature,
                                     const float* weight, float weight_scale, float* loss,
                                     void* out, int32_t out_dtype, int64_t out_stride,
                                     int32_t* status, void* cuda_stream) {
  return distill({"agnes_distill_loss_grad", kStep, logits, logits_dtype, logits_stride, rows,
                  classes, teacher, teacher_dtype, index, index_bits, top, temperature, loss,
                  nullptr, weight, weight_scale, out, out_dtype, out_stride, status,
                  (cudaStream_t)cuda_stream});
}

}  // extern "C"
