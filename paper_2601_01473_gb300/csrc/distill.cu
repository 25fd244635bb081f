// distill.cu -- the loss of a student's logits against a teacher's top logits,
// and its gradient (include/agnes_ops.h).  Of a row x of logits, with the
// teacher's entries (index_k, t_k):
//
//   p = softmax(t / T)    q = softmax(x / T)    loss = T^2 sum_k p_k (ln p_k - ln q_{index_k})
//   d loss / d x_v = T (q_v sum_k p_k - sum_{k: index_k = v} p_k)
//
// One pass over the row keeps a running maximum M and sum S of exp((x - M) / T).
// A cluster of CTAs shares a row, each a slice of it, and joins (M, S) through
// distributed shared memory.  A slice is copied to shared memory by a few bulk copies
// that are all on their way from the start, and a step that also wants the gradient
// takes it from there, so that the logits are read from memory once.  The gradient is
// written as if the teacher had no entry, and then the few entries' classes once more.
#include <cooperative_groups.h>

#include "mbarrier.cuh"
#include "ops_common.cuh"

namespace cg = cooperative_groups;

namespace agnes {

namespace {

constexpr int kMaxTop = AGNES_DISTILL_MAX_TOP;
constexpr int kMaxReaders = 384;
constexpr int kMaxThreads = kMaxReaders + 32;
constexpr int kGradThreads = 256 + 32;  // of the gradient alone, whose slices are small
constexpr int kGradCtas = 7;            // that share an SM
constexpr int kMaxCluster = 8;
constexpr int kCopies = 8;  // bulk copies of a slice
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
  bool keep;  // the slice fits shared memory
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

// The teacher's entries of a row, in shared memory.
struct Entries {
  float* p;        // the teacher's distribution
  int32_t* index;  // -1: absent
  float* x;        // the student's logit at index
};

// A warp: the entries of a row, and the logits at their classes in [lo, hi).  Returns
// the sum of p: 1, or 0 without an entry.
template <typename T>
__device__ __forceinline__ float teacher_row(const DistillArgs& a, int64_t row, const T* x_row,
                                             int32_t lo, int32_t hi, const Entries& s) {
  const int lane = lane_id();
  float top = kNegInf;
  bool bad = false;
  for (int k = lane; k < a.top; k += 32) {
    const int64_t i = row * a.top + k;
    const float t = load_teacher(a, i);  // on its way with the index
    const int64_t v = a.index_bits == 32 ? (int64_t)__ldg((const int32_t*)a.index + i)
                                         : __ldg((const int64_t*)a.index + i);
    const bool in = v >= 0 && v < a.classes;
    bad |= v >= a.classes;
    s.index[k] = in ? (int32_t)v : -1;
    s.x[k] = in && v >= lo && v < hi ? to_f32(x_row[v]) : 0.f;
    s.p[k] = in ? t : kNegInf;
    top = fmaxf(top, s.p[k]);
  }
  if (bad) op_flag(a.status, AGNES_OP_BAD_INDEX);
  top = warp_max(top);
  const float z = above(top);
  float sum = 0.f;
  for (int k = lane; k < a.top; k += 32) {
    const float e = s.index[k] < 0 ? 0.f : exp2_fast((s.p[k] - z) * a.c);
    s.p[k] = e;
    sum += e;
  }
  sum = warp_sum(sum);
  // without an entry, or with -inf alone, there is nothing to divide by
  const bool some = !(sum == 0.f);
  const float inv = some ? 1.f / sum : 0.f;
  for (int k = lane; k < a.top; k += 32) s.p[k] *= inv;
  return some ? sum * inv : 0.f;
}

// A warp: whether two entries name the same class.  `table`: `slots` words, a power of
// two of at least twice the entries.
__device__ __forceinline__ bool repeated(const DistillArgs& a, const Entries& s, int32_t* table,
                                         int slots) {
  const int lane = lane_id();
  for (int i = lane; i < slots; i += 32) table[i] = -1;
  __syncwarp();
  bool twice = false;
  for (int k = lane; k < a.top; k += 32) {
    const int32_t v = s.index[k];
    if (v < 0) continue;
    uint32_t at = (uint32_t)v * 2654435761u >> 16;
    for (int n = 0; n < slots; ++n, ++at) {
      const int32_t old = atomicCAS(table + (at & (uint32_t)(slots - 1)), -1, v);
      twice |= old == v;
      if (old == -1 || old == v) break;
    }
  }
  return __any_sync(0xffffffffu, twice);
}

// A warp: the row's loss.  logit(k): the student's logit at entry k's class.  As
//   2 T sum_k p_k (T/2 (ln p_k + ln S) - (x_k / 2 - M / 2)),
// whose terms leave fp32 only where the loss does: x_k - M itself may, and over T it does for
// a class that is masked by its type's lowest value.
template <typename Logit>
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Entries& s, MaxSum q,
                                          Logit logit) {
  const float half_t = 0.5f * a.temperature, half_m = 0.5f * q.m, log_s = logf(q.s);
  float sum = 0.f;
  for (int k = lane_id(); k < a.top; k += 32) {
    const float p = s.p[k];
    if (p != 0.f && s.index[k] >= 0)
      sum += p * (half_t * (logf(p) + log_s) - (0.5f * logit(k) - half_m));
  }
  return warp_sum(sum) * (2.f * a.temperature);
}

// The entries' classes in [v0, v0 + n) once more: out = coef (mass q - p), where p is
// the class's whole mass, by the first of the entries that name it.  logit(k, v - v0): the
// student's logit at entry k's class.
template <typename TOut, typename Logit>
__device__ __forceinline__ void put_entries(const DistillArgs& a, const Entries& s, bool twice,
                                            TOut* out, int32_t v0, int32_t n, MaxSum q, float coef,
                                            float mass_inv, int tid, int threads, Logit logit) {
  for (int k = tid; k < a.top; k += threads) {
    const int32_t v = s.index[k] - v0;
    if (s.index[k] < 0 || v < 0 || v >= n) continue;
    float p = s.p[k];
    if (twice) {
      bool first = true;
      p = 0.f;
      for (int j = 0; j < a.top; ++j) {
        if (s.index[j] != v + v0) continue;
        p += s.p[j];
        first &= j >= k;
      }
      if (!first) continue;
    }
    out[v] = from_f32<TOut>(coef * (mass_inv * exp2_fast((logit(k, v) - q.m) * a.c) - p));
  }
}

constexpr int kTable = 2 * kMaxTop;
__host__ __device__ inline int table_slots(int top) {  // of a row's table
  int n = 32;
  while (n < 2 * top) n *= 2;
  return n;
}


struct alignas(16) DistillSmem {  // the kept slice follows it, in 16-byte vectors
  float p[kMaxTop];
  int32_t index[kMaxTop];
  float x[kMaxTop];
  int32_t table[kTable];
  MaxSum part[32];         // the readers' warps'
  MaxSum joined;           // this CTA's
  uint64_t bars[kCopies];  // the copies of the slice
  float mass;
  float weight;
  float2 stats;
  bool twice;
};
static_assert(sizeof(DistillSmem) % 16 == 0, "what follows is 16-byte aligned");

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

// The copies of a slice's body: `step` vectors each, a multiple of the readers.
struct Copies {
  int32_t step, count;
  __device__ Copies(int32_t body, int readers) {
    step = (body + kCopies * readers - 1) / (kCopies * readers) * readers;
    count = step > 0 ? (body + step - 1) / step : 0;
  }
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}

// One thread: has the whole body copied to shared memory.
template <typename T>
__device__ __forceinline__ void start_copies(const T* x, const Cut<T>& cut, T* kept,
                                             const Copies& copies, uint64_t* bars) {
  for (int i = 0; i < copies.count; ++i) mbar_init(smem_addr(bars + i), 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  for (int i = 0; i < copies.count; ++i) {
    const int32_t first = i * copies.step;
    const uint32_t bytes = 16u * (uint32_t)min(copies.step, cut.body - first);
    const uint32_t bar = smem_addr(bars + i);
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
            "r"(smem_addr(kept + cut.shift + cut.head) + 16u * (uint32_t)first),
        "l"(x + cut.head + (int64_t)first * Cut<T>::kN), "r"(bytes), "r"(bar)
        : "memory");
  }
}

// Waits for copy i; a wait that ran out is reported and tried once more, as the CTA
// may not leave before its copies have landed.
__device__ __forceinline__ void wait_copy(uint64_t* bars, int i, int32_t* status) {
  const uint32_t bar = smem_addr(bars + i);
  if (mbar_wait(bar, 0)) return;
  op_flag(status, AGNES_OP_TIMEOUT);
  mbar_wait(bar, 0);
}

// A slice's few elements before and after its body to shared memory.
template <typename T, typename F>
__device__ __forceinline__ void ragged_ends(const T* x, const Cut<T>& cut, int tid, F&& f) {
  if (tid < cut.head) f(tid, x[tid]);
  const int32_t i = cut.tail0() + tid;
  if (i < cut.n) f(i, x[i]);
}

// A reader's share of a slice in shared memory.
template <typename T>
__device__ __forceinline__ MaxSum read_kept(const T* x, const Cut<T>& cut, T* kept,
                                            const Copies& copies, uint64_t* bars, int tid,
                                            int threads, float c, int32_t* status) {
  constexpr int kN = Cut<T>::kN;
  Running r = {kNegInf, pack2(0.f, 0.f)};
  ragged_ends(x, cut, tid, [&](int32_t i, T v) {
    kept[cut.shift + i] = v;
    r.take_one(to_f32(v), c);
  });
  const Vec<T, kN>* body = (const Vec<T, kN>*)(kept + cut.shift + cut.head);
  for (int i = 0; i < copies.count; ++i) {
    wait_copy(bars, i, status);
    const int32_t end = min(cut.body, (i + 1) * copies.step);
#pragma unroll 2
    for (int32_t j = i * copies.step + tid; j < end; j += threads) r.take(body[j], c);
  }
  return r.sum();
}

// The same from memory, for slices that do not fit.
template <typename T>
__device__ __forceinline__ MaxSum read_slice(const T* x, const Cut<T>& cut, int tid, int threads,
                                             float c) {
  constexpr int kN = Cut<T>::kN, kAhead = 4;
  Running r = {kNegInf, pack2(0.f, 0.f)};
  const Vec<T, kN>* body = (const Vec<T, kN>*)(x + cut.head);
  int32_t j = tid;
  for (; j + (kAhead - 1) * threads < cut.body; j += kAhead * threads) {
    Vec<T, kN> v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = body[j + u * threads];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) r.take(v[u], c);
  }
  for (; j < cut.body; j += threads) r.take(body[j], c);
  ragged_ends(x, cut, tid, [&](int32_t, T v) { r.take_one(to_f32(v), c); });
  return r.sum();
}

// out = factor * 2^((x - m) c) for the slice, from shared memory or from x.
template <typename T, typename TOut>
__device__ __forceinline__ void write_slice(const T* x, const Cut<T>& cut, const T* kept, bool keep,
                                            TOut* out, float m, float factor, float c, bool zero,
                                            int tid, int threads) {
  constexpr int kN = Cut<T>::kN;
  constexpr int kOutBytes = kN * sizeof(TOut), kPart = kOutBytes > 16 ? 16 : kOutBytes;
  constexpr int kPartN = kPart / (int)sizeof(TOut);
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
__global__ void __launch_bounds__(kMode == kGrad ? kGradThreads : kMaxThreads,
                                  kMode == kGrad ? kGradCtas : 2)
distill_kernel(DistillArgs a) {
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
  const Copies copies(cut.body, readers);
  if (a.keep) {
    if (tid == 0) start_copies(x_row + v0, cut, kept, copies, s.bars);
    __syncthreads();
  }
  const Entries entries = {s.p, s.index, s.x};
  const bool whole = a.keep && ranks == 1;  // the whole row is kept
  MaxSum q = {kNegInf, 0.f};
  if (tid >= readers) {
    const int lane = tid - readers;
    if (lane == 0 && kMode != kLoss) {
      s.weight = a.weight ? __ldg(a.weight + row) : 1.f;
      if (kMode == kGrad) s.stats = a.stats[row];
    }
    // the logits of all classes for the loss, else of this slice (others' may be
    // overwritten); none that are kept
    const bool all = kMode != kGrad && rank == 0 && !whole;
    const float mass = teacher_row(a, row, x_row, all ? 0 : v0,
                                   all ? a.classes : a.keep ? v0 : v0 + n, entries);
    const bool twice = kMode != kLoss && repeated(a, entries, s.table, table_slots(a.top));
    if (lane == 0) {
      s.mass = mass;
      s.twice = twice;
    }
  } else if (kMode == kGrad) {
    if (a.keep) ragged_ends(x_row + v0, cut, tid, [&](int32_t i, T v) { kept[cut.shift + i] = v; });
  } else {
    q = a.keep ? read_kept(x_row + v0, cut, kept, copies, s.bars, tid, readers, c, a.status)
               : read_slice(x_row + v0, cut, tid, readers, c);
    q = warp_join(q, c);
    if (lane_id() == 0) s.part[tid >> 5] = q;
  }
  __syncthreads();
  if (kMode == kGrad) {
    q = {s.stats.x, s.stats.y};
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
    if (rank == 0 && tid >= readers) {
      const bool some = s.mass != 0.f && q.s != 0.f;  // s = 0: every logit is -inf
      const float loss =
          some ? row_loss(a, entries, q,
                          [&](int k) {
                            return whole ? to_f32(kept[cut.shift + s.index[k]]) : s.x[k];
                          })
               : 0.f;
      if (tid == readers) {
        a.loss[row] = loss;
        if (kMode == kLoss) a.stats[row] = make_float2(q.m, q.s);
      }
    }
  }
  if (kMode != kLoss) {
    const float coef = s.weight * a.weight_scale * a.temperature;
    const bool zero = s.mass == 0.f || q.s == 0.f;
    TOut* out = (TOut*)a.out + row * a.out_stride + v0;
    const float mass_inv = s.mass / q.s;
    if (kMode == kGrad && a.keep)
      for (int i = 0; i < copies.count; ++i) wait_copy(s.bars, i, a.status);
    write_slice<T, TOut>(x_row + v0, cut, kept, a.keep, out, q.m, coef * mass_inv, c, zero, tid,
                         blockDim.x);
    __syncthreads();
    if (!zero)
      put_entries(a, entries, s.twice, out, v0, n, q, coef, mass_inv, tid, blockDim.x,
                  [&](int k, int32_t v) { return a.keep ? to_f32(kept[cut.shift + v]) : s.x[k]; });
  }
  if (kMode != kGrad && ranks > 1) cg::this_cluster().sync();  // the others have read s.joined
}

// Short rows, a warp to each: nothing to join but its lanes, and no barrier.  The row is
// read again for the gradient: from L1 or L2 as far as they hold the rows in flight, from
// memory past that (fp32 rows of 8192 classes and many of them, is_short).
constexpr int kShortWarps = 8;

template <typename T, typename TOut, int kMode>
__global__ void __launch_bounds__(32 * kShortWarps) distill_short_kernel(DistillArgs a,
                                                                         int64_t rows) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = lane_id();
  const int64_t row = (int64_t)blockIdx.x * kShortWarps + warp;
  if (row >= rows) return;
  const int slots = kMode == kLoss ? 0 : table_slots(a.top);
  float* const mine = (float*)smem + warp * (3 * a.top + slots);
  const Entries entries = {mine, (int32_t*)(mine + a.top), mine + 2 * a.top};
  const T* x = (const T*)a.logits + row * a.stride;
  const Cut<T> cut(x, a.classes);
  MaxSum q;
  if (kMode == kGrad) {
    const float2 st = a.stats[row];
    q = {st.x, st.y};
  } else {
    q = warp_join(read_slice(x, cut, lane, 32, a.c), a.c);
  }
  const float mass = teacher_row(a, row, x, 0, a.classes, entries);
  const bool zero = mass == 0.f || q.s == 0.f;
  __syncwarp();
  if (kMode != kGrad) {
    const float loss =
        zero ? 0.f : row_loss(a, entries, q, [&](int k) { return entries.x[k]; });
    if (lane == 0) {
      a.loss[row] = loss;
      if (kMode == kLoss) a.stats[row] = make_float2(q.m, q.s);
    }
  }
  if (kMode != kLoss) {
    const bool twice = repeated(a, entries, (int32_t*)(mine + 3 * a.top), slots);
    const float coef = (a.weight ? __ldg(a.weight + row) : 1.f) * a.weight_scale * a.temperature;
    TOut* out = (TOut*)a.out + row * a.out_stride;
    const float mass_inv = mass / q.s;
    write_slice<T, TOut>(x, cut, nullptr, false, out, q.m, coef * mass_inv, a.c, zero, lane, 32);
    __syncwarp();
    if (!zero)
      put_entries(a, entries, twice, out, 0, a.classes, q, coef, mass_inv, lane, 32,
                  [&](int k, int32_t) { return entries.x[k]; });
  }
}

// ---- host ------------------------------------------------------------------

constexpr size_t kMaxKeep = 200 * 1024;  // of a slice in shared memory
constexpr int64_t kGradSlice = 26 * 1024;
constexpr int kMidSlice = 20000;  // classes that 256 threads read
static_assert(kGradSlice / 2 <= kMidSlice, "the gradient alone runs 256 threads at most");

struct Shape {
  int threads, ranks;
  int32_t slice;
  bool keep;
  size_t smem;
};

// How a row is cut.  A CTA's barriers, joins and trips to memory for the entries take
// microseconds beside its slice, so CTAs that share an SM hide one another's: two of
// 100 KB where the slice is kept for the gradient (8192 rows of 50,000 bf16 classes, a
// step: 305 us, 396 with four of 50 KB), eight of 26 KB where nothing is joined (the
// gradient alone: 303 us, 370 with 64 KB).  Threads by what is left for each, and where
// every SM has CTAs enough: 4096 rows of 10,007 fp16 classes, a step: 128 42 us, 256 58,
// 512 76; 64 rows of 131,072 want 256.  The limits lie between those shapes and were not
// measured one by one.
Shape distill_shape(int64_t rows, int64_t classes, int64_t size, int mode, int num_sms) {
  Shape s = {};
  const auto slice_of = [&](int64_t ranks) { return ceil_div(ceil_div(classes, ranks), 64) * 64; };
  int64_t ranks = 1;
  if (mode == kGrad) {
    while (slice_of(ranks) * size > kGradSlice ||
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
  s.threads = 32 + (s.slice <= 2048 || (s.slice <= 16384 && rows >= 4 * num_sms) ? 128
                    : s.slice <= kMidSlice                                        ? 256
                                                                                  : kMaxReaders);
  const size_t kept = (size_t)(s.slice * size + 32);
  s.keep = kept <= kMaxKeep;
  s.smem = sizeof(DistillSmem) + (s.keep ? kept : 0);
  return s;
}

// Whether a row is a warp's.  A warp reads a few vectors at a time, so only very short
// rows are where there are too few of them to fill the SMs.  With the gradient, up to
// 8192 classes (4096 rows of 6000 fp16 classes, a step: 30 us, 34 by CTAs; of 10,007: 56
// and 42); for the loss alone, which reads each row once, up to 65,536 (8192 rows of
// 50,000 bf16 classes: 145 us, 188 by CTAs).  The limit is in classes, and fp32 rows of
// many classes, which are twice as long, would be better off by CTAs: a step of 16,384 rows
// of 1000 42 us (88 by CTAs) and of 2000 67 (95), but of 8192 rows of 4096 77 (63), of 6000
// 120 (70), of 8192 159 (89); in fp16 of 4096 35 (54), of 6000 58 (62), of 8192 80 (71).
bool is_short(int64_t rows, int64_t classes, int mode, int num_sms) {
  const int64_t most = mode == kLoss ? 65536 : 8192;
  return classes <= 512 || (classes <= most && rows >= 8 * num_sms);
}

template <typename T, typename TOut, int kMode>
cudaError_t launch_distill(DistillArgs a, int64_t rows, int device, cudaStream_t st) {
  if (is_short(rows, a.classes, kMode, op_num_sms(device))) {
    const size_t smem =
        4 * kShortWarps * (size_t)(3 * a.top + (kMode == kLoss ? 0 : table_slots(a.top)));
    static OncePerDevice once;
    const cudaError_t e = once.run(device, [] {
      return cudaFuncSetAttribute(distill_short_kernel<T, TOut, kMode>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  4 * kShortWarps * (3 * kMaxTop + table_slots(kMaxTop)));
    });
    if (e != cudaSuccess) return e;
    distill_short_kernel<T, TOut, kMode>
        <<<(unsigned)ceil_div(rows, kShortWarps), 32 * kShortWarps, smem, st>>>(a, rows);
    return cudaGetLastError();
  }
  const Shape s = distill_shape(rows, a.classes, sizeof(T), kMode, op_num_sms(device));
  a.slice = s.slice;
  a.keep = s.keep;
  const auto kernel = distill_kernel<T, TOut, kMode>;
  static OncePerDevice once;
  cudaError_t e = once.run(device, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)(sizeof(DistillSmem) + kMaxKeep));
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
  OP_TRY(op_status(op, c.status, device));
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
