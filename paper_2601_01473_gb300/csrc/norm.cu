// norm.cu -- the step between two blocks of a residual network (include/agnes_ops.h):
//
//   u = N(branch) after + after_bias,  sum = x + scale gate u,  next = N(sum) before + before_bias
//
// with N(v) = (v - mean v) / sqrt(var v + eps) or v / sqrt(mean v^2 + eps), and its
// gradient.  With s^ = N(sum), r = 1 / the root, D = d_next before:
//   d = d_sum + r (D - mean D - s^ mean(D s^))       (without mean D for the second N)
//   dx = d;  dgate = scale d u;  du = scale gate d
//   dbranch = the same map of du after with branch's N and root
//   dbefore = sum d_next s^, dbefore_bias = sum d_next, dafter = sum du b^, dafter_bias = sum du,
// the last ones over the rows.  Both statistics are computed again in the backward pass,
// from rows that it reads anyway.
//
// Bound by memory.  A group of threads holds a row in registers and reads it once; mean and
// variance take two turns over the registers, as their difference would lose what large
// means leave.  For the sums over rows a thread keeps to its columns while its group goes
// from row to row, each CTA writes one partial row, and a second kernel adds those up in
// order: the result is the same each time.
// 786,432 x 128 fp16, with all of it, 146 us (5.2 TB/s) and 257 back; back of 16,384 x 4096, fp32
// with bfloat16, 254 us (4.7 TB/s).
#include <algorithm>

#include "int8.cuh"

namespace agnes {

namespace {

// Of a row to a thread, forward.  Rows of up to kShortDim columns take fewer, and two rows at a
// time (786,432 x 128 fp16 to fp16 144 us and not 242, 400,000 x 256 149 and not 252), and so
// does the backward pass, which has more to hold.
constexpr int kElems = 16;
constexpr int kShortElems = 8;
constexpr int kShortDim = 256;
constexpr int kNormLanes = 512;  // threads to a row at most, forward
constexpr int64_t kNormMaxDim = 8192;
static_assert(kNormLanes * kElems >= kNormMaxDim && kRowLanesMax * kShortElems >= kNormMaxDim,
              "a row in registers");
constexpr int64_t kNormMaxRows = 0x7fffffff - 2047;
constexpr int kSums = 5;  // of before, after, gate, before_bias and after_bias

struct NormArgs {
  int64_t rows;
  int32_t dim, lanes, log_lanes, groups;
  const void *x, *branch, *gate;  // the backward pass has the sum as x
  int64_t x_stride, branch_stride, gate_stride;
  int32_t gate_kind;
  const float *after, *after_bias, *before, *before_bias;
  float scale, eps, inv_dim;
  bool layer;
  // forward
  void *sum, *next;
  int64_t sum_stride, next_stride;
  bool next_rows8;
  int32_t batches, stage_at[5];  // of the staged rows: `groups` at a time, and their buffers
  // backward
  const void *d_next, *d_sum;
  int64_t d_next_stride, d_sum_stride;
  void *dx, *dbranch, *dgate;
  int64_t dx_stride, dbranch_stride, dgate_stride;
  int32_t stages, stage_off;  // of the copies ahead, and where they lie, in 16 bytes
  int32_t run_at[8], run_stage;  // of staged runs: the buffers, and a stage's bytes
  float* partial;      // [CTAs][sums][dim]
  int32_t slot[kSums];  // a sum's place among them, or -1
  int32_t sums;
};

// Two values of fp32 in one register pair, for the packed arithmetic: each half is rounded
// as by a single instruction.
struct Two {
  uint64_t p;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.p) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ Two both(float a) { return two(a, a); }
__device__ __forceinline__ float2 apart(Two a) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(a.p));
  return f;
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.p) : "l"(a.p), "l"(b.p));
  return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.p) : "l"(a.p), "l"(b.p));
  return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.p) : "l"(a.p), "l"(b.p), "l"(c.p));
  return r;
}

// Two values rounded to T, as they are then.
template <typename T>
__device__ __forceinline__ Two rounded(Two a) {
  const float2 f = apart(a);
  if constexpr (std::is_same<T, __half>::value) {
    const float2 r = __half22float2(__floats2half2_rn(f.x, f.y));
    return two(r.x, r.y);
  } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    const uint32_t w = *(const uint32_t*)&h;
    return two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  } else {
    return a;
  }
}

// 1 / sqrt(x): the estimate corrected once by its residual, where that is a number.
__device__ __forceinline__ float inverse_root(float x) {
  const float y = rsqrtf(x), r = fmaf(-x * y, y, 1.f);
  return r == r ? fmaf(0.5f * y, r, y) : y;
}

// A thread's values of a row: vector i's are pairs i * kVec / 2 on.  kLanes: threads to a row
// where that is known.
template <int kVec, int kPer, int kLanes = 0>
struct NormRow {
  static constexpr int kPairs = kVec * kPer / 2;
  using Values = Two[kPairs];
  RowPart<kVec, kPer> part;
  RowScratch* scratch;
  int turn = 0;

  template <typename T>
  static __device__ void unpack(const RowRegs<T, kVec, kPer>& from, Values& v) {
    float f[kVec * kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) from.get(i, f + i * kVec);
#pragma unroll
    for (int e = 0; e < kPairs; ++e) v[e] = two(f[2 * e], f[2 * e + 1]);
  }
  template <typename T>
  __device__ void load(const T* row, bool valid, Values& v) const {
    RowRegs<T, kVec, kPer> r;
    r.load(part, row, valid);
    unpack(r, v);
  }
  template <typename T>
  __device__ void store(T* row, bool valid, const Values& v) const {
    float f[kVec * kPer];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      const float2 x = apart(v[e]);
      f[2 * e] = x.x;
      f[2 * e + 1] = x.y;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) part.store_one(row, valid, i, f + i * kVec);
  }
  // whether the elements of pair e are in the row: of single elements they are apart
  __device__ bool has(int e, int half) const { return part.has((2 * e + half) / kVec); }

  static __device__ float total(const Values& v) {
    Two s = v[0];
#pragma unroll
    for (int e = 1; e < kPairs; ++e) s = s + v[e];
    const float2 f = apart(s);
    return f.x + f.y;
  }
  static __device__ float total(const Values& v, const Values& w) {
    Two s = v[0] * w[0];
#pragma unroll
    for (int e = 1; e < kPairs; ++e) s = fma2(v[e], w[e], s);
    const float2 f = apart(s);
    return f.x + f.y;
  }

  template <int kCount>
  __device__ void sum(float (&v)[kCount]) {
    group_reduce<SumOp, kLanes>(v, part.lanes, scratch, turn);
  }

  // v becomes what it is without its mean (of AGNES_NORM_LAYER), zeros past the row's end;
  // inv is 1 / the root.
  template <int kRows>
  __device__ void standard(Values (&v)[kRows], bool layer, float eps, float inv_dim,
                           float (&inv)[kRows]) {
    float s[kRows];
    if (layer) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) s[r] = total(v[r]);
      sum(s);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const float mean = -(s[r] * inv_dim);
#pragma unroll
        for (int e = 0; e < kPairs; ++e)
          v[r][e] = v[r][e] + two(has(e, 0) ? mean : 0.f, has(e, 1) ? mean : 0.f);
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) s[r] = total(v[r], v[r]);
    sum(s);
#pragma unroll
    for (int r = 0; r < kRows; ++r) inv[r] = inverse_root(fmaf(s[r], inv_dim, eps));
  }

  // `standard` of two independent rows at once, either of which may be left out
  __device__ void standard_of(Values& x, bool with_x, Values& y, bool with_y, bool layer,
                              float eps, float inv_dim, float& inv_x, float& inv_y) {
    float s[2] = {0.f, 0.f};
    const auto centre = [&](Values& v, float sum) {
      const float mean = -(sum * inv_dim);
#pragma unroll
      for (int e = 0; e < kPairs; ++e)
        v[e] = v[e] + two(has(e, 0) ? mean : 0.f, has(e, 1) ? mean : 0.f);
    };
    if (layer) {
      if (with_x) s[0] = total(x);
      if (with_y) s[1] = total(y);
      sum(s);
      if (with_x) centre(x, s[0]);
      if (with_y) centre(y, s[1]);
    }
    if (with_x) s[0] = total(x, x);
    if (with_y) s[1] = total(y, y);
    sum(s);
    inv_x = inverse_root(fmaf(s[0], inv_dim, eps));
    inv_y = inverse_root(fmaf(s[1], inv_dim, eps));
  }

  // A vector over the columns; `fill` where there is none.
  __device__ void vector(const float* p, float fill, Values& v) const {
    if (p) {
      load(p, true, v);
    } else {
#pragma unroll
      for (int e = 0; e < kPairs; ++e) v[e] = both(fill);
    }
  }

  // the gradient to v of the gradient d to n = N(v)
  __device__ void through(Values& d, const Values& n, bool layer, float inv, float inv_dim) {
    float along, mean = 0.f;
    if (layer) {
      float s[2] = {total(d, n), total(d)};
      sum(s);
      along = s[0];
      mean = s[1] * inv_dim;
    } else {
      float s[1] = {total(d, n)};
      sum(s);
      along = s[0];
    }
    const Two a = both(-(along * inv_dim)), m = both(-mean), i = both(inv);
#pragma unroll
    for (int e = 0; e < kPairs; ++e) d[e] = (fma2(n[e], a, d[e]) + m) * i;
  }
};

// Where a group's rows are: in memory, or a batch of them in shared memory.
template <typename TX, typename TBranch>
struct NormRowsAt {
  const NormArgs& a;
  int64_t row0;
  __device__ int64_t row(int r) const { return row0 + (int64_t)r * a.groups; }
  __device__ bool valid(int r) const { return row(r) < a.rows; }
  __device__ const TX* x(int r) const { return (const TX*)a.x + row(r) * a.x_stride; }
  __device__ const TBranch* branch(int r) const {
    return (const TBranch*)a.branch + row(r) * a.branch_stride;
  }
  __device__ const TBranch* gate(int r) const {
    return (const TBranch*)a.gate + row(r) * a.gate_stride;
  }
  __device__ TX* sum(int r) const { return (TX*)a.sum + row(r) * a.sum_stride; }
  __device__ TBranch* next(int r) const { return (TBranch*)a.next + row(r) * a.next_stride; }
  __device__ uint8_t* next8(int r) const { return (uint8_t*)a.next + row(r) * a.next_stride; }
};

// A CTA's rows are one run of each matrix; a buffer in shared memory for each.
template <typename TX, typename TBranch>
struct NormStage {
  const NormArgs& a;
  uint8_t* base;
  int64_t row0;
  int rows, at;  // of the CTA; the group's
  __device__ bool valid(int) const { return at < rows; }
  template <typename T>
  __device__ T* first(const void* p, int64_t stride) const {
    return (T*)p + row0 * stride;
  }
  template <typename T>
  __device__ T* in(int buffer, const void* p) const {
    return (T*)(base + a.stage_at[buffer] + stage_offset(first<T>(p, a.dim))) + (int64_t)at * a.dim;
  }
  __device__ const TX* x(int) const { return in<TX>(0, a.x); }
  __device__ const TBranch* branch(int) const { return in<TBranch>(1, a.branch); }
  __device__ const TBranch* gate(int) const { return in<TBranch>(2, a.gate); }
  __device__ TX* sum(int) const { return in<TX>(3, a.sum); }
  __device__ TBranch* next(int) const { return in<TBranch>(4, a.next); }
  __device__ uint8_t* next8(int) const { return base + a.stage_at[4] + at * a.next_stride; }
  template <typename T>
  __device__ void load_one(int buffer, const void* p) const {
    stage_in(base + a.stage_at[buffer], first<T>(p, a.dim), rows * (int64_t)a.dim * (int64_t)sizeof(T),
             p, first<T>(p, a.dim) + (a.rows - row0) * a.dim);
  }
  __device__ void load() const {
    load_one<TX>(0, a.x);
    if (a.branch) load_one<TBranch>(1, a.branch);
    if (a.gate_kind == AGNES_GATE_ROWS) load_one<TBranch>(2, a.gate);
    stage_wait();
  }
  __device__ void store() const {
    __syncthreads();
    if (a.branch)
      stage_out(base + a.stage_at[3], first<TX>(a.sum, a.dim),
                rows * (int64_t)a.dim * (int64_t)sizeof(TX));
    if (!a.next) return;
    if (a.next_rows8)
      stage_out(base + a.stage_at[4], first<uint8_t>(a.next, a.next_stride), rows * a.next_stride);
    else
      stage_out(base + a.stage_at[4], first<TBranch>(a.next, a.dim),
                rows * (int64_t)a.dim * (int64_t)sizeof(TBranch));
  }
};

template <typename TX, typename TBranch, int kVec, int kPer, int kRows, int kLanes, typename At>
__device__ __forceinline__ void norm_rows(const NormArgs& a, NormRow<kVec, kPer, kLanes>& n,
                                          const At& at) {
  using Row = NormRow<kVec, kPer, kLanes>;
  constexpr int kPairs = Row::kPairs;
  RowRegs<TX, kVec, kPer> x_regs[kRows];
  RowRegs<TBranch, kVec, kPer> b_regs[kRows], g_regs[kRows];
  const bool gate_rows = a.gate_kind == AGNES_GATE_ROWS;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const bool valid = at.valid(r);
    x_regs[r].load(n.part, at.x(r), valid);
    if (a.branch) b_regs[r].load(n.part, at.branch(r), valid);
    if (gate_rows) g_regs[r].load(n.part, at.gate(r), valid);
  }
  Two x[kRows][kPairs], w[kPairs], b[kPairs];
  float inv[kRows];
  if (a.branch) {
    Two u[kRows][kPairs];
#pragma unroll
    for (int r = 0; r < kRows; ++r) Row::unpack(b_regs[r], u[r]);
    if (a.after) {
      n.standard(u, a.layer, a.eps, a.inv_dim, inv);
      n.vector(a.after, 1.f, w);
      n.vector(a.after_bias, 0.f, b);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < kPairs; ++e) u[r][e] = fma2(u[r][e] * both(inv[r]), w[e], b[e]);
    }
    // scale gate
    if (!gate_rows) {
      n.vector(a.gate_kind == AGNES_GATE_COLUMNS ? (const float*)a.gate : nullptr, 1.f, w);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) w[e] = w[e] * both(a.scale);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (gate_rows) {
        Row::unpack(g_regs[r], w);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) w[e] = w[e] * both(a.scale);
      }
      Row::unpack(x_regs[r], x[r]);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) x[r][e] = rounded<TX>(fma2(w[e], u[r][e], x[r][e]));
      n.store(at.sum(r), at.valid(r), x[r]);
    }
  } else {
#pragma unroll
    for (int r = 0; r < kRows; ++r) Row::unpack(x_regs[r], x[r]);
  }
  if (!a.next) return;
  n.standard(x, a.layer, a.eps, a.inv_dim, inv);
  n.vector(a.before, 1.f, w);
  n.vector(a.before_bias, 0.f, b);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int e = 0; e < kPairs; ++e) x[r][e] = fma2(x[r][e] * both(inv[r]), w[e], b[e]);
  if (a.next_rows8) {
    uint32_t top[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      top[r] = 0;
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const float2 f = apart(x[r][e]);
        top[r] = max(top[r], max(__float_as_uint(f.x) & 0x7fffffffu,
                                 __float_as_uint(f.y) & 0x7fffffffu));
      }
    }
    group_reduce<MaxBits, kLanes>(top, a.lanes, n.scratch, n.turn);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const Int8Scale s = int8_scale(top[r]);
      uint8_t* to = at.next8(r);
      const bool valid = at.valid(r);
      float f[2 * kPairs];
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const float2 v = apart(x[r][e]);
        f[2 * e] = v.x;
        f[2 * e + 1] = v.y;
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) int8_store(n.part, to, valid, i, f + i * kVec, s);
      int8_store_end(to, a.dim, n.part.lane, a.lanes, valid, s);
    }
  } else {
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      n.store(at.next(r), at.valid(r), x[r]);
  }
}

// kRows rows to a group at a time: the vectors over the columns are loaded once for all of
// them, and the exchanges of their sums overlap.
template <typename TX, typename TBranch, int kVec, int kPer, int kRows, int kLanes>
__global__ void __launch_bounds__(kLanes ? kRowThreads : kNormLanes)
norm_kernel(const NormArgs a) {
  __shared__ RowScratch scratch;
  const int group = threadIdx.x >> a.log_lanes, lane = threadIdx.x & (a.lanes - 1);
  NormRow<kVec, kPer, kLanes> n = {{a.lanes, lane, a.dim}, &scratch};
  const NormRowsAt<TX, TBranch> at = {a, ((int64_t)blockIdx.x * kRows) * a.groups + group};
  norm_rows<TX, TBranch, kVec, kPer, kRows, kLanes>(a, n, at);
}

// Rows that no vector divides, of contiguous matrices with branches of 16 bits, through shared
// memory: 200,000 x 301 fp16 287 us, 900 by single elements, 16,000 x 4095, fp32 with bfloat16,
// 352 and 719.  With ten or twelve values to a thread where they hold a row: 287 and 380 with
// sixteen.  Bound by its instructions on single elements.  (All in fp32, 200,000 x 301 took 401
// and 438, 8000 x 8191 537 and 415: those stay with single elements.  Two rows at a time for the
// vectors' sake: 241 there, but 419 and not 314 with an fp32 residual.)  Two CTAs to an SM leave a
// thread 64 registers: 48, 100 or 248 bytes are spilled with ten, twelve or sixteen values to it.
template <typename TX, typename TBranch, int kPer>
__global__ void __launch_bounds__(kNormLanes, 2)
norm_staged_kernel(const NormArgs a) {
  __shared__ RowScratch scratch;
  extern __shared__ uint4 norm_smem[];
  const int group = threadIdx.x >> a.log_lanes, lane = threadIdx.x & (a.lanes - 1);
  NormRow<1, kPer> n = {{a.lanes, lane, a.dim}, &scratch};
  const int64_t row0 = (int64_t)blockIdx.x * a.groups * a.batches, left = a.rows - row0;
  const int most = a.groups * a.batches;
  NormStage<TX, TBranch> at = {a, (uint8_t*)norm_smem, row0, left < most ? (int)left : most, group};
  at.load();
  for (int batch = 0; batch < a.batches; ++batch, at.at += a.groups)
    norm_rows<TX, TBranch, 1, kPer, 1, 0>(a, n, at);
  at.store();
}

// A thread's sums over the rows: in registers, or (kShared) in shared memory, where a thread
// has too few of them.
template <int kPairs, int kCount, bool kShared>
struct Totals {
  Two v[kShared ? 1 : kCount][kPairs];
  float4* mine;  // [sum][quad][thread]
  __device__ void init(float4* shared) {
    mine = shared + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kCount; ++k)
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        if constexpr (kShared) {
          if (e % 2 == 0)
            mine[(k * (kPairs / 2) + e / 2) * blockDim.x] = make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
          v[k][e] = both(0.f);
        }
      }
  }
  // of pairs e and e + 1
  __device__ void add(int k, int e, Two a, Two b) {
    if constexpr (kShared) {
      float4* at = mine + (k * (kPairs / 2) + e / 2) * blockDim.x;
      const float4 t = *at;
      const float2 x = apart(a + two(t.x, t.y)), y = apart(b + two(t.z, t.w));
      *at = make_float4(x.x, x.y, y.x, y.y);
    } else {
      v[k][e] = v[k][e] + a;
      v[k][e + 1] = v[k][e + 1] + b;
    }
  }
  __device__ void add_product(int k, int e, Two a, Two b, Two c, Two d) {
    if constexpr (kShared) {
      add(k, e, a * b, c * d);
    } else {
      v[k][e] = fma2(a, b, v[k][e]);
      v[k][e + 1] = fma2(c, d, v[k][e + 1]);
    }
  }
  __device__ float get(int k, int at) const {
    if constexpr (kShared) {
      return ((const float*)&mine[(k * (kPairs / 2) + at / 4) * blockDim.x])[at % 4];
    } else {
      const float2 f = apart(v[k][at / 2]);
      return at & 1 ? f.y : f.x;
    }
  }
};

// The vectors over the columns of the backward pass, in shared memory where there is room
// beside the sums: a thread's of one vector are kElems / 4 quads, quad q of all threads to a
// row side by side, zeros past the row's end.  What there is none of is ones, or zeros for
// the bias.
enum { kBeforeVector, kAfterVector, kAfterBiasVector, kGateVector, kVectors };
template <int kVec, int kPer, int kLanes>
struct ColumnVectors {
  using Row = NormRow<kVec, kPer, kLanes>;
  static constexpr int kQuads = kVec * kPer / 4;
  float4* at;
  __device__ void init(const NormArgs& a, const Row& r, float4* shared) {
    at = shared;
    if ((int)threadIdx.x >= a.lanes) return;  // one group's threads fill them
    const float* const from[kVectors] = {
        a.before, a.after, a.after_bias,
        a.gate_kind == AGNES_GATE_COLUMNS ? (const float*)a.gate : nullptr};
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
      Two v[Row::kPairs];
      r.vector(from[k], k == kAfterBiasVector ? 0.f : 1.f, v);
#pragma unroll
      for (int q = 0; q < kQuads; ++q) {
        const float2 x = apart(v[2 * q]), y = apart(v[2 * q + 1]);
        at[(k * kQuads + q) * a.lanes + r.part.lane] = make_float4(x.x, x.y, y.x, y.y);
      }
    }
  }
  __device__ void get(const Row& r, int k, typename Row::Values& v) const {
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
      const float4 x = at[(k * kQuads + q) * r.part.lanes + r.part.lane];
      v[2 * q] = two(x.x, x.y);
      v[2 * q + 1] = two(x.z, x.w);
    }
  }
};

// Which sums there are, so that the others take no registers: of before, after and gate, or
// of the biases too.
enum { kBefore, kAfter, kGateSum, kBeforeBias, kAfterBias, kMostSums };

// What a row of the backward pass needs.  kAsync: it is on its way for some rows ahead, copied
// to slots of shared memory that only the thread itself reads, of which there are `stages`.
// Otherwise it is loaded when its row is due.
template <typename TX, typename TBranch, int kVec, int kPer, bool kAsync, int kLanes>
struct GradRow {
  using Row = NormRow<kVec, kPer, kLanes>;
  static constexpr int kX = sizeof(TX) / 2, kB = sizeof(TBranch) / 2;  // 16-byte pieces
  enum { kPieces = 2 * (kX + kB) };
  const NormArgs& a;
  const RowPart<kVec, kPer>& part;
  uint4* slots;  // this thread's: piece p of stage s at (s * kPieces + p) * blockDim.x
  int stages;

  template <typename T>
  __device__ void copy(const void* from, int64_t row, int64_t stride, int slot, int piece) const {
    constexpr int kBytes = kVec * sizeof(T), kAccess = kBytes < 16 ? kBytes : 16;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool there = from && row < a.rows && part.has(i);
      const uint8_t* at = there ? (const uint8_t*)((const T*)from + row * stride + part.col(i))
                                : (const uint8_t*)a.x;
      const uint32_t bytes = there ? kAccess : 0;  // the others are zeros
#pragma unroll
      for (int h = 0; h < kBytes; h += kAccess) {
        const int byte = i * kBytes + h;
        const uint32_t to =
            (uint32_t)__cvta_generic_to_shared(
                slots + (slot * kPieces + piece + byte / 16) * (int)blockDim.x) + byte % 16;
        if constexpr (kAccess == 16)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to),
                       "l"(at + (there ? h : 0)), "r"(bytes)
                       : "memory");
        else
          asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to),
                       "l"(at), "r"(bytes)
                       : "memory");
      }
    }
  }
  // Starts a row's copies; one group each, of rows past the end too, so that the wait's count
  // holds.
  __device__ void start(int64_t row, int slot) const {
    if constexpr (kAsync) {
      if (row < a.rows) {
        copy<TX>(a.before ? a.x : nullptr, row, a.x_stride, slot, 0);
        copy<TX>(a.d_sum, row, a.d_sum_stride, slot, kX);
        copy<TBranch>(a.before ? a.d_next : nullptr, row, a.d_next_stride, slot, 2 * kX);
        copy<TBranch>(a.branch, row, a.branch_stride, slot, 2 * kX + kB);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  }
  __device__ void wait() const {
    if constexpr (kAsync) {
      if (stages == 4)
        asm volatile("cp.async.wait_group 3;" ::: "memory");
      else if (stages == 3)
        asm volatile("cp.async.wait_group 2;" ::: "memory");
      else  // there are two at least
        asm volatile("cp.async.wait_group 1;" ::: "memory");
    }
  }
  template <typename T>
  __device__ void get(const void* from, int64_t row, int64_t stride, int slot, int piece,
                      typename Row::Values& v) const {
    if constexpr (kAsync) {
      RowRegs<T, kVec, kPer> r;
      uint32_t* words = &r.w[0][0];
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const uint4 q = slots[(slot * kPieces + piece + h) * (int)blockDim.x];
        words[4 * h] = q.x;
        words[4 * h + 1] = q.y;
        words[4 * h + 2] = q.z;
        words[4 * h + 3] = q.w;
      }
      Row::unpack(r, v);
    } else {
      RowRegs<T, kVec, kPer> r;
      r.load(part, (const T*)from + row * stride, row < a.rows);
      Row::unpack(r, v);
    }
  }
  __device__ void x(int64_t row, int slot, typename Row::Values& v) const {
    get<TX>(a.x, row, a.x_stride, slot, 0, v);
  }
  __device__ void d_sum(int64_t row, int slot, typename Row::Values& v) const {
    get<TX>(a.d_sum, row, a.d_sum_stride, slot, kX, v);
  }
  __device__ void d_next(int64_t row, int slot, typename Row::Values& v) const {
    get<TBranch>(a.d_next, row, a.d_next_stride, slot, 2 * kX, v);
  }
  __device__ void branch(int64_t row, int slot, typename Row::Values& v) const {
    get<TBranch>(a.branch, row, a.branch_stride, slot, 2 * kX + kB, v);
  }
};

// The same of rows that no vector divides, of contiguous matrices: the rows that a CTA has at a
// time are one run of each matrix, which lies in shared memory, a turn ahead; what they give
// goes out by runs, too.
enum { kRunX, kRunDSum, kRunDNext, kRunBranch, kRunGate, kRunDx, kRunDBranch, kRunDGate };
template <typename TX, typename TBranch>
struct GradRun {
  const NormArgs& a;
  uint8_t* base;
  int group;
  int64_t first = 0;  // of the turn
  int stage = 0;
  __device__ int rows(int64_t from) const {
    const int64_t left = a.rows - from;
    return left < a.groups ? (int)left : a.groups;
  }
  template <typename T>
  __device__ void start_one(int buffer, const void* p, int64_t from, int to_stage) const {
    if (!p) return;
    const T* at = (const T*)p + from * a.dim;
    stage_in(base + to_stage * a.run_stage + a.run_at[buffer], at,
             rows(from) * (int64_t)a.dim * (int64_t)sizeof(T), p, (const T*)p + a.rows * a.dim);
  }
  // one group of copies each, past the end too, so that the wait's count holds
  __device__ void start(int64_t from, int to_stage) const {
    if (from < a.rows) {
      start_one<TX>(kRunX, a.before ? a.x : nullptr, from, to_stage);
      start_one<TX>(kRunDSum, a.d_sum, from, to_stage);
      start_one<TBranch>(kRunDNext, a.before ? a.d_next : nullptr, from, to_stage);
      start_one<TBranch>(kRunBranch, a.branch, from, to_stage);
      start_one<TBranch>(kRunGate, a.gate_kind == AGNES_GATE_ROWS ? a.gate : nullptr, from, to_stage);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ void wait() const {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();
  }
  template <typename T>
  __device__ const T* in(int buffer, const void* p) const {
    return (const T*)(base + stage * a.run_stage + a.run_at[buffer] +
                      stage_offset((const T*)p + first * a.dim)) + group * a.dim;
  }
  template <typename T>
  __device__ T* out(int buffer, void* p) const {
    return (T*)(base + a.run_at[buffer] + stage_offset((T*)p + first * a.dim)) + group * a.dim;
  }
  template <typename T>
  __device__ void store_one(int buffer, void* p) const {
    stage_out(base + a.run_at[buffer], (T*)p + first * a.dim,
              rows(first) * (int64_t)a.dim * (int64_t)sizeof(T));
  }
  __device__ void store() const {
    __syncthreads();
    store_one<TX>(kRunDx, a.dx);
    if (a.branch) store_one<TBranch>(kRunDBranch, a.dbranch);
    if (a.gate_kind == AGNES_GATE_ROWS) store_one<TBranch>(kRunDGate, a.dgate);
  }
};

template <typename TX, typename TBranch, int kVec, int kPer, int kThreads, bool kBias, bool kShared,
          int kLanes, bool kRun = false>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 2 : 1)
norm_grad_kernel(const NormArgs a) {
  using Row = NormRow<kVec, kPer, kLanes>;
  constexpr int kPairs = Row::kPairs;
  constexpr int kCount = kBias ? kMostSums : kBeforeBias;
  __shared__ RowScratch scratch;
  extern __shared__ float4 grad_smem[];  // shared sums, or [groups][dim] of the end
  const int group = threadIdx.x >> a.log_lanes, lane = threadIdx.x & (a.lanes - 1);
  Row r = {{a.lanes, lane, a.dim}, &scratch};
  Totals<kPairs, kCount, kShared> total;
  total.init(grad_smem);
  ColumnVectors<kVec, kPer, kLanes> columns;
  if constexpr (!kShared) {
    columns.init(a, r, grad_smem);
    __syncthreads();
  }
  const auto vector = [&](int k, const float* p, float fill, Two (&v)[kPairs]) {
    if constexpr (kShared)
      r.vector(p, fill, v);
    else
      columns.get(r, k, v);
  };
  const int64_t step = (int64_t)gridDim.x * a.groups;
  GradRow<TX, TBranch, kVec, kPer, kVec != 1 && !kShared, kLanes> in = {a, r.part, (uint4*)(grad_smem + a.stage_off) + threadIdx.x,
                                         a.stages};
  for (int k = 0; k + 1 < a.stages; ++k)
    in.start((int64_t)blockIdx.x * a.groups + group + k * step, k);
  GradRun<TX, TBranch> run = {a, (uint8_t*)(grad_smem + a.stage_off), group};
  if constexpr (kRun) run.start((int64_t)blockIdx.x * a.groups, 0);
  int slot = 0, fill = a.stages - 1;
  for (int64_t first = (int64_t)blockIdx.x * a.groups; first < a.rows; first += step) {
    const int64_t row = first + group;
    const bool valid = row < a.rows;
    Two d[kPairs], w[kPairs], n[kPairs], branch[kPairs];
    float inv, branch_inv;
    if constexpr (kRun) {
      run.first = first;
      run.start(first + step, run.stage ^ 1);
      run.wait();
    } else {
      in.start(row + (a.stages - 1) * step, fill);
      in.wait();
    }
    if (a.d_sum) {
      if constexpr (kRun)
        r.load(run.template in<TX>(kRunDSum, a.d_sum), valid, d);
      else
        in.d_sum(row, slot, d);
    } else {
#pragma unroll
      for (int e = 0; e < kPairs; ++e) d[e] = both(0.f);
    }
    Two g[kPairs];
    if constexpr (kRun) {
      if (a.before) {
        r.load(run.template in<TX>(kRunX, a.x), valid, n);
        r.load(run.template in<TBranch>(kRunDNext, a.d_next), valid, g);
      }
      if (a.branch) r.load(run.template in<TBranch>(kRunBranch, a.branch), valid, branch);
    } else {
      if (a.before) {
        in.x(row, slot, n);
        in.d_next(row, slot, g);
      }
      if (a.branch) in.branch(row, slot, branch);
      if (++slot == a.stages) slot = 0;
      if (++fill == a.stages) fill = 0;
    }
    r.standard_of(n, a.before, branch, a.after, a.layer, a.eps, a.inv_dim, inv, branch_inv);
    if (a.before) {
      vector(kBeforeVector, a.before, 1.f, w);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) n[e] = n[e] * both(inv);
      if (valid) {  // where there is no row and eps is 0, n is no number
#pragma unroll
        for (int e = 0; e < kPairs; e += 2) {
          total.add_product(kBefore, e, g[e], n[e], g[e + 1], n[e + 1]);
          if constexpr (kBias) total.add(kBeforeBias, e, g[e], g[e + 1]);
        }
      }
#pragma unroll
      for (int e = 0; e < kPairs; ++e) g[e] = g[e] * w[e];
      r.through(g, n, a.layer, inv, a.inv_dim);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) d[e] = d[e] + g[e];
    }
    r.store(kRun ? run.template out<TX>(kRunDx, a.dx) : (TX*)a.dx + row * a.dx_stride, valid, d);
    if (!a.branch) {
      if constexpr (kRun) {
        run.store();
        run.stage ^= 1;
      }
      continue;
    }
    if (a.after) {
#pragma unroll
      for (int e = 0; e < kPairs; ++e) branch[e] = branch[e] * both(branch_inv);
    }
#pragma unroll
    for (int e = 0; e < kPairs; ++e) d[e] = d[e] * both(a.scale);
    if (a.gate_kind != AGNES_GATE_NONE) {
      // u, then d u
      vector(kAfterVector, a.after, 1.f, w);
      Two b[kPairs];
      vector(kAfterBiasVector, a.after_bias, 0.f, b);
#pragma unroll
      for (int e = 0; e < kPairs; ++e) b[e] = fma2(branch[e], w[e], b[e]);
      if (a.gate_kind == AGNES_GATE_ROWS) {
        Two gate[kPairs];
        r.load(kRun ? run.template in<TBranch>(kRunGate, a.gate)
                    : (const TBranch*)a.gate + row * a.gate_stride, valid, gate);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          b[e] = d[e] * b[e];
          d[e] = d[e] * gate[e];
        }
        r.store(kRun ? run.template out<TBranch>(kRunDGate, a.dgate)
                     : (TBranch*)a.dgate + row * a.dgate_stride, valid, b);
      } else {
        if (valid) {
#pragma unroll
          for (int e = 0; e < kPairs; e += 2)
            total.add_product(kGateSum, e, d[e], b[e], d[e + 1], b[e + 1]);
        }
        vector(kGateVector, (const float*)a.gate, 1.f, b);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) d[e] = d[e] * b[e];
      }
    }
    if (a.after) {
      vector(kAfterVector, a.after, 1.f, w);
      if (valid) {
#pragma unroll
        for (int e = 0; e < kPairs; e += 2) {
          total.add_product(kAfter, e, d[e], branch[e], d[e + 1], branch[e + 1]);
          if constexpr (kBias) total.add(kAfterBias, e, d[e], d[e + 1]);
        }
      }
#pragma unroll
      for (int e = 0; e < kPairs; ++e) d[e] = d[e] * w[e];
      r.through(d, branch, a.layer, branch_inv, a.inv_dim);
    }
    r.store(kRun ? run.template out<TBranch>(kRunDBranch, a.dbranch)
                 : (TBranch*)a.dbranch + row * a.dbranch_stride, valid, d);
    if constexpr (kRun) {
      run.store();
      run.stage ^= 1;
    }
  }
  // a CTA's sums: its groups' added in order
#pragma unroll
  for (int k = 0; k < kCount; ++k) {
    if (a.slot[k] < 0) continue;
    float* to = a.partial + ((int64_t)blockIdx.x * a.sums + a.slot[k]) * a.dim;
    if (a.groups == 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (r.part.has(i)) to[r.part.col(i) + e] = total.get(k, i * kVec + e);
      continue;
    }
    float* group_sums = (float*)grad_smem;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (r.part.has(i)) group_sums[group * a.dim + r.part.col(i) + e] = total.get(k, i * kVec + e);
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += blockDim.x) {
      float sum = 0.f;
      for (int g = 0; g < a.groups; ++g) sum += group_sums[g * a.dim + c];
      to[c] = sum;
    }
  }
}

struct JoinArgs {
  const float* partial;
  int32_t parts, sums, dim;
  float* out[kSums];  // by place
};

// A warp to 32 columns of a sum would wait for `parts` loads in a row: 32 threads share a
// column's parts, and their sums are added up in order.
constexpr int kJoinShares = 32;
__global__ void __launch_bounds__(32 * kJoinShares)
norm_join_kernel(const JoinArgs a) {
  grid_dep_wait();
  __shared__ float part_sum[kJoinShares][32];
  const int lane = threadIdx.x & 31, share = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane, k = blockIdx.y;
  float sum = 0.f;
  if (c < a.dim)
#pragma unroll 4
    for (int p = share; p < a.parts; p += kJoinShares)
      sum += a.partial[((int64_t)p * a.sums + k) * a.dim + c];
  part_sum[share][lane] = sum;
  __syncthreads();
  if (share == 0 && c < a.dim) {
#pragma unroll
    for (int s = 1; s < kJoinShares; ++s) sum += part_sum[s][lane];
    a.out[k][c] = sum;
  }
}

// f(TypeTag of x, TypeTag of branch): x's type is the branch's or fp32.
template <typename F>
cudaError_t with_norm_types(int32_t x_dtype, int32_t branch_dtype, F&& f) {
  return with_float_type(branch_dtype, [&](auto b) {
    using TBranch = typename decltype(b)::type;
    if (x_dtype == branch_dtype) return f(TypeTag<TBranch>(), b);
    return f(TypeTag<float>(), b);
  });
}

agnes_status check_sizes(const char* op, int64_t rows, int64_t dim) {
  if (rows < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, dim %lld", op, (long long)rows, (long long)dim);
  if (rows > kNormMaxRows || dim > kNormMaxDim)
    return op_error(AGNES_ERANGE, "%s: rows %lld, dim %lld are too large", op, (long long)rows,
                    (long long)dim);
  return AGNES_OK;
}

agnes_status check_matrix(const char* op, const char* name, const void* p, int64_t rows,
                          int64_t dim, int64_t stride, int64_t size, int* device) {
  if (*device < 0)
    OP_TRY(op_device_of(op, name, p, device));
  else
    OP_TRY(op_on_device(op, name, p, *device));
  OP_TRY(op_aligned(op, name, p, size));
  if (rows > 1 && stride < dim)
    return op_error(AGNES_EINVAL, "%s: a stride of %lld of %s is below dim %lld", op,
                    (long long)stride, name, (long long)dim);
  return AGNES_OK;
}

agnes_status check_vector(const char* op, const char* name, const void* p, int device) {
  if (!p) return AGNES_OK;
  OP_TRY(op_on_device(op, name, p, device));
  return op_aligned(op, name, p, 4);
}

// What both passes have in common.
agnes_status check_kinds(const char* op, const NormArgs& a, int32_t x_dtype, int32_t branch_dtype,
                         int32_t kind) {
  OP_TRY(op_float_type(op, "x", x_dtype));
  OP_TRY(op_float_type(op, "branch", branch_dtype));
  if (x_dtype != branch_dtype && x_dtype != AGNES_F32)
    return op_error(AGNES_EINVAL, "%s: x has neither branch's type nor fp32", op);
  if (kind != AGNES_NORM_RMS && kind != AGNES_NORM_LAYER)
    return op_error(AGNES_EINVAL, "%s: an unknown kind of norm (%d)", op, kind);
  if (a.gate_kind != AGNES_GATE_NONE && a.gate_kind != AGNES_GATE_COLUMNS &&
      a.gate_kind != AGNES_GATE_ROWS)
    return op_error(AGNES_EINVAL, "%s: an unknown kind of gate (%d)", op, a.gate_kind);
  if (!(a.eps >= 0.f)) return op_error(AGNES_EINVAL, "%s: eps is below zero", op);
  // a matrix without rows may be NULL
  if (a.rows > 0 && !a.branch && (a.after || a.after_bias || a.gate_kind != AGNES_GATE_NONE))
    return op_error(AGNES_EINVAL, "%s: a gate or a norm of a branch that is NULL", op);
  if (a.rows > 0 && !a.branch && !a.before)
    return op_error(AGNES_EINVAL, "%s: neither branch nor before: nothing to compute", op);
  if ((a.after_bias && !a.after) || (a.before_bias && !a.before))
    return op_error(AGNES_EINVAL, "%s: a bias without its norm", op);
  return AGNES_OK;
}

agnes_status check_inputs(const char* op, const NormArgs& a, int32_t x_dtype, int32_t branch_dtype,
                          int* device) {
  OP_TRY(check_matrix(op, "x", a.x, a.rows, a.dim, a.x_stride, float_size(x_dtype), device));
  if (a.branch)
    OP_TRY(check_matrix(op, "branch", a.branch, a.rows, a.dim, a.branch_stride,
                        float_size(branch_dtype), device));
  if (a.gate_kind == AGNES_GATE_ROWS) {
    OP_TRY(check_matrix(op, "gate", a.gate, a.rows, a.dim, a.gate_stride, float_size(branch_dtype),
                        device));
  } else if (a.gate_kind == AGNES_GATE_COLUMNS) {
    if (!a.gate) return op_error(AGNES_EINVAL, "%s: gate is NULL", op);
    OP_TRY(check_vector(op, "gate", a.gate, *device));
  }
  OP_TRY(check_vector(op, "after", a.after, *device));
  OP_TRY(check_vector(op, "after_bias", a.after_bias, *device));
  OP_TRY(check_vector(op, "before", a.before, *device));
  return check_vector(op, "before_bias", a.before_bias, *device);
}

// Whether every access of a row's matrices and vectors can have 16 bytes.
class Wide {
 public:
  explicit Wide(const NormArgs& a) : next_(a.rows > 1 ? 1 : 0), ok_(a.dim % 8 == 0) {}
  Wide& rows(const void* p, int64_t stride, int64_t size) {
    if (p) ok_ = ok_ && aligned_rows(p, next_ * stride * size, 16);
    return *this;
  }
  Wide& vector(const void* p) { return rows(p, 0, 4); }
  bool ok() const { return ok_; }

 private:
  int64_t next_;
  bool ok_;
};

bool wide_inputs(const NormArgs& a, int64_t x_size, int64_t branch_size) {
  return Wide(a)
      .rows(a.x, a.x_stride, x_size)
      .rows(a.branch, a.branch_stride, branch_size)
      .rows(a.gate_kind == AGNES_GATE_ROWS ? a.gate : nullptr, a.gate_stride, branch_size)
      .vector(a.gate_kind == AGNES_GATE_COLUMNS ? a.gate : nullptr)
      .vector(a.after)
      .vector(a.after_bias)
      .vector(a.before)
      .vector(a.before_bias)
      .ok();
}

// Of rows of up to kShortDim columns, for kernels that know their threads to a row: 8, 16
// or 32.
RowShape short_shape(int64_t dim) {
  RowShape s = row_shape(dim, kShortElems);
  if (s.lanes < 8) s = {8, 3, kRowThreads / 8};
  return s;
}

void set_shape(NormArgs& a, const RowShape& shape) {
  a.lanes = shape.lanes;
  a.log_lanes = shape.log_lanes;
  a.groups = shape.groups;
  a.inv_dim = 1.f / (float)a.dim;
}

// Of matrices that are one run each.
template <typename TX, typename TBranch>
cudaError_t launch_staged(NormArgs a, int device, cudaStream_t st) {
  set_shape(a, row_shape(a.dim, kElems, kNormLanes));
  const int64_t x_row = a.dim * (int64_t)sizeof(TX), b_row = a.dim * (int64_t)sizeof(TBranch);
  const int64_t next_row = !a.next ? 0 : a.next_rows8 ? int8_row_bytes(a.dim) : b_row;
  const int64_t row[5] = {x_row, a.branch ? b_row : 0, a.gate_kind == AGNES_GATE_ROWS ? b_row : 0,
                          a.branch ? x_row : 0, next_row};
  a.next_stride = a.next_rows8 ? int8_row_bytes(a.dim) : a.dim;
  a.batches = stage_batches(a.rows, a.groups, row[0] + row[1] + row[2] + row[3] + row[4],
                            op_num_sms(device));
  const int64_t rows = a.groups * (int64_t)a.batches;
  int64_t smem = 0;
  for (int k = 0; k < 5; ++k) {
    a.stage_at[k] = (int32_t)smem;
    if (row[k]) smem += staged_bytes(rows * row[k]);
  }
  const int per = (a.dim + a.lanes - 1) / a.lanes, which = per <= 10 ? 0 : per <= 12 ? 1 : 2;
  const auto kernel = which == 0   ? norm_staged_kernel<TX, TBranch, 10>
                      : which == 1 ? norm_staged_kernel<TX, TBranch, 12>
                                   : norm_staged_kernel<TX, TBranch, kElems>;
  // the longest rows take most, one to a CTA: an fp32 residual and its sum, a branch, a full gate
  // and next in 16 bits, 114,768 bytes with what their first and last pieces have besides
  constexpr int kMost = (int)(kNormMaxDim * (2 * 4 + 3 * 2) + 5 * 16);
  static_assert(kMost > staged_bytes(49152) + 4 * 32, "or a batch of shorter ones");
  static OncePerDevice once[3];
  const cudaError_t e = once[which].run(device, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
  });
  if (e != cudaSuccess) return e;
  kernel<<<(unsigned)ceil_div(a.rows, rows), (unsigned)(a.lanes * a.groups), (size_t)smem, st>>>(a);
  return cudaGetLastError();
}

// CTAs of the backward pass: each writes a row of partial sums, so no more than keep the
// device busy.
int64_t grad_ctas(int64_t rows, int64_t dim, int sms) {
  const RowShape shape = short_shape(dim);
  const int64_t ctas = ceil_div(rows, shape.groups);
  // a thread's sums and the row ahead leave room for 512 threads to an SM
  const int64_t most = (int64_t)sms * (shape.threads() <= 256 ? 2 : 1);
  return ctas < most ? ctas : most;
}
constexpr int kMostSms = 256;  // for the size of a workspace, whatever device it will be on

// A sum's bytes of shared memory where the threads keep it there.
size_t dim_smem(const NormArgs& a) { return (size_t)a.lanes * kShortElems * 4; }

template <typename TX, typename TBranch, bool kBias>
cudaError_t launch_grad(NormArgs a, bool wide, bool contiguous, int64_t ctas, size_t smem,
                        int device, cudaStream_t st) {
  using Kernel = void (*)(NormArgs);
  constexpr int kPer = kShortElems;
  // With a residual in fp32 a thread has two vectors of four columns, so that each access of
  // a warp is one run of memory (16,384 x 4096, bf16 branch, 253 us; with eight columns to a
  // thread 346 past L1 and 328 through it).
  constexpr int kV = sizeof(TX) == 4 ? 4 : 8, kP = kShortElems / kV;
  const Kernel kernels[8] = {norm_grad_kernel<TX, TBranch, kV, kP, 1024, kBias, true, 0>,
                             norm_grad_kernel<TX, TBranch, 1, kPer, 1024, kBias, true, 0>,
                             norm_grad_kernel<TX, TBranch, 1, kPer, 512, kBias, false, 0>,
                             norm_grad_kernel<TX, TBranch, kV, kP, 512, kBias, false, 0>,
                             norm_grad_kernel<TX, TBranch, kV, kP, 256, kBias, false, 8>,
                             norm_grad_kernel<TX, TBranch, kV, kP, 256, kBias, false, 16>,
                             norm_grad_kernel<TX, TBranch, kV, kP, 256, kBias, false, 32>,
                             norm_grad_kernel<TX, TBranch, 1, kPer, 512, kBias, false, 0, true>};
  int which = a.lanes > 512 ? (wide ? 0 : 1) : !wide ? 2 : a.lanes > 32 ? 3
                    : a.lanes == 8 ? 4 : a.lanes == 16 ? 5 : 6;
  // as many rows ahead as there is room for in the 227 KB of an SM's CTAs
  a.stages = 1;
  a.stage_off = (int32_t)ceil_div((int64_t)smem, 16);
  // with more than two turns: 200,000 x 301 fp16 718 us, 871 by single elements, all in fp32 678
  // and 742, 500,000 x 100 fp16 382 and 488; in one turn 100 x 301 takes 11.6 and 9.9
  if (which == 2 && contiguous && a.rows > 2 * ctas * a.groups) {
    const int64_t x_run = staged_bytes(a.groups * (int64_t)a.dim * (int64_t)sizeof(TX));
    const int64_t b_run = staged_bytes(a.groups * (int64_t)a.dim * (int64_t)sizeof(TBranch));
    const bool gate = a.gate_kind == AGNES_GATE_ROWS;
    const int64_t bytes[8] = {a.before ? x_run : 0, a.d_sum ? x_run : 0, a.before ? b_run : 0,
                              a.branch ? b_run : 0, gate ? b_run : 0, x_run, a.branch ? b_run : 0,
                              gate ? b_run : 0};
    int64_t at = 0;
    for (int k = 0; k < 5; ++k) {
      a.run_at[k] = (int32_t)at;
      at += bytes[k];
    }
    a.run_stage = (int32_t)at;
    at *= 2;
    for (int k = 5; k < 8; ++k) {
      a.run_at[k] = (int32_t)at;
      at += bytes[k];
    }
    // Without room for two stages (all in fp32 with a full gate above some 3,100 columns) single
    // elements are read from memory after all: 16,000 x 3501 779 us, 539 with a gate by column.
    if ((int64_t)a.stage_off * 16 + at <= 224 * 1024) {
      which = 7;
      smem = (size_t)a.stage_off * 16 + (size_t)at;
    }
  } else if (which >= 3) {
    const int threads = a.lanes * a.groups;
    const size_t stage = (size_t)GradRow<TX, TBranch, kV, kP, true, 0>::kPieces * 16 * threads;
    const size_t room = (threads <= 256 ? 110 : 224) * 1024 - (size_t)a.stage_off * 16;
    a.stages = (int32_t)std::min((size_t)4, room / stage);
    smem = (size_t)a.stage_off * 16 + a.stages * stage;
  }
  const Kernel kernel = kernels[which];
  static OncePerDevice once[8];
  const cudaError_t e = once[which].run(device, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 * 1024);
  });
  if (e != cudaSuccess) return e;
  kernel<<<(unsigned)ctas, (unsigned)(a.lanes * a.groups), smem, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_residual_norm(const void* x, int32_t x_dtype, int64_t x_stride,
                                 const void* branch, int32_t branch_dtype, int64_t branch_stride,
                                 int64_t rows, int64_t dim, const void* gate, int32_t gate_kind,
                                 int64_t gate_stride, float scale, const float* after,
                                 const float* after_bias, const float* before,
                                 const float* before_bias, int32_t kind, float eps, void* sum,
                                 int64_t sum_stride, void* next, int32_t next_dtype,
                                 int64_t next_stride, void* cuda_stream) {
  const char* op = "agnes_residual_norm";
  OP_TRY(check_sizes(op, rows, dim));
  NormArgs a = {};
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.x = x;
  a.x_stride = x_stride;
  a.branch = branch;
  a.branch_stride = branch_stride;
  a.gate = gate;
  a.gate_kind = gate_kind;
  a.gate_stride = gate_stride;
  a.scale = scale;
  a.after = after;
  a.after_bias = after_bias;
  a.before = before;
  a.before_bias = before_bias;
  a.layer = kind == AGNES_NORM_LAYER;
  a.eps = eps;
  a.sum = sum;
  a.sum_stride = sum_stride;
  OP_TRY(check_kinds(op, a, x_dtype, branch_dtype, kind));
  if (before) {
    a.next = next;
    a.next_stride = next_stride;
    a.next_rows8 = next_dtype == AGNES_INT8_ROWS;
    if (a.next_rows8)
      OP_TRY(int8_check_stride(op, "next", rows, dim, next_stride));
    else if (next_dtype != branch_dtype)
      return op_error(AGNES_EINVAL, "%s: next has another type than branch", op);
  }
  if (rows == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(check_inputs(op, a, x_dtype, branch_dtype, &device));
  const int64_t x_size = float_size(x_dtype), branch_size = float_size(branch_dtype);
  if (branch) OP_TRY(check_matrix(op, "sum", sum, rows, dim, sum_stride, x_size, &device));
  if (before && a.next_rows8) {
    OP_TRY(op_on_device(op, "next", next, device));
    OP_TRY(op_aligned(op, "next", next, 16));
  } else if (before) {
    OP_TRY(check_matrix(op, "next", next, rows, dim, next_stride, branch_size, &device));
  }
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const bool wide = wide_inputs(a, x_size, branch_size) &&
                    Wide(a)
                        .rows(branch ? sum : nullptr, sum_stride, x_size)
                        .rows(a.next_rows8 ? nullptr : a.next, next_stride, branch_size)
                        .ok();
  const auto one_run = [&](int64_t stride) { return rows == 1 || stride == dim; };
  const bool contiguous = one_run(x_stride) &&
                          (!branch || (one_run(branch_stride) && one_run(sum_stride))) &&
                          (gate_kind != AGNES_GATE_ROWS || one_run(gate_stride)) &&
                          (!before || (a.next_rows8 ? rows == 1 || next_stride == int8_row_bytes(dim)
                                                    : one_run(next_stride)));
  return op_launched(op, with_norm_types(x_dtype, branch_dtype, [&](auto tx, auto tb) {
    using TX = typename decltype(tx)::type;
    using TBranch = typename decltype(tb)::type;
    if constexpr (sizeof(TBranch) == 2)
      if (!wide && contiguous)
        return launch_staged<TX, TBranch>(a, device, (cudaStream_t)cuda_stream);
    const bool brief = wide && dim <= kShortDim;
    set_shape(a, brief ? short_shape(dim) : row_shape(dim, kElems, kNormLanes));
    const auto kernel = !wide          ? norm_kernel<TX, TBranch, 1, kElems, 1, 0>
                        : !brief       ? norm_kernel<TX, TBranch, 8, 2, 1, 0>
                        : a.lanes == 8 ? norm_kernel<TX, TBranch, 8, 1, 2, 8>
                        : a.lanes == 16 ? norm_kernel<TX, TBranch, 8, 1, 2, 16>
                                        : norm_kernel<TX, TBranch, 8, 1, 2, 32>;
    kernel<<<(unsigned)ceil_div(rows, a.groups * (brief ? 2 : 1)), (unsigned)(a.lanes * a.groups), 0,
             (cudaStream_t)cuda_stream>>>(a);
    return cudaGetLastError();
  }));
}

agnes_status agnes_residual_norm_grad_workspace(int64_t rows, int64_t dim, int64_t* bytes) {
  const char* op = "agnes_residual_norm_grad_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_sizes(op, rows, dim));
  *bytes = grad_ctas(rows, dim, kMostSms) * kSums * dim * 4;
  return AGNES_OK;
}

agnes_status agnes_residual_norm_grad(
    const void* d_next, int64_t d_next_stride, const void* d_sum, int64_t d_sum_stride,
    const void* sum, int32_t x_dtype, int64_t sum_stride, const void* branch, int32_t branch_dtype,
    int64_t branch_stride, int64_t rows, int64_t dim, const void* gate, int32_t gate_kind,
    int64_t gate_stride, float scale, const float* after, const float* after_bias,
    const float* before, int32_t kind, float eps, void* dx, int64_t dx_stride, void* dbranch,
    int64_t dbranch_stride, void* dgate, int64_t dgate_stride, float* dafter, float* dafter_bias,
    float* dbefore, float* dbefore_bias, void* workspace, int64_t workspace_bytes,
    void* cuda_stream) {
  const char* op = "agnes_residual_norm_grad";
  OP_TRY(check_sizes(op, rows, dim));
  NormArgs a = {};
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.x = sum;
  a.x_stride = sum_stride;
  a.branch = branch;
  a.branch_stride = branch_stride;
  a.gate = gate;
  a.gate_kind = gate_kind;
  a.gate_stride = gate_stride;
  a.scale = scale;
  a.after = after;
  a.after_bias = after_bias;
  a.before = before;
  a.layer = kind == AGNES_NORM_LAYER;
  a.eps = eps;
  a.d_next = d_next;
  a.d_next_stride = d_next_stride;
  a.d_sum = d_sum;
  a.d_sum_stride = d_sum_stride;
  a.dx = dx;
  a.dx_stride = dx_stride;
  a.dbranch = dbranch;
  a.dbranch_stride = dbranch_stride;
  a.dgate = dgate;
  a.dgate_stride = dgate_stride;
  OP_TRY(check_kinds(op, a, x_dtype, branch_dtype, kind));
  if ((dafter || dafter_bias) && !after)
    return op_error(AGNES_EINVAL, "%s: dafter without after", op);
  if ((dbefore || dbefore_bias) && !before)
    return op_error(AGNES_EINVAL, "%s: dbefore without before", op);
  float* const outs[kSums] = {dbefore, dafter,
                              gate_kind == AGNES_GATE_COLUMNS ? (float*)dgate : nullptr,
                              dbefore_bias, dafter_bias};
  const char* const names[kSums] = {"dbefore", "dafter", "dgate", "dbefore_bias", "dafter_bias"};
  JoinArgs join = {};
  for (int k = 0; k < kSums; ++k) {
    a.slot[k] = outs[k] ? a.sums++ : -1;
    if (outs[k]) join.out[a.slot[k]] = outs[k];
  }
  int device = -1;
  if (rows > 0) {
    OP_TRY(check_inputs(op, a, x_dtype, branch_dtype, &device));
    const int64_t x_size = float_size(x_dtype), branch_size = float_size(branch_dtype);
    if (before)
      OP_TRY(check_matrix(op, "d_next", d_next, rows, dim, d_next_stride, branch_size, &device));
    if (d_sum) OP_TRY(check_matrix(op, "d_sum", d_sum, rows, dim, d_sum_stride, x_size, &device));
    OP_TRY(check_matrix(op, "dx", dx, rows, dim, dx_stride, x_size, &device));
    if (branch)
      OP_TRY(check_matrix(op, "dbranch", dbranch, rows, dim, dbranch_stride, branch_size, &device));
    if (gate_kind == AGNES_GATE_ROWS)
      OP_TRY(check_matrix(op, "dgate", dgate, rows, dim, dgate_stride, branch_size, &device));
    else if (gate_kind == AGNES_GATE_COLUMNS && !dgate)
      return op_error(AGNES_EINVAL, "%s: dgate is NULL", op);
  }
  for (int k = 0; k < kSums; ++k) {
    if (!outs[k]) continue;
    if (device < 0) OP_TRY(op_device_of(op, names[k], outs[k], &device));
    OP_TRY(check_vector(op, names[k], outs[k], device));
  }
  if (device < 0) return AGNES_OK;
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (rows == 0) {  // sums over no rows
    for (int k = 0; k < kSums; ++k)
      if (outs[k])
        OP_TRY(op_launched(op, cudaMemsetAsync(outs[k], 0, (size_t)dim * 4, st)));
    return AGNES_OK;
  }
  const int64_t ctas = grad_ctas(rows, dim, op_num_sms(device));
  if (a.sums) {
    OP_TRY(op_on_device(op, "workspace", workspace, device));
    OP_TRY(op_aligned(op, "workspace", workspace, 256));
    if (workspace_bytes < ctas * a.sums * dim * 4)
      return op_error(AGNES_EINVAL, "%s: a workspace of %lld bytes, %lld are needed", op,
                      (long long)workspace_bytes, (long long)(ctas * a.sums * dim * 4));
  }
  a.partial = (float*)workspace;
  set_shape(a, short_shape(dim));
  const int64_t x_size = float_size(x_dtype), branch_size = float_size(branch_dtype);
  const bool wide = wide_inputs(a, x_size, branch_size) &&
                    Wide(a)
                        .rows(before ? d_next : nullptr, d_next_stride, branch_size)
                        .rows(d_sum, d_sum_stride, x_size)
                        .rows(dx, dx_stride, x_size)
                        .rows(branch ? dbranch : nullptr, dbranch_stride, branch_size)
                        .rows(gate_kind == AGNES_GATE_ROWS ? dgate : nullptr, dgate_stride,
                              branch_size)
                        .ok();
  const auto one_run = [&](const void* p, int64_t stride) {
    return !p || rows == 1 || stride == dim;
  };
  const bool contiguous =
      one_run(sum, sum_stride) && one_run(branch, branch_stride) && one_run(d_sum, d_sum_stride) &&
      one_run(before ? d_next : nullptr, d_next_stride) && one_run(dx, dx_stride) &&
      one_run(branch ? dbranch : nullptr, dbranch_stride) &&
      (gate_kind != AGNES_GATE_ROWS || (one_run(gate, gate_stride) && one_run(dgate, dgate_stride)));
  const bool biases = dbefore_bias || dafter_bias, shared = a.lanes > 512;
  // the sums; or the vectors, and in their place a group's share of a sum at the end
  const size_t smem = shared ? (size_t)(biases ? kSums : kBeforeBias) * dim_smem(a)
                             : std::max((size_t)kVectors * dim_smem(a),
                                        a.groups > 1 ? (size_t)a.groups * dim * 4 : 0);
  const cudaError_t e = with_norm_types(x_dtype, branch_dtype, [&](auto tx, auto tb) {
    using TX = typename decltype(tx)::type;
    using TBranch = typename decltype(tb)::type;
    return biases ? launch_grad<TX, TBranch, true>(a, wide, contiguous, ctas, smem, device, st)
                  : launch_grad<TX, TBranch, false>(a, wide, contiguous, ctas, smem, device, st);
  });
  OP_TRY(op_launched(op, e));
  if (!a.sums) return AGNES_OK;
  join.partial = a.partial;
  join.parts = (int32_t)ctas;
  join.sums = a.sums;
  join.dim = (int32_t)dim;
  return op_launched(op, launch_next(norm_join_kernel,
                                     dim3((unsigned)ceil_div(dim, 32), (unsigned)a.sums),
                                     32 * kJoinShares, 0, st, join));
}

}  // extern "C"
