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
#include "int8.cuh"

namespace agnes {

namespace {

constexpr int kElems = 8;  // of a row to a thread
constexpr int64_t kNormMaxDim = (int64_t)kRowLanesMax * kElems;
constexpr int64_t kNormMaxRows = 0x7fffffff - 2047;
constexpr int kSums = 5;  // before, before_bias, after, after_bias, gate

struct NormArgs {
  int64_t rows;
  int32_t dim, lanes, groups;
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
  // backward
  const void *d_next, *d_sum;
  int64_t d_next_stride, d_sum_stride;
  void *dx, *dbranch, *dgate;
  int64_t dx_stride, dbranch_stride, dgate_stride;
  float* partial;      // [CTAs][sums][dim]
  int32_t slot[kSums];  // a sum's place among them, or -1
  int32_t sums;
};

struct RowStats {
  float mean, inv;
};

template <int kVec, int kPer>
struct NormRow {
  static constexpr int kN = kVec * kPer;
  RowPart<kVec, kPer> part;
  RowScratch* scratch;
  int turn = 0;

  template <int kCount>
  __device__ void sum(float (&v)[kCount]) {
    group_reduce<SumOp>(v, part.lanes, scratch, turn);
  }

  // v becomes N(v); zeros past the row's end
  __device__ RowStats standard(float (&v)[kN], bool layer, float eps, float inv_dim) {
    RowStats r = {0.f, 0.f};
    if (layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < kN; ++e) s[0] += v[e];
      sum(s);
      r.mean = s[0] * inv_dim;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[i * kVec + e] = part.has(i) ? v[i * kVec + e] - r.mean : 0.f;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < kN; ++e) s[0] = fmaf(v[e], v[e], s[0]);
    sum(s);
    r.inv = 1.f / sqrtf(fmaf(s[0], inv_dim, eps));
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] *= r.inv;
    return r;
  }

  // A vector over the columns; `fill` where there is none.
  __device__ void vector(const float* p, float fill, float (&v)[kN]) const {
    if (p) {
      part.load(p, true, v);
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e) v[e] = fill;
    }
  }

  // the gradient to v of the gradient d to n = N(v)
  __device__ void through(float (&d)[kN], const float (&n)[kN], bool layer, float inv,
                          float inv_dim) {
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      s[0] = fmaf(d[e], n[e], s[0]);
      s[1] += d[e];
    }
    sum(s);
    const float along = s[0] * inv_dim, mean = layer ? s[1] * inv_dim : 0.f;
#pragma unroll
    for (int e = 0; e < kN; ++e) d[e] = (d[e] - mean - n[e] * along) * inv;
  }
};

// A row times a gate's values, as gate_kind has them.
template <typename TBranch, int kVec, int kPer>
__device__ __forceinline__ void load_gate(const NormRow<kVec, kPer>& r, const NormArgs& a,
                                          int64_t row, bool valid, float (&g)[kVec * kPer]) {
  if (a.gate_kind == AGNES_GATE_ROWS)
    r.part.load((const TBranch*)a.gate + row * a.gate_stride, valid, g);
  else
    r.vector(a.gate_kind == AGNES_GATE_COLUMNS ? (const float*)a.gate : nullptr, 1.f, g);
}

template <typename TX, typename TBranch, int kVec, int kPer>
__global__ void __launch_bounds__(kRowLanesMax)
norm_kernel(const NormArgs a) {
  constexpr int kN = kVec * kPer;
  __shared__ RowScratch scratch;
  const int group = threadIdx.x / a.lanes, lane = threadIdx.x - group * a.lanes;
  NormRow<kVec, kPer> r = {{a.lanes, lane, a.dim}, &scratch};
  const int64_t row = (int64_t)blockIdx.x * a.groups + group;
  const bool valid = row < a.rows;
  float x[kN];
  r.part.load((const TX*)a.x + row * a.x_stride, valid, x);
  if (a.branch) {
    float u[kN], w[kN];
    r.part.load((const TBranch*)a.branch + row * a.branch_stride, valid, u);
    if (a.after) {
      r.standard(u, a.layer, a.eps, a.inv_dim);
      r.vector(a.after, 1.f, w);
#pragma unroll
      for (int e = 0; e < kN; ++e) u[e] *= w[e];
      if (a.after_bias) {
        r.vector(a.after_bias, 0.f, w);
#pragma unroll
        for (int e = 0; e < kN; ++e) u[e] += w[e];
      }
    }
    if (a.gate_kind != AGNES_GATE_NONE) {
      load_gate<TBranch>(r, a, row, valid, w);
#pragma unroll
      for (int e = 0; e < kN; ++e) u[e] *= w[e];
    }
#pragma unroll
    for (int e = 0; e < kN; ++e) x[e] = to_f32(from_f32<TX>(fmaf(a.scale, u[e], x[e])));
    r.part.store((TX*)a.sum + row * a.sum_stride, valid, x);
  }
  if (!a.next) return;
  float w[kN];
  r.standard(x, a.layer, a.eps, a.inv_dim);
  r.vector(a.before, 1.f, w);
#pragma unroll
  for (int e = 0; e < kN; ++e) x[e] *= w[e];
  if (a.before_bias) {
    r.vector(a.before_bias, 0.f, w);
#pragma unroll
    for (int e = 0; e < kN; ++e) x[e] += w[e];
  }
  if (a.next_rows8) {
    uint32_t top[1] = {0};
#pragma unroll
    for (int e = 0; e < kN; ++e) top[0] = max(top[0], __float_as_uint(x[e]) & 0x7fffffffu);
    group_reduce<MaxBits>(top, a.lanes, &scratch, r.turn);
    const Int8Scale s = int8_scale(top[0]);
    uint8_t* to = (uint8_t*)a.next + row * a.next_stride;
    for (int i = 0; i < kPer; ++i) int8_store(r.part, to, valid, i, x + i * kVec, s);
    int8_store_end(to, a.dim, lane, a.lanes, valid, s);
  } else {
    r.part.store((TBranch*)a.next + row * a.next_stride, valid, x);
  }
}

// kThreads: the most that a CTA has.  A thread's sums stay in registers, of which a CTA of
// 1024 has 64 a thread.
template <typename TX, typename TBranch, int kVec, int kPer, int kThreads>
__global__ void __launch_bounds__(kThreads)
norm_grad_kernel(const NormArgs a) {
  constexpr int kN = kVec * kPer;
  __shared__ RowScratch scratch;
  extern __shared__ float group_sums[];  // [groups][dim], where a CTA has several rows
  const int group = threadIdx.x / a.lanes, lane = threadIdx.x - group * a.lanes;
  NormRow<kVec, kPer> r = {{a.lanes, lane, a.dim}, &scratch};
  float total[kSums][kN];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int e = 0; e < kN; ++e) total[k][e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * a.groups;
  for (int64_t first = (int64_t)blockIdx.x * a.groups; first < a.rows; first += step) {
    const int64_t row = first + group;
    const bool valid = row < a.rows;
    float d[kN], w[kN];
    if (a.d_sum) {
      r.part.load((const TX*)a.d_sum + row * a.d_sum_stride, valid, d);
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e) d[e] = 0.f;
    }
    if (a.before) {
      float n[kN], g[kN];
      r.part.load((const TX*)a.x + row * a.x_stride, valid, n);
      r.part.load((const TBranch*)a.d_next + row * a.d_next_stride, valid, g);
      const RowStats s = r.standard(n, a.layer, a.eps, a.inv_dim);
      r.vector(a.before, 1.f, w);
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        if (valid) {  // where there is no row and eps is 0, n is no number
          total[0][e] = fmaf(g[e], n[e], total[0][e]);
          total[1][e] += g[e];
        }
        g[e] *= w[e];
      }
      r.through(g, n, a.layer, s.inv, a.inv_dim);
#pragma unroll
      for (int e = 0; e < kN; ++e) d[e] += g[e];
    }
    r.part.store((TX*)a.dx + row * a.dx_stride, valid, d);
    if (!a.branch) continue;
    float n[kN], b[kN];
    r.part.load((const TBranch*)a.branch + row * a.branch_stride, valid, n);
    RowStats s = {0.f, 1.f};
    if (a.after) s = r.standard(n, a.layer, a.eps, a.inv_dim);
#pragma unroll
    for (int e = 0; e < kN; ++e) d[e] *= a.scale;
    if (a.gate_kind != AGNES_GATE_NONE) {
      // u, then d u
      r.vector(a.after, 1.f, w);
      r.vector(a.after_bias, 0.f, b);
#pragma unroll
      for (int e = 0; e < kN; ++e) b[e] = d[e] * fmaf(n[e], w[e], b[e]);
      load_gate<TBranch>(r, a, row, valid, w);
      if (a.gate_kind == AGNES_GATE_ROWS) {
        r.part.store((TBranch*)a.dgate + row * a.dgate_stride, valid, b);
      } else if (valid) {
#pragma unroll
        for (int e = 0; e < kN; ++e) total[4][e] += b[e];
      }
#pragma unroll
      for (int e = 0; e < kN; ++e) d[e] *= w[e];
    }
    if (a.after) {
      r.vector(a.after, 1.f, w);
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        if (valid) {
          total[2][e] = fmaf(d[e], n[e], total[2][e]);
          total[3][e] += d[e];
        }
        d[e] *= w[e];
      }
      r.through(d, n, a.layer, s.inv, a.inv_dim);
    }
    r.part.store((TBranch*)a.dbranch + row * a.dbranch_stride, valid, d);
  }
  // a CTA's sums: its groups' added in order
  for (int k = 0; k < kSums; ++k) {
    if (a.slot[k] < 0) continue;
    float* to = a.partial + ((int64_t)blockIdx.x * a.sums + a.slot[k]) * a.dim;
    if (a.groups == 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (r.part.has(i)) to[r.part.col(i) + e] = total[k][i * kVec + e];
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (r.part.has(i)) group_sums[group * a.dim + r.part.col(i) + e] = total[k][i * kVec + e];
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

// A warp to 32 columns of a sum would wait for `parts` loads in a row: eight threads share
// a column's parts, and add theirs up in order.
constexpr int kJoinShares = 8;
__global__ void __launch_bounds__(32 * kJoinShares)
norm_join_kernel(const JoinArgs a) {
  grid_dep_wait();
  __shared__ float part_sum[kJoinShares][32];
  const int lane = threadIdx.x & 31, share = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane, k = blockIdx.y;
  float sum = 0.f;
  if (c < a.dim)
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

void set_shape(NormArgs& a) {
  const RowShape shape = row_shape(a.dim, kElems);
  a.lanes = shape.lanes;
  a.groups = shape.groups;
  a.inv_dim = 1.f / (float)a.dim;
}

// CTAs of the backward pass: each writes a row of partial sums, so no more than keep the
// device busy.
int64_t grad_ctas(int64_t rows, int64_t dim, int sms) {
  const RowShape shape = row_shape(dim, kElems);
  const int64_t ctas = ceil_div(rows, shape.groups);
  const int64_t most = (int64_t)sms * (1024 / shape.threads());
  return ctas < most ? ctas : most;
}
constexpr int kMostSms = 256;  // for the size of a workspace, whatever device it will be on

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
  set_shape(a);
  const bool wide = wide_inputs(a, x_size, branch_size) &&
                    Wide(a)
                        .rows(branch ? sum : nullptr, sum_stride, x_size)
                        .rows(a.next_rows8 ? nullptr : a.next, next_stride, branch_size)
                        .ok();
  return op_launched(op, with_norm_types(x_dtype, branch_dtype, [&](auto tx, auto tb) {
    using TX = typename decltype(tx)::type;
    using TBranch = typename decltype(tb)::type;
    const auto kernel =
        wide ? norm_kernel<TX, TBranch, 8, 1> : norm_kernel<TX, TBranch, 1, kElems>;
    kernel<<<(unsigned)ceil_div(rows, a.groups), (unsigned)(a.lanes * a.groups), 0,
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
  float* const outs[kSums] = {dbefore, dbefore_bias, dafter, dafter_bias,
                              gate_kind == AGNES_GATE_COLUMNS ? (float*)dgate : nullptr};
  const char* const names[kSums] = {"dbefore", "dbefore_bias", "dafter", "dafter_bias", "dgate"};
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
  set_shape(a);
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
  const size_t smem = a.groups > 1 && a.sums ? (size_t)a.groups * dim * 4 : 0;
  const cudaError_t e = with_norm_types(x_dtype, branch_dtype, [&](auto tx, auto tb) {
    using TX = typename decltype(tx)::type;
    using TBranch = typename decltype(tb)::type;
    const auto kernel = a.lanes <= 512 ? (wide ? norm_grad_kernel<TX, TBranch, 8, 1, 512>
                                               : norm_grad_kernel<TX, TBranch, 1, kElems, 512>)
                                       : (wide ? norm_grad_kernel<TX, TBranch, 8, 1, 1024>
                                               : norm_grad_kernel<TX, TBranch, 1, kElems, 1024>);
    kernel<<<(unsigned)ctas, (unsigned)(a.lanes * a.groups), smem, st>>>(a);
    return cudaGetLastError();
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
