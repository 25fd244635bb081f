// int8_linear.cu -- 8-bit rows times 8-bit weights, and the gradient of that product to the
// rows (include/agnes_ops.h; the format is in int8.cuh; the gradient to the weights is in
// int8_grad_weight.cu).
//
//   out[r][j] = s_x[r] s_w[j] sum_i q_x[r][i] q_w[j][i] + bias[j]
//   dx[r][i]  = sum_j grad[r][j] s_w[j] q_w[j][i]
//
// Few rows: the weights' bytes count, so a group of lanes takes a column's whole numbers,
// four products an instruction, for all rows.
// Otherwise the tensor cores (tcgen05.mma), in 16-bit operands: whole numbers are exact in
// fp16, and a scaled one is the sum of two bfloat16 values (int8.cuh).  The weights are laid
// out for them by a kernel before; the rows come as they are.  A persistent CTA, or a pair:
//   the producer      has the TMA copy slices of 64 of the contraction;
//   the convert warps make the rows' whole numbers fp16 (forward);
//   the MMA warp      issues a slice's products into one of two accumulators;
//   the epilogue warps scale the sums, add the bias and hand them to the TMA by way of shared
//                     memory, while the next tile's products run.
// Long rows are bound by the tensor cores (16,384 x 4096 to 4096, bf16: 357 us, 1540 TFLOP/s,
// the tensor pipe 68% active; the gradient of 8192 x 4096 to 2048 170 us, two terms, 74%: its sums
// are drained, undrained it took 151 and 95%), short ones by what they write (786,432 x 128 to 256,
// fp16: 97 us; a memset of the output takes 101).
#include <type_traits>

#include "int8_product.cuh"

namespace agnes {

namespace {

// ---- few rows ------------------------------------------------------------------

// A group of up to 32 lanes has a column, 16 of its whole numbers to a lane at a time, which meet
// all the rows' (from L1: the rows are as often read as there are columns, and bound the larger
// calls).  Columns by twos would halve those reads, and the groups as well: 4 x 1024 to 1024 took
// 4.1 us so and takes 3.1.  Times by rows against those of the tiles below, fp16:
// 128 to 256     1.9 us (1 row), 2.3 (4), 3.1 (8), 6.7 (16)     7.3
// 1024 to 4096   3.0, 4.3, 5.9, 11.3                           15.1
// 4096 to 4096   4.2, 6.9, 10.4, 20.0                          38.7
// of which the weights' bytes are 0.01, 0.6 and 2.5.  With 32 rows they are 8.4, 26.6 and 46.7
// against 7.2, 15.2 and 38.8, so tiles have those.
constexpr int kFewRows = 16;
constexpr int kFewThreads = 256;

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
__global__ void __launch_bounds__(kFewThreads, kRows > 8 ? 1 : 4)
linear_few_kernel(int lanes, const LinearArgs a) {
  const int lane = threadIdx.x % lanes;
  const int64_t groups = (int64_t)gridDim.x * (kFewThreads / lanes);
  const int chunks = (a.dim + 15) / 16;
  for (int64_t j = (int64_t)blockIdx.x * (kFewThreads / lanes) + threadIdx.x / lanes;
       // whole warps stay together for the exchange
       j - (threadIdx.x % 32) / lanes < a.width; j += groups) {
    const uint8_t* w_row = a.w + (j < a.width ? j : a.width - 1) * a.w_stride;
    int32_t sum[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) sum[r] = 0;
#pragma unroll 1
    for (int c = lane; c < chunks; c += lanes) {
      uint4 w = __ldg((const uint4*)w_row + c);
      if (c == chunks - 1) {  // the row's scale may be in its last 16 bytes
        const int left = a.dim - c * 16;
        const auto mask = [&](int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; };
        w = make_uint4(w.x & mask(left), w.y & mask(left - 4), w.z & mask(left - 8),
                       w.w & mask(left - 12));
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        // past the end the last row again: all rows' loads are on their way together
        const uint4 x = __ldg((const uint4*)(a.x + (r < a.rows ? r : a.rows - 1) * a.x_stride) + c);
        int32_t s = __dp4a((int)x.x, (int)w.x, sum[r]);
        s = __dp4a((int)x.y, (int)w.y, s);
        s = __dp4a((int)x.z, (int)w.z, s);
        sum[r] = __dp4a((int)x.w, (int)w.w, s);
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      for (int d = lanes / 2; d > 0; d >>= 1) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], d);
    if (j >= a.width) continue;
    const float sw = *(const float*)(w_row + a.row_bytes - 4);
    const float b = a.bias ? __ldg(a.bias + j) : 0.f;
    for (int r0 = 0; r0 < a.rows; r0 += lanes) {  // a row to a lane
      int32_t mine = 0;
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (r == r0 + lane) mine = sum[r];
      const int r = r0 + lane;
      if (r >= a.rows) break;
      const float sx = *(const float*)(a.x + r * a.x_stride + a.row_bytes - 4);
      ((TOut*)a.out)[r * a.out_stride + j] = from_f32<TOut>(scaled((float)mine, sx, sw) + b);
    }
  }
}

// ---- operands in 16 bits --------------------------------------------------------

constexpr int kPrepThreads = 256;

// Whole numbers as fp16, `kpad` to a row, and the rows' scales.
__global__ void __launch_bounds__(kPrepThreads)
expand_kernel(const uint8_t* __restrict__ q, int64_t stride, int64_t rows, int32_t dim,
              int32_t row_bytes, int32_t groups, uint32_t inv_groups, __half* __restrict__ out,
              int64_t kpad, float* __restrict__ scales) {
  const FlatRows flat(blockIdx.x, groups, inv_groups);
#pragma unroll
  for (int u = 0; u < kFlat / kPrepThreads; ++u) {
    int64_t row;
    uint32_t g;
    flat.at(threadIdx.x + u * kPrepThreads, &row, &g);
    if (row >= rows) continue;
    const uint8_t* from = q + row * stride;
    float v[8];
    const uint2 w = *(const uint2*)(from + g * 8);
    int8_values4(w.x, v);
    int8_values4(w.y, v + 4);
    store_vec<__half, 8>(out + row * kpad + g * 8, v);  // past dim: not looked at
    if (scales && g == 0) scales[row] = *(const float*)(from + row_bytes - 4);
  }
}

// The weights' values, transposed and as sums of two bfloat16 values: term t of column i of
// row j at out[(t * dim + i) * wpad + j].
constexpr int kTransTile = 64;
struct TransposeArgs {
  const uint8_t* q;
  int64_t stride, width;
  int32_t dim, row_bytes;
  __nv_bfloat16* out;
  int64_t wpad;
  int32_t tiles_i;
};
__device__ __forceinline__ void transpose_tile(const TransposeArgs& a, int64_t block) {
  const uint8_t* q = a.q;
  const int64_t stride = a.stride, width = a.width, wpad = a.wpad;
  const int32_t dim = a.dim, row_bytes = a.row_bytes;
  __nv_bfloat16* out = a.out;
  __shared__ __align__(16) uint8_t tile[kTransTile][kTransTile + 16];
  __shared__ float scale[kTransTile];
  const int64_t j0 = block / a.tiles_i * kTransTile;
  const int32_t i0 = (int32_t)(block % a.tiles_i) * kTransTile;
  {
    const int j = threadIdx.x / 4, c = threadIdx.x % 4 * 16;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (j0 + j < width && i0 + c < row_bytes) v = *(const uint4*)(q + (j0 + j) * stride + i0 + c);
    *(uint4*)&tile[j][c] = v;
    if (c == 0) scale[j] = j0 + j < width ? *(const float*)(q + (j0 + j) * stride + row_bytes - 4) : 0.f;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = threadIdx.x / 4, j = (threadIdx.x % 4 * 2 + u) * 8;
    if (i0 + i >= dim || j0 + j >= wpad) continue;
    float hi[8], lo[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) int8_split((float)(int8_t)tile[j + e][i] * scale[j + e], hi[e], lo[e]);
    __nv_bfloat16* to = out + (int64_t)(i0 + i) * wpad + j0 + j;
    store_vec<__nv_bfloat16, 8>(to, hi);
    store_vec<__nv_bfloat16, 8>(to + (int64_t)dim * wpad, lo);
  }
}

// Eight values of a row to a thread; see split_grad.  kWide: rows that are 16-byte aligned and
// whole eights.
struct SplitArgs {
  const void* x;
  int64_t stride, rows, width;
  int32_t groups;
  uint32_t inv_groups;
  __nv_bfloat16* out;
  int64_t wpad;
};
template <typename T, bool kWide>
__device__ __forceinline__ void split_rows(const SplitArgs& a, int64_t block) {
  const T* x = (const T*)a.x;
  const int64_t stride = a.stride, rows = a.rows, width = a.width, wpad = a.wpad;
  __nv_bfloat16* out = a.out;
  const FlatRows flat(block, a.groups, a.inv_groups);
#pragma unroll
  for (int u = 0; u < kFlat / kPrepThreads; ++u) {
    int64_t row;
    uint32_t g;
    flat.at(threadIdx.x + u * kPrepThreads, &row, &g);
    if (row >= rows) continue;
    const T* from = x + row * stride + g * 8;
    float v[8], rest[8];
    if constexpr (kWide) {
      load_vec<T, 8>(from, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (int64_t)g * 8 + e < width ? to_f32(from[e]) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) int8_split(v[e], v[e], rest[e]);
    __nv_bfloat16* to = out + row * wpad + g * 8;
    store_vec<__nv_bfloat16, 8>(to, v);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) continue;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 8; ++e) int8_split(rest[e], rest[e], v[e]);
      store_vec<__nv_bfloat16, 8>(to + 2 * rows * wpad, v);
    }
    store_vec<__nv_bfloat16, 8>(to + rows * wpad, rest);
  }
}

// The operands of the backward pass in one launch: the first `transposes` CTAs have the
// weights, the others the gradient.
template <typename T, bool kWide>
__global__ void __launch_bounds__(kPrepThreads)
prepare_kernel(const TransposeArgs w, int64_t transposes, const SplitArgs g) {
  if ((int64_t)blockIdx.x < transposes)
    transpose_tile(w, blockIdx.x);
  else
    split_rows<T, kWide>(g, (int64_t)blockIdx.x - transposes);
}

// The weights where t.q is set; the gradient of `dtype` where g.x is.
cudaError_t prepare_operands(TransposeArgs t, SplitArgs g, int32_t dtype, cudaStream_t st) {
  int64_t transposes = 0, splits = 0;
  if (t.q) {
    t.tiles_i = (int32_t)ceil_div(t.dim, kTransTile);
    transposes = ceil_div(t.width, kTransTile) * t.tiles_i;
  }
  if (g.x) {
    g.groups = (int32_t)(g.wpad / 8);
    g.inv_groups = flat_inverse(g.groups);
    splits = ceil_div(g.rows * g.groups, kFlat);
  }
  return with_float_type(dtype, [&](auto tag) {
    using T = typename decltype(tag)::type;
    const bool wide = g.width % 8 == 0 && aligned_rows(g.x, g.stride * (int64_t)sizeof(T), 16);
    (wide ? prepare_kernel<T, true> : prepare_kernel<T, false>)
        <<<(unsigned)(transposes + splits), kPrepThreads, 0, st>>>(t, transposes, g);
    return cudaGetLastError();
  });
}

// ---- tiles ----------------------------------------------------------------------

// Warps: 0-7 epilogue (two to a quarter of tensor memory's lanes, half the columns each),
// 8-11 whole numbers to fp16, 12 producer, 13 MMA.
constexpr int kTileM = 128;
constexpr int kSliceK = 64;  // of the contraction to a stage: 128 bytes in 16 bits
constexpr int kEpilogueWarps = 8;
constexpr int kConvertWarp0 = kEpilogueWarps, kConvertWarps = 4;
constexpr int kProducerWarp = kConvertWarp0 + kConvertWarps;
constexpr int kMmaWarp = kProducerWarp + 1;
constexpr int kTileThreads = 32 * (kMmaWarp + 1);
constexpr int kOperandBytes = kTileM * 128;  // of one term of A
constexpr int kRawBytes = kTileM * kSliceK;
constexpr int kMaxSlots = 8;
constexpr int kOutBytes = 32 * 128;  // an epilogue warp's output on its way to memory
constexpr int kColumnBytes = kEpilogueWarps * 2 * 128 * 4;  // the epilogue warps' scales and biases
constexpr int kTileBars = 3 * kMaxSlots + 6;
constexpr int kSmemLimit = 232448;
// Shared memory beside those (of kConvert alone) and the mbarriers.
constexpr int tile_smem(bool convert) {
  return kSmemLimit - 1024 - (convert ? kColumnBytes : 0) - 8 * kTileBars - 16;
}

struct TileArgs {
  int64_t rows, cols;  // of the output
  int32_t steps;       // slices of the contraction
  int32_t last;        // products of 16 in the last one
  int32_t ta, tb;      // terms of A and of B
  int32_t chain;       // slices that one accumulator sums
  const uint8_t* x;    // rows whose scales the output takes, or null
  int64_t x_stride;
  int32_t row_bytes;
  const float *col_scale, *bias;
  void* out;
  int64_t out_stride;
  int32_t slots, slot_bytes, out_buffers;
  bool resident;  // B's slices stay in shared memory: a CTA keeps to one tile of columns
  bool tma_out;
  int32_t* status;
};

// The output tiles of a CTA (or of a pair, kGroup = 2), every one of as many as there are
// CTAs, columns fastest.
template <int kGroup>
struct TileWalk {
  int64_t m, n, tiles_m, tiles_n, step_m, step_n;
  __device__ TileWalk(const TileArgs& a, int cols) {
    const uint32_t at = blockIdx.x / kGroup, count = gridDim.x / kGroup;
    tiles_n = (a.cols + cols - 1) / cols;
    tiles_m = (a.rows + kGroup * kTileM - 1) / (kGroup * kTileM);
    m = at / tiles_n;
    n = at - m * tiles_n;
    step_m = count / tiles_n;
    step_n = count - step_m * tiles_n;
  }
  __device__ bool any() const { return m < tiles_m; }
  __device__ void next() {
    m += step_m;
    n += step_n;
    if (n >= tiles_n) {
      n -= tiles_n;
      ++m;
    }
  }
};

// The mbarriers: full[s] (the TMA has brought slot s), ready[s] (A's whole numbers are fp16),
// empty[s] (its products are done); done[d] / taken[d] of the accumulators; b_full of the
// resident B; drained, when the MMA warp gives up.
struct TileBars {
  uint32_t base;
  __device__ uint32_t at(int i) const { return base + 8u * (uint32_t)i; }
  __device__ uint32_t full(int s) const { return at(s); }
  __device__ uint32_t ready(int s) const { return at(kMaxSlots + s); }
  __device__ uint32_t empty(int s) const { return at(2 * kMaxSlots + s); }
  __device__ uint32_t done(int d) const { return at(3 * kMaxSlots + d); }
  __device__ uint32_t taken(int d) const { return at(3 * kMaxSlots + 2 + d); }
  __device__ uint32_t b_full() const { return at(3 * kMaxSlots + 4); }
  __device__ uint32_t drained() const { return at(3 * kMaxSlots + 5); }
};

// A warp's columns of a vector, kHalf / 32 to a lane, from c0 on; zeros past its end or where
// there is none.
template <int kHalf>
struct Columns {
  float v[kHalf / 32];
  __device__ void load(const float* p, int64_t c0, int64_t cols, bool any) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kHalf / 32; ++i) {
      const int64_t c = c0 + i * 32 + lane;
      v[i] = p && any && c < cols ? __ldg(p + c) : 0.f;
    }
  }
  __device__ void put(float* to) const {
#pragma unroll
    for (int i = 0; i < kHalf / 32; ++i) to[i * 32 + (threadIdx.x & 31)] = v[i];
  }
};

// 32 columns of a lane's row into its warp's buffer, from byte `first` of its 128 on, in
// 16-byte pieces permuted as the TMA's 128-byte swizzle has them.
template <typename TOut>
__device__ __forceinline__ void stage_values(uint8_t* buffer, int lane, int first,
                                             const float (&v)[32]) {
  constexpr int kN = 16 / sizeof(TOut);
#pragma unroll
  for (int q = 0; q < 32 / kN; ++q) {
    Vec<TOut, kN> y;
#pragma unroll
    for (int e = 0; e < kN; ++e) y.v[e] = from_f32<TOut>(v[q * kN + e]);
    *(Vec<TOut, kN>*)(buffer + lane * 128 + (((first / 16 + q) ^ (lane & 7)) << 4)) = y;
  }
}

// Four whole numbers as two pairs of fp16, in order: 1024 + (q + 128) are the bytes of the
// word xor 0x80, each under 0x64.
__device__ __forceinline__ uint2 int8_halves4(uint32_t word) {
  word ^= 0x80808080u;
  const uint32_t low = __byte_perm(word, 0x64646464u, 0x4140);
  const uint32_t high = __byte_perm(word, 0x64646464u, 0x4342);
  const __half2 offset = __half2half2(__ushort_as_half(0x6480));  // 1152
  const __half2 a = __hsub2(*(const __half2*)&low, offset);
  const __half2 b = __hsub2(*(const __half2*)&high, offset);
  return make_uint2(*(const uint32_t*)&a, *(const uint32_t*)&b);
}

// A slice's products, n of 16 for each two terms but the third with the second.  The thread
// that issues them has one at a time to prepare, so their descriptors are sums of constants
// (looked up term by term a product took some 250 cycles to issue, twice its own time).
template <int kTermsA, int kTermsB, int kBRows, bool kPair>
__device__ __forceinline__ void slice_products(uint32_t to, uint32_t a_at, uint32_t b_at, int n,
                                               uint32_t idesc, uint32_t accumulate) {
  const uint64_t a0 = operand_desc(a_at), b0 = operand_desc(b_at);
#pragma unroll
  for (int i = 0; i < kSliceK / 16; ++i) {
    if (i >= n) break;
#pragma unroll
    for (int p = 0; p < kTermsA; ++p)
#pragma unroll
      for (int q = 0; q < kTermsB; ++q) {
        if (p + q >= 3) continue;
        const uint64_t a = a0 + (uint64_t)(p * (kOperandBytes >> 4) + 2 * i);
        const uint64_t b = b0 + (uint64_t)(q * (kBRows * 128 >> 4) + 2 * i);
        const uint32_t more = accumulate | (uint32_t)(i + p + q > 0);
        if constexpr (kPair)
          mma_16bit_pair(to, a, b, idesc, more);
        else
          mma_16bit(to, a, b, idesc, more);
      }
  }
}

// out = A B^T over tiles of 128 x kCols.  kConvert: A is 8-bit rows, brought as they are and
// made fp16 in shared memory, and B fp16; else both are bfloat16, of several terms each.
// kDrain: an accumulator sums `chain` slices, and the epilogue warps add those up in
// registers: tensor memory's sums are cut off, not rounded, after each product, which adds
// up over long chains.  (With kConvert 8 bytes a thread are spilled, some 26 for fp32 results.)
// kPair: two CTAs have a tile of 256 x kCols, each the rows and the output of its half and half
// of B, so that B is copied and read once for both.
template <typename TOut, bool kConvert, int kCols, bool kDrain, bool kPair>
__global__ void __launch_bounds__(kTileThreads, 1)
tile_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
            const __grid_constant__ CUtensorMap out_map, const TileArgs a) {
  grid_dep_wait();
  constexpr int kHalf = kCols / 2;  // columns of an epilogue warp
  constexpr int kTmemCols = 2 * kCols;
  constexpr uint32_t kIdesc = idesc_16bit(!kConvert, false, kPair ? 2 * kTileM : kTileM, kCols);
  constexpr int kBRows = kPair ? kCols / 2 : kCols;  // of B in this CTA
  constexpr uint32_t kBBytes = kBRows * 128;
  const uint32_t rank = kPair ? cluster_rank() : 0;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  uint8_t* resident_b = smem + a.slots * a.slot_bytes;
  uint8_t* out_stage =
      resident_b + (a.resident ? a.steps * a.tb * (int)kBBytes : 0);
  float* column_stage = (float*)(out_stage + kEpilogueWarps * a.out_buffers * kOutBytes);
  uint64_t* bars = (uint64_t*)((uint8_t*)column_stage + (kConvert ? kColumnBytes : 0));
  uint32_t* tmem_slot = (uint32_t*)(bars + kTileBars);
  const TileBars bar = {smem_addr(bars)};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == kMmaWarp) {
    if constexpr (kPair)
      tmem_alloc_pair(tmem_slot, kTmemCols);
    else
      tmem_alloc(tmem_slot, kTmemCols);
  }
  if (tid == 0) {
    constexpr int kBoth = kPair ? 2 : 1;  // a pair's first CTA is told by the warps of both
    for (int s = 0; s < kMaxSlots; ++s) {
      mbar_init(bar.full(s), 1);
      mbar_init(bar.ready(s), (kConvert ? kConvertWarps : 1) * kBoth);
      mbar_init(bar.empty(s), 1);
    }
    for (int d = 0; d < 2; ++d) {
      mbar_init(bar.done(d), 1);
      mbar_init(bar.taken(d), kEpilogueWarps * kBoth);
    }
    mbar_init(bar.b_full(), 1);
    mbar_init(bar.drained(), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tcgen05_fence_before();
  __syncthreads();
  if constexpr (kPair) cluster_sync();  // the other CTA's barriers are there
  tcgen05_fence_after();
  const uint32_t tmem = *tmem_slot;
  // for the thread that issues the products: of this CTA, or of the pair's first
  const auto tell = [&](uint32_t b) {
    if constexpr (kPair)
      mbar_arrive_at(b, 0);
    else
      mbar_arrive(b);
  };
  using Walk = TileWalk<kPair ? 2 : 1>;
  Walk t(a, kCols);
  const auto first_row = [&](const Walk& at) {
    return kPair ? (at.m * 2 + rank) * kTileM : at.m * kTileM;
  };
  const int slots = a.slots;
  const uint32_t ring_at = smem_addr(smem), resident_at = smem_addr(resident_b);
  // in a slot: A's terms, B's (unless they are resident), A's raw bytes
  const uint32_t b_off = (uint32_t)(a.ta * kOperandBytes);
  const uint32_t raw_off = b_off + (a.resident ? 0u : (uint32_t)a.tb * kBBytes);
  bool ok = true;

  if (warp == kProducerWarp) {
    if (lane == 0) {
      if (a.resident) {
        mbar_expect(bar.b_full(), (uint32_t)(a.steps * a.tb) * kBBytes);
        for (int k = 0; k < a.steps; ++k)
          for (int b = 0; b < a.tb; ++b)
            tma_load(resident_at + (uint32_t)(k * a.tb + b) * kBBytes, &b_map, k * kSliceK,
                     (int32_t)(b * a.cols + t.n * kCols + rank * kBRows), bar.b_full());
      }
      const uint32_t bytes = (kConvert ? (uint32_t)kRawBytes : b_off) +
                             (a.resident ? 0u : (uint32_t)a.tb * kBBytes);
      Ring ring;
      int64_t issued = 0;
      for (; ok && t.any(); t.next()) {
        for (int k = 0; k < a.steps; ++k) {
          const int s = ring.slot;
          if (!ring.first && !mbar_wait(bar.empty(s), ring.parity ^ 1u)) {
            ok = false;
            break;
          }
          const uint32_t at = ring_at + (uint32_t)(s * a.slot_bytes);
          mbar_expect(bar.full(s), bytes);
          if constexpr (kConvert) {
            tma_load(at + raw_off, &a_map, k * kSliceK, (int32_t)first_row(t), bar.full(s));
          } else {
            for (int i = 0; i < a.ta; ++i)
              tma_load(at + (uint32_t)(i * kOperandBytes), &a_map, k * kSliceK,
                       (int32_t)(i * a.rows + first_row(t)), bar.full(s));
          }
          if (!a.resident)
            for (int i = 0; i < a.tb; ++i)
              tma_load(at + b_off + (uint32_t)i * kBBytes, &b_map, k * kSliceK,
                       (int32_t)(i * a.cols + t.n * kCols + rank * kBRows), bar.full(s));
          ring.next(slots);
          ++issued;
        }
      }
      if (kPair && ok) {  // the other CTA's last arrivals here land before this one may leave
        for (int s = 0; ok && s < slots; ++s) {
          ok = ring.first || mbar_wait(bar.empty(ring.slot), ring.parity ^ 1u);
          ring.next(slots);
        }
      }
      if (!ok) {  // the copies in flight land before the CTA may leave
        if (a.resident) mbar_wait(bar.b_full(), 0);
        Ring r;
        for (int64_t i = 0; i < issued; ++i, r.next(slots))
          if (i + slots >= issued) mbar_wait(bar.full(r.slot), r.parity);
      }
    }
  } else if (warp == kMmaWarp) {
    // the whole warp goes through the loop, so that its addresses are the same for all lanes and
    // stay in uniform registers, as the products take them
    if (rank == 0) {
      const bool lead = elect_one();
      const auto commit = [](uint32_t b) {
        if constexpr (kPair)
          mma_commit_pair(b);
        else
          mma_commit(b);
      };
      if (a.resident) ok = __all_sync(0xffffffffu, mbar_wait(bar.b_full(), 0));
      Ring ring, acc;
      for (; ok && t.any(); t.next()) {
        for (int k0 = 0; ok && k0 < a.steps; k0 += a.chain) {
          const int d = acc.slot;
          if (!acc.first && !__all_sync(0xffffffffu, mbar_wait(bar.taken(d), acc.parity ^ 1u))) {
            ok = false;
            break;
          }
          tcgen05_fence_after();
          const uint32_t to = tmem + (uint32_t)(d * kCols);
          uint32_t accumulate = 0;
          const int k1 = min(k0 + a.chain, a.steps);
          for (int k = k0; k < k1; ++k) {
            const int s = ring.slot;
            // what is ready is full as well
            const uint32_t b = kConvert || kPair ? bar.ready(s) : bar.full(s);
            if (!__all_sync(0xffffffffu, mbar_wait(b, ring.parity))) {
              ok = false;
              break;
            }
            tcgen05_fence_after();
            const uint32_t a_at = ring_at + (uint32_t)(s * a.slot_bytes);
            const uint32_t b_at =
                a.resident ? resident_at + (uint32_t)(k * a.tb) * kBBytes : a_at + b_off;
            const int n = k + 1 == a.steps ? a.last : kSliceK / 16;
            if (lead) {
              if (kConvert)
                slice_products<1, 1, kBRows, kPair>(to, a_at, b_at, n, kIdesc, accumulate);
              else if (a.ta == 1)
                slice_products<1, 2, kBRows, kPair>(to, a_at, b_at, n, kIdesc, accumulate);
              else if (a.ta == 2)
                slice_products<2, 2, kBRows, kPair>(to, a_at, b_at, n, kIdesc, accumulate);
              else
                slice_products<3, 2, kBRows, kPair>(to, a_at, b_at, n, kIdesc, accumulate);
              commit(bar.empty(s));
            }
            __syncwarp();
            accumulate = 1;
            ring.next(slots);
          }
          if (!ok) break;
          if (lead) commit(bar.done(d));
          __syncwarp();
          acc.next(2);
        }
      }
      if (!ok) {  // the products in flight end before the tensor memory is freed
        if (lead) commit(bar.drained());
        mbar_wait(bar.drained(), 0);
      }
    }
  } else if (warp >= kConvertWarp0) {
    if constexpr (!kConvert && kPair) {
      // one warp tells the pair's first CTA of this one's slices
      if (warp == kConvertWarp0) {
        Ring ring;
        for (; ok && t.any(); t.next()) {
          for (int k = 0; k < a.steps; ++k) {
            if (!__all_sync(0xffffffffu, mbar_wait(bar.full(ring.slot), ring.parity))) {
              ok = false;
              break;
            }
            if (lane == 0) tell(bar.ready(ring.slot));
            ring.next(slots);
          }
        }
      }
    }
    if constexpr (kConvert) {
      const int r = tid - 32 * kConvertWarp0;  // this thread's row of the tile
      Ring ring;
      for (; ok && t.any(); t.next()) {
        for (int k = 0; k < a.steps; ++k) {
          const int s = ring.slot;
          if (!__all_sync(0xffffffffu, mbar_wait(bar.full(s), ring.parity))) {
            ok = false;
            break;
          }
          uint8_t* slot = smem + s * a.slot_bytes;
          const uint8_t* from = slot + raw_off + r * kSliceK;
          uint4 v[4];
#pragma unroll
          for (int c = 0; c < 4; ++c)  // the TMA's 64-byte swizzle
            v[c] = *(const uint4*)(from + ((c ^ ((r >> 1) & 3)) << 4));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint2 p0 = int8_halves4(v[c].x), p1 = int8_halves4(v[c].y);
            const uint2 p2 = int8_halves4(v[c].z), p3 = int8_halves4(v[c].w);
            *(uint4*)(slot + r * 128 + (((2 * c) ^ (r & 7)) << 4)) =
                make_uint4(p0.x, p0.y, p1.x, p1.y);
            *(uint4*)(slot + r * 128 + (((2 * c + 1) ^ (r & 7)) << 4)) =
                make_uint4(p2.x, p2.y, p3.x, p3.y);
          }
          fence_async_proxy();
          __syncwarp();
          if (lane == 0) tell(bar.ready(s));
          ring.next(slots);
        }
      }
    }
  } else {
    constexpr int kGroup = 128 / sizeof(TOut);  // columns of a staged buffer
    uint8_t* mine = out_stage + warp * a.out_buffers * kOutBytes;
    int buffer = 0;
    Ring acc;
    // a tile ahead, as it is some trip away
    const auto scale_of = [&](const Walk& at) {
      const int64_t row = first_row(at) + (warp & 3) * 32 + lane;
      return kConvert && at.any() && row < a.rows
                 ? __ldg((const float*)(a.x + row * a.x_stride + a.row_bytes - 4)) : 1.f;
    };
    float next_scale = scale_of(t);
    // the columns' scales and biases, too, on their way to shared memory
    float* my_scales = column_stage + warp * 256;
    float* my_biases = my_scales + 128;
    Columns<kHalf> next_scales, next_biases;
    const auto columns_of = [&](const Walk& at) {
      if constexpr (kConvert) {
        const int64_t c0 = at.n * kCols + (warp >> 2) * kHalf;
        next_scales.load(a.col_scale, c0, a.cols, at.any());
        next_biases.load(a.bias, c0, a.cols, at.any());
      }
    };
    columns_of(t);
    for (; ok && t.any(); t.next()) {
      const float scale = next_scale;
      if constexpr (kConvert) {
        __syncwarp();
        next_scales.put(my_scales);
        next_biases.put(my_biases);
        __syncwarp();
      }
      Walk after = t;
      after.next();
      next_scale = scale_of(after);
      columns_of(after);
      const int64_t row0 = first_row(t) + (warp & 3) * 32;
      const int64_t n0 = t.n * kCols + (warp >> 2) * kHalf;
      // a warp whose rows are all past the end has nothing to store, and its buffers may
      // still be on their way
      const int cols = row0 < a.rows ? kHalf : 0;
      const uint32_t lanes_at = tmem + ((uint32_t)((warp & 3) * 32) << 16) +
                                (uint32_t)((warp >> 2) * kHalf);
      // A sum (up to 2^31) times a row's scale between 2^-90 and 2^90 does not leave fp32 unless
      // the whole product does.  Another scale is taken in two, its power of two last: that
      // costs a product more for each value, where a branch between the two took 18 us more of
      // 786,432 x 128 to 256 and a choice for each value 45.
      const float far = scale > 0x1p90f ? 0x1p60f : scale < 0x1p-90f ? 0x1p-60f : 1.f;
      const float near = scale > 0x1p90f ? scale * 0x1p-60f : scale < 0x1p-90f ? scale * 0x1p60f
                                                                               : scale;
      float total[kDrain ? kHalf : 1];
      if constexpr (kDrain) {
#pragma unroll
        for (int e = 0; e < kHalf; ++e) total[e] = 0.f;
      }
      uint32_t from = 0;
      for (int k0 = 0; k0 < a.steps; k0 += a.chain) {
        const int d = acc.slot;
        if (!__all_sync(0xffffffffu, mbar_wait(bar.done(d), acc.parity))) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        from = lanes_at + (uint32_t)(d * kCols);
        if constexpr (kDrain) {
#pragma unroll
          for (int c = 0; c < kHalf; c += 32) {
            uint32_t v[32];
            tmem_load32(from + (uint32_t)c, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) total[c + e] += __uint_as_float(v[e]);
          }
          tcgen05_fence_before();
          __syncwarp();
          if (lane == 0) tell(bar.taken(d));
        }
        acc.next(2);
      }
      if (!ok) break;
#pragma unroll(kDrain ? kHalf / kGroup : 1)
      for (int c = 0; c < kHalf; c += kGroup) {
        if (c >= cols || n0 + c >= a.cols) break;
        // an earlier store has read the buffer
        if (lane == 0) {
          if (a.out_buffers == 2)
            asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          else
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        }
        __syncwarp();
        uint8_t* to = mine + buffer * kOutBytes;
#pragma unroll
        for (int h = 0; h < kGroup; h += 32) {
          float y[32];
          if constexpr (kDrain) {
#pragma unroll
            for (int e = 0; e < 32; ++e) y[e] = total[c + h + e];
          } else {
            uint32_t v[32];
            tmem_load32(from + (uint32_t)(c + h), v);
#pragma unroll
            for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(v[e]);
          }
          if constexpr (kConvert) {
            const float4* w4 = (const float4*)(my_scales + c + h);
            const float4* b4 = (const float4*)(my_biases + c + h);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float4 w = w4[q], b = b4[q];
              y[4 * q] = fmaf(y[4 * q] * near * w.x, far, b.x);
              y[4 * q + 1] = fmaf(y[4 * q + 1] * near * w.y, far, b.y);
              y[4 * q + 2] = fmaf(y[4 * q + 2] * near * w.z, far, b.z);
              y[4 * q + 3] = fmaf(y[4 * q + 3] * near * w.w, far, b.w);
            }
          }
          stage_values<TOut>(to, lane, h * (int)sizeof(TOut), y);
        }
        // whole groups only: at a ragged end the TMA writes up to a 16-byte boundary
        if (a.tma_out && n0 + c + kGroup <= a.cols) {
          fence_async_proxy();
          __syncwarp();
          if (lane == 0)  // rows past the end are left out
            tma_store(&out_map, (int32_t)(n0 + c), (int32_t)row0, smem_addr(to));
        } else {
          __syncwarp();
          const int64_t rows = a.rows - row0, left = a.cols - n0 - c;
          store_rows<TOut>(to, lane, (TOut*)a.out + row0 * a.out_stride + n0 + c, a.out_stride,
                           rows < 32 ? (int)rows : 32, left < kGroup ? (int)left : kGroup);
          __syncwarp();
        }
        // a group for each use of a buffer, an empty one too, so that the wait's count holds
        if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        if (a.out_buffers == 2) buffer ^= 1;
      }
      if constexpr (!kDrain) {
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) tell(bar.taken(acc.slot ^ 1));
      }
    }
    // the stores in flight have read shared memory before the CTA leaves
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  }
  if (!ok) op_flag(a.status, AGNES_OP_TIMEOUT);
  tcgen05_fence_before();
  __syncthreads();
  if constexpr (kPair) cluster_sync();  // nobody arrives at or reads this CTA's any more
  if (warp == kMmaWarp) {
    tcgen05_fence_after();
    if constexpr (kPair)
      tmem_free_pair(tmem, kTmemCols);
    else
      tmem_free(tmem, kTmemCols);
  }
}

// What a launch of tile_kernel is given: operands in 16 bits, `k` values to a row.
struct TileOperands {
  const void *a, *b;  // A of kConvert: 8-bit rows
  int64_t a_stride, b_stride;  // in bytes
  int64_t k;
};

template <typename TOut, bool kConvert, int kCols, bool kDrain, bool kPair>
cudaError_t launch_tiles(TileArgs a, const TileOperands& o, int device, cudaStream_t st) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return cudaErrorNotSupported;
  CUtensorMap a_map, b_map, out_map = {};
  const CUtensorMapDataType type = kConvert ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                            : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const bool mapped =
      (kConvert ? map_rows(encode, &a_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, o.a, o.k, a.rows,
                           o.a_stride, kSliceK, kTileM, CU_TENSOR_MAP_SWIZZLE_64B)
                : map_rows(encode, &a_map, type, o.a, o.k, a.ta * a.rows, o.a_stride, kSliceK,
                           kTileM, CU_TENSOR_MAP_SWIZZLE_128B)) &&
      map_rows(encode, &b_map, type, o.b, o.k, a.tb * a.cols, o.b_stride, kSliceK,
               kPair ? kCols / 2 : kCols, CU_TENSOR_MAP_SWIZZLE_128B);
  if (!mapped) return cudaErrorInvalidValue;
  const int64_t out_bytes = a.out_stride * (int64_t)sizeof(TOut);
  a.tma_out = aligned_rows(a.out, out_bytes, 16) && out_bytes < (1ll << 40);
  if (a.tma_out &&
      !map_rows(encode, &out_map, kMapType<TOut>, a.out, a.cols, a.rows, out_bytes,
                (int)(128 / sizeof(TOut)), 32, CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  static OncePerDevice once;
  const cudaError_t e = once.run(device, [] {
    return cudaFuncSetAttribute(tile_kernel<TOut, kConvert, kCols, kDrain, kPair>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
  });
  if (e != cudaSuccess) return e;
  a.steps = (int32_t)ceil_div(o.k, kSliceK);
  a.last = (int32_t)ceil_div(o.k - (int64_t)(a.steps - 1) * kSliceK, 16);
  if (!kDrain) a.chain = a.steps;
  const int group = kPair ? 2 : 1;
  const int num_sms = op_num_sms(device) / group;  // or pairs of them
  const int64_t tiles_m = ceil_div(a.rows, group * kTileM), tiles_n = ceil_div(a.cols, kCols);
  const int b_slice = a.tb * kCols * 128 / group;
  const int a_slice = a.ta * kOperandBytes + (kConvert ? kRawBytes : 0);
  // 786,432 x 128 to 256 97 us, and 103 with B's slices copied for every tile
  a.resident = !kPair && tiles_n <= num_sms &&
               (int64_t)a.steps * b_slice + 3 * a_slice + kEpilogueWarps * kOutBytes <= tile_smem(kConvert);
  a.slot_bytes = a_slice + (a.resident ? 0 : b_slice);
  const int fixed = a.resident ? a.steps * b_slice : 0;
  const auto slots_with = [&](int buffers) {
    return (tile_smem(kConvert) - fixed - kEpilogueWarps * buffers * kOutBytes) / a.slot_bytes;
  };
  a.out_buffers = slots_with(2) >= 4 ? 2 : 1;
  const int slots = slots_with(a.out_buffers);
  a.slots = slots < kMaxSlots ? slots : kMaxSlots;
  const size_t smem = (size_t)kSmemLimit - tile_smem(kConvert) + (size_t)a.slots * a.slot_bytes + fixed +
                      (size_t)kEpilogueWarps * a.out_buffers * kOutBytes;
  int64_t grid = num_sms;
  if (a.resident) grid = num_sms / tiles_n * tiles_n;  // a CTA's columns stay the same
  if (tiles_m <= grid / tiles_n) grid = tiles_m * tiles_n;
  return launch_next_cluster(tile_kernel<TOut, kConvert, kCols, kDrain, kPair>,
                             dim3((unsigned)(grid * group)), (unsigned)kTileThreads, smem,
                             (unsigned)group, st, a_map, b_map, out_map, a);
}

template <typename TOut, int kRows>
cudaError_t launch_few(const LinearArgs& a, int device, cudaStream_t st) {
  int lanes = 1;
  while (lanes < 32 && lanes < (a.dim + 15) / 16) lanes *= 2;
  const int64_t ctas = ceil_div(a.width, kFewThreads / lanes);
  const int64_t most = 8 * (int64_t)op_num_sms(device);
  linear_few_kernel<TOut, kRows>
      <<<(unsigned)(ctas < most ? ctas : most), kFewThreads, 0, st>>>(lanes, a);
  return cudaGetLastError();
}

// The forward pass' workspace: the weights as fp16, then their scales.
struct LinearSpace {
  int64_t kpad, scales, bytes;
  LinearSpace(int64_t rows, int64_t width, int64_t dim) {
    const bool tiles = rows > kFewRows && width > 0;
    kpad = ceil_div(dim, 8) * 8;
    scales = ceil_div(width * kpad * 2, 256) * 256;
    bytes = tiles ? scales + width * 4 : 0;
  }
};

// The backward pass': the transposed weights' two terms, then the gradient's where it cannot
// be taken as it is.
struct GradInputSpace {
  int64_t wpad, grad, bytes;
  GradInputSpace(int64_t rows, int64_t width, int64_t dim, int32_t dtype, bool direct) {
    wpad = ceil_div(width, 8) * 8;
    grad = ceil_div(2 * dim * wpad * 2, 256) * 256;
    bytes = rows > 0 && width > 0 ? grad + (direct ? 0 : grad_terms(dtype) * rows * wpad * 2) : 0;
  }
};

template <typename TOut, bool kConvert>
cudaError_t launch_product(const TileArgs& a, const TileOperands& o, bool drain, int device,
                           cudaStream_t st) {
  if (drain) {
    // By pairs: the gradient of 8192 x 4096 to 2048 in fp32 418 us and 539 by CTAs of their own,
    // which have the short contractions; those are drained in the gradient in fp32 alone.
    if constexpr (!kConvert && sizeof(TOut) == 4)
      if (o.k <= 128) return launch_tiles<TOut, kConvert, 128, true, false>(a, o, device, st);
    return launch_tiles<TOut, kConvert, 128, true, true>(a, o, device, st);
  }
  // 786,432 x 128 to 128 68 us, and 82 by tiles of 256 columns
  if (a.cols <= 128) return launch_tiles<TOut, kConvert, 128, false, false>(a, o, device, st);
  // Pairs for contractions of more than two slices: 16,384 x 4096 to 4096 356 us and 466 by CTAs
  // of their own, 300,000 x 200 to 256 53 and 65.  A pair's start costs 0.9 us more, and its B is
  // not resident: 300 x 128 to 256 8.8 and 7.9, 786,432 x 128 to 256 98.3 and 97.3.
  if (o.k > 128 && op_num_sms(device) >= 2)
    return launch_tiles<TOut, kConvert, 256, false, true>(a, o, device, st);
  return launch_tiles<TOut, kConvert, 256, false, false>(a, o, device, st);
}

template <typename TOut>
cudaError_t launch_linear(const LinearArgs& l, void* workspace, int32_t* status, int device,
                          cudaStream_t st) {
  const LinearSpace space(l.rows, l.width, l.dim);
  __half* w = (__half*)workspace;
  float* scales = (float*)((uint8_t*)workspace + space.scales);
  const int64_t groups = space.kpad / 8;
  expand_kernel<<<(unsigned)ceil_div(l.width * groups, kFlat), kPrepThreads, 0, st>>>(
      l.w, l.w_stride, l.width, l.dim, l.row_bytes, (int32_t)groups, flat_inverse(groups), w,
      space.kpad, scales);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  TileArgs a = {};
  a.rows = l.rows;
  a.cols = l.width;
  a.ta = a.tb = 1;
  a.chain = 16;  // 1024 products, whose sum of whole numbers is exact
  a.x = l.x;
  a.x_stride = l.x_stride;
  a.row_bytes = l.row_bytes;
  a.col_scale = scales;
  a.bias = l.bias;
  a.out = l.out;
  a.out_stride = l.out_stride;
  a.status = status;
  const TileOperands o = {l.x, w, l.x_stride, space.kpad * 2, l.dim};
  // Whole sums are exact up to 2^24, that of 1040 of the largest products; beyond, a product of
  // 16 loses 2^-23 of the sum at most, so 2048 columns lose 8e-6 where all values are the
  // largest, and nothing else.  Uniform values of one sign lose 7e-6 in 8192 columns, 3e-5 in 16,384
  // and 1e-4 in 32,768, where half a unit of an fp16 result is 2^-12 of it or more and of a bfloat16
  // one 2^-9.  Drained they lose nothing, but the rows are made fp16 for half as many columns:
  // 8192 x 16,384 to 2048 fp16 737 us and not 455.
  const int64_t most = sizeof(TOut) == 4 ? 2048 : std::is_same<TOut, __half>::value ? 8192 : 32768;
  const bool drain = l.dim > most;
  return launch_product<TOut, true>(a, o, drain, device, st);
}

}  // namespace

cudaError_t split_grad(const void* grad, int32_t dtype, int64_t stride, int64_t rows,
                       int64_t width, __nv_bfloat16* out, int64_t wpad, cudaStream_t st) {
  return prepare_operands({}, {grad, stride, rows, width, 0, 0, out, wpad}, dtype, st);
}

agnes_status product_check_sizes(const char* op, int64_t rows, int64_t width, int64_t dim) {
  if (rows < 0 || width < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, width %lld, dim %lld", op, (long long)rows,
                    (long long)width, (long long)dim);
  if (rows >= kProductMaxRows || width >= kProductMaxRows || dim > kInt8MaxDim)
    return op_error(AGNES_ERANGE, "%s: rows %lld, width %lld, dim %lld are too large", op,
                    (long long)rows, (long long)width, (long long)dim);
  return AGNES_OK;
}

agnes_status product_check_step(const char* op, const char* name, int64_t rows, int64_t cols,
                                int64_t stride) {
  if (rows > 1 && stride < cols)
    return op_error(AGNES_EINVAL, "%s: a stride of %lld of %s is below %lld", op, (long long)stride,
                    name, (long long)cols);
  return AGNES_OK;
}

agnes_status product_check_workspace(const char* op, const void* p, int64_t bytes, int64_t need,
                                     int device) {
  if (need == 0) return AGNES_OK;
  OP_TRY(op_on_device(op, "workspace", p, device));
  OP_TRY(op_aligned(op, "workspace", p, 256));
  if (bytes < need)
    return op_error(AGNES_EINVAL, "%s: a workspace of %lld bytes, %lld are needed", op,
                    (long long)bytes, (long long)need);
  return AGNES_OK;
}

agnes_status check_direct(const char* op, int32_t grad_dtype, int32_t direct) {
  if ((direct != 0 && direct != 1) || (direct && grad_dtype != AGNES_BF16))
    return op_error(AGNES_EINVAL, "%s: direct is %d", op, direct);
  return AGNES_OK;
}

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_int8_linear_workspace(int64_t rows, int64_t width, int64_t dim,
                                         int64_t* bytes) {
  const char* op = "agnes_int8_linear_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(product_check_sizes(op, rows, width, dim));
  *bytes = LinearSpace(rows, width, dim).bytes;
  return AGNES_OK;
}

agnes_status agnes_int8_linear(const void* x, int64_t x_stride, int64_t rows, const void* w,
                               int64_t w_stride, int64_t width, int64_t dim, const float* bias,
                               void* out, int32_t out_dtype, int64_t out_stride, void* workspace,
                               int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  const char* op = "agnes_int8_linear";
  OP_TRY(product_check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(int8_check_stride(op, "x", rows, dim, x_stride));
  OP_TRY(int8_check_stride(op, "w", width, dim, w_stride));
  OP_TRY(product_check_step(op, "out", rows, width, out_stride));
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
  OP_TRY(product_check_workspace(op, workspace, workspace_bytes, LinearSpace(rows, width, dim).bytes,
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
    if (rows <= 8) return launch_few<TOut, 8>(a, device, st);
    if (rows <= kFewRows) return launch_few<TOut, kFewRows>(a, device, st);
    return launch_linear<TOut>(a, workspace, status, device, st);
  }));
}

agnes_status agnes_int8_linear_grad_input_workspace(int64_t rows, int64_t width, int64_t dim,
                                                    int32_t grad_dtype, int32_t direct,
                                                    int64_t* bytes) {
  const char* op = "agnes_int8_linear_grad_input_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(product_check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(check_direct(op, grad_dtype, direct));
  *bytes = GradInputSpace(rows, width, dim, grad_dtype, direct).bytes;
  return AGNES_OK;
}

agnes_status agnes_int8_linear_grad_input(const void* grad, int32_t grad_dtype,
                                          int64_t grad_stride, int64_t rows, int64_t width,
                                          const void* w, int64_t w_stride, int64_t dim, void* out,
                                          int32_t out_dtype, int64_t out_stride, void* workspace,
                                          int64_t workspace_bytes, int32_t* status,
                                          void* cuda_stream) {
  const char* op = "agnes_int8_linear_grad_input";
  OP_TRY(product_check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(product_check_step(op, "grad", rows, width, grad_stride));
  OP_TRY(int8_check_stride(op, "w", width, dim, w_stride));
  OP_TRY(product_check_step(op, "out", rows, dim, out_stride));
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
  const int64_t step = rows > 1 ? grad_stride : width;
  const bool direct = takes_grad(grad, grad_dtype, rows > 1 ? grad_stride : 0);
  const GradInputSpace space(rows, width, dim, grad_dtype, direct);
  OP_TRY(product_check_workspace(op, workspace, workspace_bytes, space.bytes, device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const int64_t out_step = rows > 1 ? out_stride : dim;
  if (width == 0)  // a sum over nothing
    return op_launched(op, cudaMemset2DAsync(out, (size_t)(out_step * float_size(out_dtype)), 0,
                                             (size_t)(dim * float_size(out_dtype)), (size_t)rows,
                                             st));
  __nv_bfloat16* wt = (__nv_bfloat16*)workspace;
  __nv_bfloat16* terms = (__nv_bfloat16*)((uint8_t*)workspace + space.grad);
  const int64_t row_bytes = int8_row_bytes(dim);
  TileOperands o = {grad, wt, rows > 1 ? step * 2 : space.wpad * 2, space.wpad * 2, width};
  TileArgs a = {};
  a.ta = 1;
  const TransposeArgs t = {(const uint8_t*)w, width > 1 ? w_stride : row_bytes, width,
                           (int32_t)dim, (int32_t)row_bytes, wt, space.wpad, 0};
  SplitArgs g = {};
  if (!direct) {
    a.ta = grad_terms(grad_dtype);
    g = {grad, step, rows, width, 0, 0, terms, space.wpad};
    o.a = terms;
    o.a_stride = space.wpad * 2;
  }
  OP_TRY(op_launched(op, prepare_operands(t, g, grad_dtype, st)));
  a.rows = rows;
  a.cols = dim;
  a.tb = 2;
  a.out = out;
  a.out_stride = out_step;
  a.status = status;
  return op_launched(op, with_float_type(out_dtype, [&](auto t) {
    using TOut = typename decltype(t)::type;
    // Of values of one sign a product of 16 loses 5e-8 to 9e-8 of the result.  Some 20 to an
    // accumulator where the sum stays in fp32: 8e-7 (1.6e-6 of a gradient in fp32).  16-bit results
    // have 128 undrained at most (7e-6, a thirtieth of half a unit of fp16, which is 2^-12 of a value
    // or more) or 64 (3e-6); undrained sums of 4096 columns lost 3e-5 to 7e-5, of 16,384 2e-4 to 3e-4.
    // It costs 8192 x 4096 to 2048 bfloat16 180 us and not 166 (177 with 128 products to an
    // accumulator, 190 with 24).
    const int per_slice = 4 * (a.ta == 1 ? 2 : a.ta == 2 ? 4 : 5);
    a.chain = (sizeof(TOut) == 4 ? 24 : 64) / per_slice;
    const bool drain = sizeof(TOut) == 4 || ceil_div(width, kSliceK) * per_slice > 128;
    return launch_product<TOut, false>(a, o, drain, device, st);
  }));
}

}  // extern "C"
