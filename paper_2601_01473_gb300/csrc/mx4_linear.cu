// mx4_linear.cu -- 4-bit rows times 4-bit weights (include/agnes_ops.h; the format
// is in mx4.cuh):  out[r][j] = sum_i x[r][i] w[j][i] + bias[j].
//
// Many rows: the block-scaled tensor-core product (tcgen05.mma kind::mxf4), which
// takes e2m1 codes from shared memory and the blocks' scale bytes from tensor
// memory.  Persistent CTAs, one per SM, over output tiles of 128 x 128:
//   the producer      has the TMA copy a stage: 256 codes of 128 rows of x and of w;
//   the scale warps   load the rows' scale bytes, a thread to a row and 512 values
//                     at a time, and lay them out in shared memory as tensor memory
//                     takes them: four blocks' bytes of row 32 g + l in lane l, column g;
//   the MMA warp      has the scales copied to tensor memory (tcgen05.cp) and issues
//                     the stage's products (K = 64 each) into one of two accumulators;
//   the epilogue warps read the accumulator, add the bias, round, and have the TMA
//                     store it from shared memory.
// Rows of up to 512 values: a CTA keeps to one tile of columns and its weights stay in
// shared and tensor memory, so a tile costs the copy of x's rows alone; the grid is then a
// multiple of the tiles across, which leaves SMs idle where those are many (launch_linear).
//
// Short rows are bound by the output's stores: 786,432 rows of 128 to 256 columns in
// fp16 take 92 us, a memset of the same 402 MB 102 us.  Longer rows are bound by no rate:
// 6,000 x 1024 to 4096 columns take 35 us, 1430 TFLOP/s, with the tensor pipe active 16% of
// the time, L2 at 17% of its rate and DRAM at 2%; 100,000 x 300 to 600 columns 51 us with
// 10%, 19% and 19%.  What is left is how long a tile's chain of stages takes: the copies and
// scales on their way, the products, the epilogue, of which a CTA has few at a time.
// Tried without gain: two tiles of columns to each
// stage of x with three accumulators taken in turn by the two sets of epilogue warps
// (93 us; long rows 15% slower), three sets (97 us).
// Every wait is bounded (mbarrier.cuh).  Rows and columns past the matrices' ends
// come as zeros from the TMA.
//
// Few rows: the weights' bytes count and there is little to multiply, so a warp's
// lanes take a block of 32 weights each, for all rows.
#include "mx4.cuh"
#include "tcgen05.cuh"

namespace agnes {

namespace {

constexpr int kTile = 128;        // rows, and columns, of an output tile
constexpr int kStageBytesK = 128;  // bytes of codes of a row per stage: 256 values
constexpr int kCodeBytes = kTile * kStageBytesK;
// The ring: stages of x's codes and w's, or of x's alone beside w's resident ones.
constexpr int kSharedSlots = 4;
constexpr int kResidentStages = 2;
constexpr int kResidentSlots = 6;
constexpr int kMaxSlots = kResidentSlots;
constexpr int kRingBytes = 8 * kCodeBytes;
static_assert(kSharedSlots * 2 == 8 && kResidentSlots + kResidentStages == 8, "the ring");
// Scale bytes: a thread loads 16 of its row, for two stages; a stage of 128 rows is
// two words a row, in two blocks of 512 bytes.
constexpr int kScaleRun = 16;
constexpr int kScaleBlock = kTile * 4;
constexpr int kScaleBytes = 2 * kScaleBlock;
constexpr int kScaleStage = (2 * kMaxSlots + kResidentStages) * kScaleBytes;
constexpr int kRunsAhead = 4;  // runs on their way to a thread, further than a trip to memory
// Tensor memory: two accumulators, each slot's scales (x's eight columns, w's
// eight), the resident w's.
constexpr int kScaleCols = 16;
constexpr int kScaleCol0 = 2 * kTile;
constexpr int kResidentCol0 = kScaleCol0 + kMaxSlots * kScaleCols;
constexpr int kTmemCols = 512;
static_assert(kResidentCol0 + kResidentStages * 8 <= kTmemCols, "tensor memory");
// warps: 0-7 epilogue (two to a quarter of tensor memory's lanes, half the columns
// each), 8-11 scales, 12 producer, 13 MMA
constexpr int kEpilogueWarps = 8;
constexpr int kEpilogueCols = kTile / (kEpilogueWarps / 4);
constexpr int kScaleWarp0 = kEpilogueWarps;
constexpr int kProducerWarp = kScaleWarp0 + 4;
constexpr int kMmaWarp = kProducerWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 1);
static_assert(kScaleWarp0 % 4 == 0, "a scale warp's quarter is its place among the four");
static_assert(kEpilogueCols % 64 == 0, "whole groups of the widest output");
// An epilogue warp's output on its way to memory: 32 rows of 128 bytes, twice.
constexpr int kOutBytes = 32 * 128;
constexpr int kOutBuffers = 2;
constexpr int kOutStage = kEpilogueWarps * kOutBuffers * kOutBytes;
constexpr int kBars = 3 * kMaxSlots + 7;
constexpr size_t kSmemBytes =
    (size_t)kRingBytes + kOutStage + kScaleStage + 1024 + 8 * kBars + 16;
static_assert(kCodeBytes % 1024 == 0 && kOutBytes % 1024 == 0,
              "the swizzled tiles stay 1024-byte aligned");
static_assert(kSmemBytes <= 232448, "shared memory of a CTA");

struct LinearArgs {
  const uint8_t *x, *w;
  int64_t x_stride, w_stride;
  int64_t rows, width;
  int32_t blocks;  // of 32 values
  const float* bias;
  void* out;
  int64_t out_stride;
  bool resident;   // w's stages stay in shared memory: a CTA keeps to one tile of columns
  bool tma_out;    // the output's rows suit the TMA
  bool bias_wide;  // there is a bias, 16-byte aligned
  int32_t* status;
};

// Instruction descriptor of kind::mxf4: e2m1 operands (bits 7-9 and 10-11 = 1), both
// K-major, N >> 3 at bits 17-22, scales of type ue8m0 (bit 23), M >> 7 at bits
// 27-28, K = 64 (bit 31 = 0).  Of the four scale bytes of a tensor-memory word a
// product takes two: from byte `half` * 2, at bits 4-5 (w) and 29-30 (x).
__device__ __forceinline__ uint32_t mx4_idesc(int half) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 3) << 17) | (1u << 23) |
         ((uint32_t)(kTile >> 7) << 27) | ((uint32_t)(2 * half) << 4) |
         ((uint32_t)(2 * half) << 29);
}

__device__ __forceinline__ void mma_mx4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                        uint32_t scale_a, uint32_t scale_b, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], "
      "[%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate)
      : "memory");
}

// A block of 512 bytes from shared memory to four columns of all four quarters of
// tensor memory: lane l takes 16 bytes.
__device__ __forceinline__ void tmem_copy_scales(uint32_t to, uint32_t from) {
  // no swizzle; groups of eight lanes' 16 bytes are 128 bytes apart (bits 32-45)
  const uint64_t desc =
      (uint64_t)((from & 0x3FFFF) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
}

// The mbarriers: full[s] (the TMA has brought slot s), scaled[s] (its scales are laid
// out), empty[s] (its products are done); done[d] / taken[d] of the accumulators;
// w_full / w_scaled of the resident weights; drained, when the MMA warp gives up.
struct Bars {
  uint32_t base;
  __device__ uint32_t at(int i) const { return base + 8u * (uint32_t)i; }
  __device__ uint32_t full(int s) const { return at(s); }
  __device__ uint32_t scaled(int s) const { return at(kMaxSlots + s); }
  __device__ uint32_t empty(int s) const { return at(2 * kMaxSlots + s); }
  __device__ uint32_t done(int d) const { return at(3 * kMaxSlots + d); }
  __device__ uint32_t taken(int d) const { return at(3 * kMaxSlots + 2 + d); }
  __device__ uint32_t w_full() const { return at(3 * kMaxSlots + 4); }
  __device__ uint32_t w_scaled() const { return at(3 * kMaxSlots + 5); }
  __device__ uint32_t drained() const { return at(3 * kMaxSlots + 6); }
};

// The output tiles of a CTA, every gridDim.x-th: columns change fastest, so they stay
// the same where the grid is a multiple of the tiles across.
struct Tiles {
  int64_t m, n;  // tile coordinates
  int64_t tiles_n, tiles_m, step_m, step_n;
  __device__ explicit Tiles(const LinearArgs& a) {
    tiles_n = (a.width + kTile - 1) / kTile;
    tiles_m = (a.rows + kTile - 1) / kTile;
    m = blockIdx.x / tiles_n;
    n = blockIdx.x - m * tiles_n;
    step_m = gridDim.x / tiles_n;
    step_n = gridDim.x - step_m * tiles_n;
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

// The scale bytes of two stages of a row, zeros past the matrix and past the row's
// blocks (the bytes there are not the row's).
__device__ __forceinline__ uint4 scale_run(const uint8_t* p, int64_t stride, int64_t row,
                                           int64_t rows, int32_t blocks, int pair) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (row >= rows) return v;
  v = __ldg((const uint4*)(p + row * stride + (int64_t)blocks * 16) + pair);
  const int left = blocks - pair * kScaleRun;
  if (left < kScaleRun) {
    const auto keep = [&](uint32_t word, int first) {
      const int n = left - first;
      return n >= 4 ? word : n <= 0 ? 0u : word & ((1u << (8 * n)) - 1u);
    };
    v = make_uint4(keep(v.x, 0), keep(v.y, 4), keep(v.z, 8), keep(v.w, 12));
  }
  return v;
}

// A row's two words of a stage to their blocks.
__device__ __forceinline__ void put_scales(uint8_t* blocks, int r, uint32_t first,
                                           uint32_t second) {
  uint8_t* to = blocks + (r & 31) * 16 + (r >> 5) * 4;
  *(uint32_t*)to = first;
  *(uint32_t*)(to + kScaleBlock) = second;
}

// The bias of 32 columns from c0 on; of those past the width, zeros.
__device__ __forceinline__ void load_bias(const LinearArgs& a, int64_t c0, float (&b)[32]) {
  const bool full = c0 + 32 <= a.width;
  if (a.bias_wide && full) {
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
      const float4 v = __ldg((const float4*)(a.bias + c0 + e));
      b[e] = v.x;
      b[e + 1] = v.y;
      b[e + 2] = v.z;
      b[e + 3] = v.w;
    }
  } else if (!a.bias) {
#pragma unroll
    for (int e = 0; e < 32; ++e) b[e] = 0.f;
  } else {
    const int left = full ? 32 : (int)(a.width - c0);
#pragma unroll
    for (int e = 0; e < 32; ++e) b[e] = e < left ? __ldg(a.bias + c0 + e) : 0.f;
  }
}

// 32 columns of a lane's row into its warp's buffer, from byte `first` of its 128 on:
// 16-byte pieces permuted by the row as the TMA's 128-byte swizzle has them, so that
// eight lanes' pieces lie in different banks.
template <typename TOut>
__device__ __forceinline__ void stage_columns(uint8_t* buffer, int lane, int first,
                                              const uint32_t (&v)[32], const float (&b)[32]) {
  constexpr int kN = 16 / sizeof(TOut);
#pragma unroll
  for (int q = 0; q < 32 / kN; ++q) {
    Vec<TOut, kN> y;
#pragma unroll
    for (int e = 0; e < kN; ++e)
      y.v[e] = from_f32<TOut>(__uint_as_float(v[q * kN + e]) + b[q * kN + e]);
    *(Vec<TOut, kN>*)(buffer + lane * 128 + (((first / 16 + q) ^ (lane & 7)) << 4)) = y;
  }
}

template <typename TOut>
__global__ void __launch_bounds__(kThreads, 1)
linear_kernel(const __grid_constant__ CUtensorMap x_codes,
              const __grid_constant__ CUtensorMap w_codes,
              const __grid_constant__ CUtensorMap out_map, const LinearArgs a) {
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  uint8_t* out_stage = smem + kRingBytes;
  uint8_t* scale_stage = out_stage + kOutStage;
  uint64_t* bars = (uint64_t*)(scale_stage + kScaleStage);
  uint32_t* tmem_slot = (uint32_t*)(bars + kBars);
  const Bars bar = {smem_addr(bars)};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_addr(tmem_slot)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int s = 0; s < kMaxSlots; ++s) {
      mbar_init(bar.full(s), 1);
      mbar_init(bar.scaled(s), 4);
      mbar_init(bar.empty(s), 1);
    }
    for (int d = 0; d < 2; ++d) {
      mbar_init(bar.done(d), 1);
      mbar_init(bar.taken(d), kEpilogueWarps);
    }
    mbar_init(bar.w_full(), 1);
    mbar_init(bar.w_scaled(), 4);
    mbar_init(bar.drained(), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  Tiles t(a);
  const int stages = (a.blocks + 7) / 8;  // of 256 values, per tile
  const int steps = (a.blocks + 1) / 2;   // products of 64 values, per tile
  const bool resident = a.resident;
  const int slots = resident ? kResidentSlots : kSharedSlots;
  const int slot_bytes = resident ? kCodeBytes : 2 * kCodeBytes;
  const uint32_t ring_at = smem_addr(smem);
  const uint32_t w_ring_at = ring_at + kResidentSlots * kCodeBytes;  // the resident stages
  uint8_t* w_scale_stage = scale_stage + 2 * kMaxSlots * kScaleBytes;
  bool ok = true;

  if (warp == kProducerWarp) {
    if (lane == 0) {
      if (resident) {
        mbar_expect(bar.w_full(), (uint32_t)(stages * kCodeBytes));
        for (int k = 0; k < stages; ++k)
          tma_load(w_ring_at + (uint32_t)(k * kCodeBytes), &w_codes, k * kStageBytesK,
                   (int32_t)(t.n * kTile), bar.w_full());
      }
      Ring ring;
      int64_t issued = 0;
      for (; ok && t.any(); t.next()) {
        const int32_t m0 = (int32_t)(t.m * kTile), n0 = (int32_t)(t.n * kTile);
        for (int k = 0; k < stages; ++k) {
          const int s = ring.slot;
          if (!ring.first && !mbar_wait(bar.empty(s), ring.parity ^ 1u)) {
            ok = false;
            break;
          }
          const uint32_t at = ring_at + (uint32_t)(s * slot_bytes);
          mbar_expect(bar.full(s), (uint32_t)slot_bytes);
          tma_load(at, &x_codes, k * kStageBytesK, m0, bar.full(s));
          if (!resident)
            tma_load(at + kCodeBytes, &w_codes, k * kStageBytesK, n0, bar.full(s));
          ring.next(slots);
          ++issued;
        }
      }
      if (!ok) {  // the copies in flight land before the CTA may leave
        if (resident) mbar_wait(bar.w_full(), 0);
        Ring r;
        for (int64_t i = 0; i < issued; ++i, r.next(slots))
          if (i + slots >= issued) mbar_wait(bar.full(r.slot), r.parity);
      }
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0) {
      if (resident) {
        ok = mbar_wait(bar.w_full(), 0) && mbar_wait(bar.w_scaled(), 0);
        if (ok)
          for (int c = 0; c < 2 * stages; ++c)
            tmem_copy_scales(tmem + kResidentCol0 + (uint32_t)(c * 4),
                             smem_addr(w_scale_stage + c * kScaleBlock));
      }
      Ring ring, acc;
      for (; ok && t.any(); t.next()) {
        const int d = acc.slot;
        if (!acc.first && !mbar_wait(bar.taken(d), acc.parity ^ 1u)) {
          ok = false;
          break;
        }
        for (int k = 0; k < stages; ++k) {
          const int s = ring.slot;
          if (!mbar_wait(bar.full(s), ring.parity) || !mbar_wait(bar.scaled(s), ring.parity)) {
            ok = false;
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t x_at = ring_at + (uint32_t)(s * slot_bytes);
          const uint32_t w_at =
              resident ? w_ring_at + (uint32_t)(k * kCodeBytes) : x_at + kCodeBytes;
          const uint32_t x_scale = tmem + kScaleCol0 + (uint32_t)(s * kScaleCols);
          const uint32_t w_scale =
              resident ? tmem + kResidentCol0 + (uint32_t)(k * 8) : x_scale + 8u;
          const int n = min(4, steps - 4 * k);
          const uint32_t scales = smem_addr(scale_stage + s * 2 * kScaleBytes);
          for (int c = 0; c < (n + 1) / 2; ++c) {
            tmem_copy_scales(x_scale + 4u * (uint32_t)c, scales + (uint32_t)(c * kScaleBlock));
            if (!resident)
              tmem_copy_scales(w_scale + 4u * (uint32_t)c,
                               scales + (uint32_t)(kScaleBytes + c * kScaleBlock));
          }
          for (int i = 0; i < n; ++i)
            mma_mx4(tmem + (uint32_t)(d * kTile), operand_desc(x_at + 32u * (uint32_t)i),
                    operand_desc(w_at + 32u * (uint32_t)i), mx4_idesc(i & 1),
                    x_scale + 4u * (uint32_t)(i >> 1), w_scale + 4u * (uint32_t)(i >> 1),
                    k > 0 || i > 0);
          mma_commit(bar.empty(s));
          ring.next(slots);
        }
        if (!ok) break;
        mma_commit(bar.done(d));
        acc.next(2);
      }
      if (!ok) {  // the products in flight end before the tensor memory is freed
        mma_commit(bar.drained());
        mbar_wait(bar.drained(), 0);
      }
    }
  } else if (warp >= kScaleWarp0) {
    const int r = tid - 32 * kScaleWarp0;  // this thread's row of the tile
    const int pairs = (stages + 1) / 2;
    // what the tensor core reads has been written, for the thread that waits for `b`
    const auto tell = [&](uint32_t b) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(b);
    };
    if (resident) {  // one pair at most
      const uint4 v = scale_run(a.w, a.w_stride, t.n * kTile + r, a.width, a.blocks, 0);
      put_scales(w_scale_stage, r, v.x, v.y);
      put_scales(w_scale_stage + kScaleBytes, r, v.z, v.w);
      tell(bar.w_scaled());
    }
    Tiles ahead = t;
    int ahead_pair = 0;
    const auto load = [&](uint4& x, uint4& w) {
      if (!ahead.any()) return;
      x = scale_run(a.x, a.x_stride, ahead.m * kTile + r, a.rows, a.blocks, ahead_pair);
      if (!resident)
        w = scale_run(a.w, a.w_stride, ahead.n * kTile + r, a.width, a.blocks, ahead_pair);
      if (++ahead_pair == pairs) {
        ahead_pair = 0;
        ahead.next();
      }
    };
    uint4 x_run[kRunsAhead], w_run[kRunsAhead];
#pragma unroll
    for (int q = 0; q < kRunsAhead; ++q) {
      x_run[q] = w_run[q] = make_uint4(0, 0, 0, 0);
      load(x_run[q], w_run[q]);
    }
    Ring ring;
    int p = 0;
    while (ok && t.any()) {
      // unrolled, so that a run stays in its registers until it is used
#pragma unroll
      for (int q = 0; q < kRunsAhead; ++q) {
        if (!ok || !t.any()) break;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (2 * p + h >= stages) break;
          const int s = ring.slot;
          if (!ring.first &&
              !__all_sync(0xffffffffu, mbar_wait(bar.empty(s), ring.parity ^ 1u))) {
            ok = false;
            break;
          }
          uint8_t* to = scale_stage + s * 2 * kScaleBytes;
          const uint4 &x = x_run[q], &w = w_run[q];
          put_scales(to, r, h ? x.z : x.x, h ? x.w : x.y);
          if (!resident) put_scales(to + kScaleBytes, r, h ? w.z : w.x, h ? w.w : w.y);
          tell(bar.scaled(s));
          ring.next(slots);
        }
        load(x_run[q], w_run[q]);
        if (++p == pairs) {
          p = 0;
          t.next();
        }
      }
    }
  } else {
    constexpr int kGroup = 128 / sizeof(TOut);  // columns of a staged buffer
    uint8_t* mine = out_stage + warp * kOutBuffers * kOutBytes;
    int buffer = 0;
    Ring acc;
    for (; t.any(); t.next()) {
      const int d = acc.slot;
      if (!__all_sync(0xffffffffu, mbar_wait(bar.done(d), acc.parity))) {
        ok = false;
        break;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int64_t row0 = t.m * kTile + (warp & 3) * 32;
      const int64_t n0 = t.n * kTile + (warp >> 2) * kEpilogueCols;
      const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) +
                            (uint32_t)(d * kTile + (warp >> 2) * kEpilogueCols);
      // a warp whose rows are all past the end has nothing to store, and its buffers
      // may still be on their way
      const int cols = row0 < a.rows ? kEpilogueCols : 0;
      for (int c = 0; c < cols && n0 + c < a.width; c += kGroup) {
        // the store before the last has read the buffer
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int h = 0; h < kGroup / 32; ++h) {
          uint32_t v[32];
          float b[32];
          load_bias(a, n0 + c + h * 32, b);  // on its way with the accumulator's
          tmem_load32(from + (uint32_t)(c + h * 32), v);
          stage_columns<TOut>(mine + buffer * kOutBytes, lane, h * 64, v, b);
        }
        // whole groups only: at a ragged end the TMA writes up to a 16-byte boundary
        if (a.tma_out && n0 + c + kGroup <= a.width) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0)  // rows past the end are left out
            tma_store(&out_map, (int32_t)(n0 + c), (int32_t)row0,
                      smem_addr(mine + buffer * kOutBytes));
        } else {
          __syncwarp();
          const int64_t rows = a.rows - row0, left = a.width - n0 - c;
          store_rows<TOut>(mine + buffer * kOutBytes, lane,
                           (TOut*)a.out + row0 * a.out_stride + n0 + c, a.out_stride,
                           rows < 32 ? (int)rows : 32, left < kGroup ? (int)left : kGroup);
          __syncwarp();
        }
        // a group for each use of a buffer, an empty one too, so that the wait's count holds
        if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        buffer ^= 1;
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar.taken(d));
      acc.next(2);
    }
    // the stores in flight have read shared memory before the CTA leaves
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  }
  if (!ok) op_flag(a.status, AGNES_OP_TIMEOUT);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                 "r"(kTmemCols)
                 : "memory");
  }
}

// ---- few rows ----------------------------------------------------------------

constexpr int kFewRows = 8;
constexpr int kFewThreads = 256;
constexpr size_t kFewSmem = 200 * 1024;

// Shared memory: the rows' values without their scales, in vectors of 8 halves,
// vector q of block b of row r at (r * 4 + q) * blocks + b; then the scales,
// row by row.
size_t few_smem(int64_t rows, int64_t blocks) { return (size_t)(rows * blocks * (64 + 4)); }

// kLanes lanes per column of the output.
template <typename TOut, int kRows>
__global__ void __launch_bounds__(kFewThreads)
linear_few_kernel(int lanes, const LinearArgs a) {
  extern __shared__ __align__(16) uint8_t few_raw[];
  uint4* values = (uint4*)few_raw;
  float* scales = (float*)(values + (size_t)kRows * 4 * a.blocks);
  for (int i = threadIdx.x; i < kRows * a.blocks; i += kFewThreads) {
    const int r = i / a.blocks, b = i - r * a.blocks;
    uint4 codes = make_uint4(0, 0, 0, 0);
    uint32_t byte = 0;
    if (r < a.rows) {
      codes = __ldg((const uint4*)(a.x + r * a.x_stride) + b);
      byte = __ldg(a.x + r * a.x_stride + (int64_t)a.blocks * 16 + b);
    }
    const uint32_t word[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      __half2 h[4];
      mx4_values(word[q], h);
      values[(size_t)(r * 4 + q) * a.blocks + b] = *(const uint4*)h;
    }
    scales[i] = mx4_scale(byte);
  }
  __syncthreads();
  const int lane = threadIdx.x % lanes;
  const int64_t per_cta = kFewThreads / lanes;
  for (int64_t j0 = (int64_t)blockIdx.x * per_cta; j0 < a.width; j0 += gridDim.x * per_cta) {
    const int64_t j = j0 + threadIdx.x / lanes;
    float sum[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) sum[r] = 0.f;
    if (j < a.width) {
      const uint8_t* row = a.w + j * a.w_stride;
      for (int b = lane; b < a.blocks; b += lanes) {
        const uint4 codes = __ldg((const uint4*)row + b);
        const float scale = mx4_scale(__ldg(row + (int64_t)a.blocks * 16 + b));
        const uint32_t word[4] = {codes.x, codes.y, codes.z, codes.w};
        __half2 h[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) mx4_values(word[q], h[q]);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          // a half of an accumulator sums 8 products, multiples of 1/4 of at most 36:
          // exact in fp16
          float dot = 0.f;
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            __half2 acc = __float2half2_rn(0.f);
#pragma unroll
            for (int q = 2 * p; q < 2 * p + 2; ++q) {
              const uint4 v = values[(size_t)(r * 4 + q) * a.blocks + b];
              const __half2* xv = (const __half2*)&v;
#pragma unroll
              for (int e = 0; e < 4; ++e) acc = __hfma2(xv[e], h[q][e], acc);
            }
            const float2 f = __half22float2(acc);
            dot += f.x + f.y;
          }
          // the smaller scale first: |dot| <= 1152 and a multiple of 1/4, so that product is
          // exact (2^-129 at the least) or no larger than the whole one
          const float other = scales[r * a.blocks + b];
          const bool less = other < scale;  // a NaN is a factor either way
          sum[r] += dot * (less ? other : scale) * (less ? scale : other);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      for (int d = lanes / 2; d > 0; d >>= 1)
        sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], d);
    if (lane == 0 && j < a.width) {
      const float b = a.bias ? __ldg(a.bias + j) : 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (r < a.rows) ((TOut*)a.out)[r * a.out_stride + j] = from_f32<TOut>(sum[r] + b);
    }
  }
}

// ---- host ----------------------------------------------------------------------

template <typename TOut>
cudaError_t launch_linear(LinearArgs a, int device, cudaStream_t st) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return cudaErrorNotSupported;
  const int64_t codes = (int64_t)a.blocks * 16;
  CUtensorMap x_map, w_map, out_map = {};
  const auto codes_map = [&](CUtensorMap* map, const uint8_t* p, int64_t rows, int64_t stride) {
    return map_rows(encode, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, p, codes, rows, stride,
                    kStageBytesK, kTile, CU_TENSOR_MAP_SWIZZLE_128B);
  };
  if (!codes_map(&x_map, a.x, a.rows, a.x_stride) || !codes_map(&w_map, a.w, a.width, a.w_stride))
    return cudaErrorInvalidValue;
  const int64_t out_bytes = a.out_stride * (int64_t)sizeof(TOut);
  a.tma_out = aligned_rows(a.out, out_bytes, 16) && out_bytes < (1ll << 40);
  if (a.tma_out &&
      !map_rows(encode, &out_map, kMapType<TOut>, a.out, a.width, a.rows, out_bytes,
                (int)(128 / sizeof(TOut)), 32, CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  static OncePerDevice once;
  const cudaError_t e = once.run(device, [] {
    return cudaFuncSetAttribute(linear_kernel<TOut>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int num_sms = op_num_sms(device);
  const int64_t tiles_m = ceil_div(a.rows, kTile), tiles_n = ceil_div(a.width, kTile);
  // Resident or not, 50,000 rows to fp16 (us): of 128 values to 256 columns 13 and 17, 3328
  // 86 and 109, 6656 183 and 210, 9856 (77 of the 152 SMs at work) 338 and 311; of 512
  // values to 3328 columns 130 and 113, 6656 308 and 216, 9856 606 and 317; 100,000 rows of
  // 300 to 600 51 and 54.  So a narrower rule would serve wide outputs better, those of
  // rows of two stages above all.
  a.resident = ceil_div(a.blocks, 8) <= kResidentStages && tiles_n <= num_sms;
  int64_t grid = num_sms;
  if (a.resident) grid = num_sms / tiles_n * tiles_n;  // a CTA's columns stay the same
  if (tiles_m <= grid / tiles_n) grid = tiles_m * tiles_n;
  linear_kernel<TOut><<<(unsigned)grid, kThreads, kSmemBytes, st>>>(x_map, w_map, out_map, a);
  return cudaGetLastError();
}

template <typename TOut, int kRows>
cudaError_t launch_few(const LinearArgs& a, int device, cudaStream_t st) {
  int lanes = 1;
  while (lanes < 32 && lanes < a.blocks) lanes *= 2;
  const int64_t ctas = ceil_div(a.width, kFewThreads / lanes);
  const size_t smem = few_smem(kRows, a.blocks);
  const int num_sms = op_num_sms(device);
  static OncePerDevice once;
  const cudaError_t e = once.run(device, [] {
    return cudaFuncSetAttribute(linear_few_kernel<TOut, kRows>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem);
  });
  if (e != cudaSuccess) return e;
  linear_few_kernel<TOut, kRows>
      <<<(unsigned)(ctas < 8 * num_sms ? ctas : 8 * num_sms), kFewThreads, smem, st>>>(
          lanes, a);
  return cudaGetLastError();
}

constexpr int64_t kMaxDim = 1 << 26;
constexpr int64_t kMaxRows = 0x7fffffff - 255;

}  // namespace

}  // namespace agnes

using namespace agnes;

extern "C" agnes_status agnes_mx4_linear(const void* x, int64_t x_stride, int64_t rows,
                                         const void* w, int64_t w_stride, int64_t width,
                                         int64_t dim, const float* bias, void* out,
                                         int32_t out_dtype, int64_t out_stride, int32_t* status,
                                         void* cuda_stream) {
  const char* op = "agnes_mx4_linear";
  if (rows < 0 || width < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, width %lld, dim %lld", op, (long long)rows,
                    (long long)width, (long long)dim);
  if (rows > kMaxRows || width > kMaxRows || dim > kMaxDim)
    return op_error(AGNES_ERANGE, "%s: rows %lld, width %lld, dim %lld are too large", op,
                    (long long)rows, (long long)width, (long long)dim);
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(mx4_check_stride(op, "x", rows, dim, x_stride));
  OP_TRY(mx4_check_stride(op, "w", width, dim, w_stride));
  if (rows > 1 && out_stride < width)
    return op_error(AGNES_EINVAL, "%s: out_stride %lld is below width %lld", op,
                    (long long)out_stride, (long long)width);
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
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  LinearArgs a = {};
  a.rows = rows;
  a.width = width;
  a.blocks = (int32_t)mx4_blocks(dim);
  a.bias = bias;
  a.bias_wide = bias && (uintptr_t)bias % 16 == 0;
  a.out = out;
  a.out_stride = out_stride;
  a.status = status;
  // a single row has no next one: any stride will do
  a.x = (const uint8_t*)x;
  a.w = (const uint8_t*)w;
  a.x_stride = rows > 1 ? x_stride : mx4_row_bytes(dim);
  a.w_stride = width > 1 ? w_stride : mx4_row_bytes(dim);
  if (rows == 1) a.out_stride = width;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = with_float_type(out_dtype, [&](auto t) {
    using TOut = typename decltype(t)::type;
    if (rows <= kFewRows && few_smem(rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8,
                                     a.blocks) <= kFewSmem) {
      if (rows == 1) return launch_few<TOut, 1>(a, device, st);
      if (rows == 2) return launch_few<TOut, 2>(a, device, st);
      if (rows <= 4) return launch_few<TOut, 4>(a, device, st);
      return launch_few<TOut, 8>(a, device, st);
    }
    return launch_linear<TOut>(a, device, st);
  });
  return op_launched(op, e);
}
