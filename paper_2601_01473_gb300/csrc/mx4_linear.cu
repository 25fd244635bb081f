// mx4_linear.cu -- 4-bit rows times 4-bit weights (include/agnes_ops.h; the format
// is in mx4.cuh):  out[r][j] = sum_i x[r][i] w[j][i] + bias[j].
//
// Many rows: the block-scaled tensor-core product (tcgen05.mma kind::mxf4), which
// takes e2m1 codes from shared memory and the blocks' scale bytes from tensor
// memory.  Persistent CTAs, one per SM, over output tiles of 128 x 128:
//   the producer      has the TMA copy a stage: 256 codes of 128 rows of x and of
//                     w, and the 16-byte runs that hold their scale bytes;
//   the scale warps   put the stage's scale bytes from shared into tensor
//                     memory: lane l of each quarter, column g, holds those of
//                     row 32 g + l for four blocks;
//   the MMA warp      issues the stage's products (K = 64 each) into one of two
//                     accumulators;
//   the epilogue warps read the accumulator, add the bias, round and store.
// Every wait is bounded (mbarrier.cuh).  Rows and columns past the matrices' ends
// come as zeros from the TMA.
//
// Few rows: the weights' bytes count and there is little to multiply, so a warp's
// lanes take a block of 32 weights each, for all rows.
#include <cuda.h>

#include <atomic>

#include "mbarrier.cuh"
#include "mx4.cuh"
#include "ops_common.cuh"

namespace agnes {

namespace {

constexpr int kTile = 128;        // rows, and columns, of an output tile
constexpr int kStageBytesK = 128;  // bytes of codes of a row per stage: 256 values
constexpr int kCodeBytes = kTile * kStageBytesK;
constexpr int kScaleRun = 16;     // scale bytes the TMA brings per row, for two stages
constexpr int kScaleBytes = kTile * kScaleRun;
constexpr int kStageBytes = 2 * kCodeBytes + 2 * kScaleBytes;
constexpr int kStages = 4;
constexpr int kScaleCols = 16;    // tensor-memory columns of a stage's scales
constexpr int kScaleCol0 = 2 * kTile;  // after two accumulators
constexpr int kTmemCols = 512;
// warps: 0-7 epilogue (two to a quarter of tensor memory's lanes, half the columns
// each), 8-11 scales, 12 producer, 13 MMA
constexpr int kEpilogueWarps = 8;
constexpr int kEpilogueCols = kTile / (kEpilogueWarps / 4);
constexpr int kScaleWarp0 = kEpilogueWarps;
constexpr int kProducerWarp = kScaleWarp0 + 4;
constexpr int kMmaWarp = kProducerWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 1);
constexpr int kBars = 3 * kStages + 5;
// An epilogue warp's output on its way to memory: 32 rows of 128 bytes, twice.
constexpr int kOutBytes = 32 * 128;
constexpr int kOutBuffers = 2;
constexpr int kOutStage = kEpilogueWarps * kOutBuffers * kOutBytes;
constexpr size_t kSmemBytes =
    (size_t)kStages * kStageBytes + kOutStage + 1024 + 8 * kBars + 16;
static_assert(kStageBytes % 1024 == 0 && kOutBytes % 1024 == 0,
              "the swizzled tiles stay 1024-byte aligned");
static_assert(kSmemBytes <= 232448, "shared memory of a CTA");
static_assert(kEpilogueCols % 64 == 0, "whole groups of the widest output");
static_assert(kScaleCol0 + kStages * kScaleCols <= kTmemCols, "tensor memory");

struct LinearArgs {
  int64_t rows, width;
  int32_t blocks;  // of 32 values
  const float* bias;
  void* out;
  int64_t out_stride;
  bool tma_out;    // the output's rows suit the TMA
  bool bias_wide;  // there is a bias, 16-byte aligned
  int32_t* status;
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}

__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y,
                                         uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

// A K-major operand with 128-byte swizzle: atoms of 8 rows x 128 bytes, 1024 bytes
// apart (bits 32-45), descriptor version 1 (bits 46-48), swizzle mode 2 (bits 61-63).
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}

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

__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
      : "memory");
}

__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, "
      "%10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
      "%26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
        "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
        "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
        "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(addr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
      "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// The mbarriers: full[s] (the TMA has brought stage s), scaled[s] (its scales are in
// tensor memory), empty[s] (its products are done); done[d] / taken[d] of the
// accumulators; drained, when the MMA warp gives up.
struct Bars {
  uint32_t base;
  __device__ uint32_t full(int s) const { return base + 8u * (uint32_t)s; }
  __device__ uint32_t scaled(int s) const { return base + 8u * (uint32_t)(kStages + s); }
  __device__ uint32_t empty(int s) const { return base + 8u * (uint32_t)(2 * kStages + s); }
  __device__ uint32_t done(int d) const { return base + 8u * (uint32_t)(3 * kStages + d); }
  __device__ uint32_t taken(int d) const { return base + 8u * (uint32_t)(3 * kStages + 2 + d); }
  __device__ uint32_t drained() const { return base + 8u * (uint32_t)(3 * kStages + 4); }
};

struct Ring {
  int slot = 0;
  uint32_t parity = 0;  // of the phase that this use completes
  bool first = true;    // no earlier use to wait for
  __device__ void next(int n) {
    if (++slot == n) {
      slot = 0;
      parity ^= 1u;
      first = false;
    }
  }
};

// 32 columns of a row of the output from column c0 on, for rows that do not suit
// the TMA.
template <typename TOut>
__device__ __forceinline__ void store_columns(const LinearArgs& a, TOut* row, int64_t c0,
                                              const uint32_t (&v)[32]) {
#pragma unroll
  for (int e = 0; e < 32; ++e) {
    if (c0 + e >= a.width) break;
    const float b = a.bias ? __ldg(a.bias + c0 + e) : 0.f;
    row[c0 + e] = from_f32<TOut>(__uint_as_float(v[e]) + b);
  }
}

// 32 columns of a lane's row into its warp's buffer, from byte `first` of its 128 on:
// 16-byte pieces permuted by the row as the TMA's 128-byte swizzle has them, so that
// eight lanes' pieces lie in different banks.
template <typename TOut>
__device__ __forceinline__ void stage_columns(const LinearArgs& a, uint8_t* buffer, int lane,
                                              int first, int64_t c0, const uint32_t (&v)[32]) {
  constexpr int kN = 16 / sizeof(TOut);
  float f[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]);
  if (a.bias_wide) {
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
      const float4 b = __ldg((const float4*)(a.bias + c0 + e));
      f[e] += b.x;
      f[e + 1] += b.y;
      f[e + 2] += b.z;
      f[e + 3] += b.w;
    }
  } else if (a.bias) {
#pragma unroll
    for (int e = 0; e < 32; ++e) f[e] += __ldg(a.bias + c0 + e);
  }
#pragma unroll
  for (int q = 0; q < 32 / kN; ++q) {
    Vec<TOut, kN> y;
#pragma unroll
    for (int e = 0; e < kN; ++e) y.v[e] = from_f32<TOut>(f[q * kN + e]);
    *(Vec<TOut, kN>*)(buffer + lane * 128 + (((first / 16 + q) ^ (lane & 7)) << 4)) = y;
  }
}

__device__ __forceinline__ void tma_store(const CUtensorMap* map, int32_t x, int32_t y,
                                          uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                   map),
               "r"(x), "r"(y), "r"(src)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

template <typename TOut>
__global__ void __launch_bounds__(kThreads, 1)
linear_kernel(const __grid_constant__ CUtensorMap x_codes, const __grid_constant__ CUtensorMap x_scales,
              const __grid_constant__ CUtensorMap w_codes, const __grid_constant__ CUtensorMap w_scales,
              const __grid_constant__ CUtensorMap out_map, const LinearArgs a) {
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  uint8_t* out_stage = smem + (size_t)kStages * kStageBytes;
  uint64_t* bars = (uint64_t*)(out_stage + kOutStage);
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
    for (int s = 0; s < kStages; ++s) {
      mbar_init(bar.full(s), 1);
      mbar_init(bar.scaled(s), 4);
      mbar_init(bar.empty(s), 1);
    }
    for (int d = 0; d < 2; ++d) {
      mbar_init(bar.done(d), 1);
      mbar_init(bar.taken(d), kEpilogueWarps);
    }
    mbar_init(bar.drained(), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  const int64_t tiles_n = (a.width + kTile - 1) / kTile;
  const int64_t tiles = (a.rows + kTile - 1) / kTile * tiles_n;
  const int stages = (a.blocks + 7) / 8;  // of 256 values, per tile
  const int steps = (a.blocks + 1) / 2;   // products of 64 values, per tile
  bool ok = true;

  if (warp == kProducerWarp) {
    if (lane == 0) {
      Ring ring;
      int64_t issued = 0;
      for (int64_t t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
        const int32_t m0 = (int32_t)(t / tiles_n * kTile), n0 = (int32_t)(t % tiles_n * kTile);
        for (int k = 0; k < stages; ++k) {
          const int s = ring.slot;
          if (!ring.first && !mbar_wait(bar.empty(s), ring.parity ^ 1u)) {
            ok = false;
            break;
          }
          const uint32_t at = smem_addr(smem) + (uint32_t)(s * kStageBytes);
          mbar_expect(bar.full(s), kStageBytes);
          tma_load(at, &x_codes, k * kStageBytesK, m0, bar.full(s));
          tma_load(at + kCodeBytes, &w_codes, k * kStageBytesK, n0, bar.full(s));
          // two stages' scale bytes: the copy starts on a 16-byte boundary
          tma_load(at + 2 * kCodeBytes, &x_scales, k / 2 * kScaleRun, m0, bar.full(s));
          tma_load(at + 2 * kCodeBytes + kScaleBytes, &w_scales, k / 2 * kScaleRun, n0,
                   bar.full(s));
          ring.next(kStages);
          ++issued;
        }
      }
      if (!ok) {  // the copies in flight land before the CTA may leave
        Ring r;
        for (int64_t i = 0; i < issued; ++i, r.next(kStages))
          if (i + kStages >= issued) mbar_wait(bar.full(r.slot), r.parity);
      }
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0) {
      Ring ring, acc;
      for (int64_t t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
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
          const uint32_t x_at = smem_addr(smem) + (uint32_t)(s * kStageBytes);
          const uint32_t w_at = x_at + kCodeBytes;
          const uint32_t scale = tmem + kScaleCol0 + (uint32_t)(s * kScaleCols);
          const int n = min(4, steps - 4 * k);
          for (int i = 0; i < n; ++i)
            mma_mx4(tmem + (uint32_t)(d * kTile), operand_desc(x_at + 32u * (uint32_t)i),
                    operand_desc(w_at + 32u * (uint32_t)i), mx4_idesc(i & 1),
                    scale + 4u * (uint32_t)(i >> 1), scale + 8u + 4u * (uint32_t)(i >> 1),
                    k > 0 || i > 0);
          mma_commit(bar.empty(s));
          ring.next(kStages);
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
    // columns of a stage: x's first four blocks, x's next four, w's likewise; four
    // columns each, column g for rows 32 g .. 32 g + 31
    const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
    Ring ring;
    for (int64_t t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
      for (int k = 0; k < stages; ++k) {
        const int s = ring.slot;
        if (!__all_sync(0xffffffffu, mbar_wait(bar.full(s), ring.parity))) {
          ok = false;
          break;
        }
        const uint8_t* at = smem + s * kStageBytes + 2 * kCodeBytes + (k & 1) * 8;
        uint32_t v[16];
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint2 b =
                *(const uint2*)(at + o * kScaleBytes + (32 * g + lane) * kScaleRun);
            v[8 * o + g] = b.x;
            v[8 * o + 4 + g] = b.y;
          }
        tmem_store16(tmem + quarter + kScaleCol0 + (uint32_t)(s * kScaleCols), v);
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar.scaled(s));
        ring.next(kStages);
      }
    }
  } else {
    constexpr int kGroup = 128 / sizeof(TOut);  // columns of a staged buffer
    uint8_t* mine = out_stage + warp * kOutBuffers * kOutBytes;
    int buffer = 0;
    Ring acc;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
      const int d = acc.slot;
      if (!__all_sync(0xffffffffu, mbar_wait(bar.done(d), acc.parity))) {
        ok = false;
        break;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int64_t row0 = t / tiles_n * kTile + (warp & 3) * 32;
      const int64_t n0 = t % tiles_n * kTile + (warp >> 2) * kEpilogueCols;
      const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) +
                            (uint32_t)(d * kTile + (warp >> 2) * kEpilogueCols);
      for (int c = 0; c < kEpilogueCols && n0 + c < a.width; c += kGroup) {
        // whole groups only: at a ragged end the TMA writes up to a 16-byte boundary
        const bool staged = a.tma_out && n0 + c + kGroup <= a.width;
        if (staged) {  // the store before the last has read the buffer
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          __syncwarp();
        }
#pragma unroll
        for (int h = 0; h < kGroup / 32; ++h) {
          uint32_t v[32];
          tmem_load32(from + (uint32_t)(c + h * 32), v);
          if (staged)
            stage_columns<TOut>(a, mine + buffer * kOutBytes, lane, h * 64, n0 + c + h * 32, v);
          else if (row0 + lane < a.rows)
            store_columns<TOut>(a, (TOut*)a.out + (row0 + lane) * a.out_stride, n0 + c + h * 32, v);
        }
        if (staged) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0 && row0 < a.rows)  // rows past the end are left out
            tma_store(&out_map, (int32_t)(n0 + c), (int32_t)row0,
                      smem_addr(mine + buffer * kOutBytes));
          buffer ^= 1;
        }
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
linear_few_kernel(const uint8_t* __restrict__ x, int64_t x_stride, const uint8_t* __restrict__ w,
                  int64_t w_stride, int lanes, const LinearArgs a) {
  extern __shared__ __align__(16) uint8_t few_raw[];
  uint4* values = (uint4*)few_raw;
  float* scales = (float*)(values + (size_t)kRows * 4 * a.blocks);
  for (int i = threadIdx.x; i < kRows * a.blocks; i += kFewThreads) {
    const int r = i / a.blocks, b = i - r * a.blocks;
    uint4 codes = make_uint4(0, 0, 0, 0);
    uint32_t byte = 0;
    if (r < a.rows) {
      codes = __ldg((const uint4*)(x + r * x_stride) + b);
      byte = __ldg(x + r * x_stride + (int64_t)a.blocks * 16 + b);
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
      const uint8_t* row = w + j * w_stride;
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
          sum[r] += dot * scales[r * a.blocks + b] * scale;
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

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                 const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static std::atomic<void*> known{nullptr};
  void* fn = known.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault,
                                         &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    known.store(fn, std::memory_order_release);
  }
  return (EncodeTiled)fn;
}

// `rows` rows of `cols` elements of `type`, `stride` bytes apart, in boxes of
// box_rows x box_cols; zeros past either end.
bool map_rows(EncodeTiled encode, CUtensorMap* map, CUtensorMapDataType type, const void* p,
              int64_t cols, int64_t rows, int64_t stride, int box_cols, int box_rows,
              CUtensorMapSwizzle swizzle) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, type, 2, (void*)p, size, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T>
constexpr CUtensorMapDataType kMapType = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
template <>
constexpr CUtensorMapDataType kMapType<__half> = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
template <>
constexpr CUtensorMapDataType kMapType<__nv_bfloat16> = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;

template <typename TOut>
cudaError_t launch_linear(const void* x, int64_t x_stride, const void* w, int64_t w_stride,
                          LinearArgs a, int device, cudaStream_t st) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return cudaErrorNotSupported;
  const int64_t codes = (int64_t)a.blocks * 16;
  const uint8_t *xb = (const uint8_t*)x, *wb = (const uint8_t*)w;
  CUtensorMap xc, xs, wc, ws, out = {};
  const auto bytes = [&](CUtensorMap* map, const void* p, int64_t cols, int64_t rows,
                         int64_t stride, int box, CUtensorMapSwizzle swizzle) {
    return map_rows(encode, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, p, cols, rows, stride, box, kTile,
                    swizzle);
  };
  if (!bytes(&xc, xb, codes, a.rows, x_stride, kStageBytesK, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !bytes(&xs, xb + codes, a.blocks, a.rows, x_stride, kScaleRun,
             CU_TENSOR_MAP_SWIZZLE_NONE) ||
      !bytes(&wc, wb, codes, a.width, w_stride, kStageBytesK, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !bytes(&ws, wb + codes, a.blocks, a.width, w_stride, kScaleRun, CU_TENSOR_MAP_SWIZZLE_NONE))
    return cudaErrorInvalidValue;
  const int64_t out_bytes = a.out_stride * (int64_t)sizeof(TOut);
  a.tma_out = aligned_rows(a.out, out_bytes, 16) && out_bytes < (1ll << 40);
  if (a.tma_out &&
      !map_rows(encode, &out, kMapType<TOut>, a.out, a.width, a.rows, out_bytes,
                (int)(128 / sizeof(TOut)), 32, CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  static OncePerDevice once;
  const cudaError_t e = once.run(device, [] {
    return cudaFuncSetAttribute(linear_kernel<TOut>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int64_t tiles = ceil_div(a.rows, kTile) * ceil_div(a.width, kTile);
  const int num_sms = op_num_sms(device);
  linear_kernel<TOut><<<(unsigned)(tiles < num_sms ? tiles : num_sms), kThreads, kSmemBytes, st>>>(
      xc, xs, wc, ws, out, a);
  return cudaGetLastError();
}

template <typename TOut, int kRows>
cudaError_t launch_few(const void* x, int64_t x_stride, const void* w, int64_t w_stride,
                       const LinearArgs& a, int device, cudaStream_t st) {
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
          (const uint8_t*)x, x_stride, (const uint8_t*)w, w_stride, lanes, a);
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
  if (status) OP_TRY(op_on_device(op, "status", status, device));
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
  if (rows == 1) x_stride = mx4_row_bytes(dim);
  if (width == 1) w_stride = mx4_row_bytes(dim);
  if (rows == 1) a.out_stride = width;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = with_float_type(out_dtype, [&](auto t) {
    using TOut = typename decltype(t)::type;
    if (rows <= kFewRows && few_smem(rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8,
                                     a.blocks) <= kFewSmem) {
      if (rows == 1) return launch_few<TOut, 1>(x, x_stride, w, w_stride, a, device, st);
      if (rows == 2) return launch_few<TOut, 2>(x, x_stride, w, w_stride, a, device, st);
      if (rows <= 4) return launch_few<TOut, 4>(x, x_stride, w, w_stride, a, device, st);
      return launch_few<TOut, 8>(x, x_stride, w, w_stride, a, device, st);
    }
    return launch_linear<TOut>(x, x_stride, w, w_stride, a, device, st);
  });
  return op_launched(op, e);
}
