// int8_grad_weight.cu -- the gradient of the product of 8-bit rows and 8-bit weights to the
// weights and the bias (include/agnes_ops.h; the format is in int8.cuh):
//
//   dw[j][i] = sum_r grad[r][j] s[r] q[r][i],  dbias[j] = sum_r grad[r][j]
//
// The rows are the contraction, so both operands are taken as they lie in memory, a row of
// shared memory to a row (MN-major).  A whole number times a scale of eight bits is exactly
// the sum of two bfloat16 values, its leading eight bits and the rest (of other scales' rows
// 16 bits are kept; they take the convert warps longer, 786,432 x 128 to 256 160 us); the two
// matrices lie side by side, so that one product of 128 x 256 makes both sums and reads the
// gradient once.
//
// A CTA takes a tile of 128 x 128 of the output and a share of the rows:
//   the producer      has the TMA copy slices of 64 rows, the gradient's terms and the whole
//                     numbers as they are;
//   the convert warps scale the whole numbers and write both terms (kReady: a kernel before has,
//                     once for all tiles);
//   the MMA warp      issues the products into one of two accumulators, `chain` slices each;
//   the epilogue warps add the accumulators up in registers and write a partial tile, and
//                     meanwhile add the gradient's columns up, of the first tile of columns.
// Tensor memory's sums are cut off, not rounded, after each product, which loses 5e-8 to 9e-8 of
// a sum of values of one sign: a CTA's share of a hyperbatch's rows, some 300 products, would lose
// 2e-5 in one chain, so chains are short.  A second
// kernel adds the shares' tiles up in order, so the result is the same each time.
// 786,432 rows of 128 to 256 columns, bfloat16: 102 us, 5.1 TB/s (memory); 8192 rows of 2048 to
// 4096 columns 232 us, of which 205 here, the tensor pipe 62% active, 22 the shares' sum.
#include <type_traits>

#include "int8_product.cuh"

namespace agnes {

namespace {

constexpr int kTile = 128;
constexpr int kSlice = 64;  // rows to a stage
constexpr int kEpilogueWarps = 8;
constexpr int kConvertWarp0 = kEpilogueWarps, kConvertWarps = 4;
constexpr int kProducerWarp = kConvertWarp0 + kConvertWarps;
constexpr int kMmaWarp = kProducerWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 1);
constexpr int kBox = kSlice * 128;           // 64 columns of a slice in 16 bits
constexpr int kGradBytes = 2 * kBox;         // a term of the gradient
// Of the scaled whole numbers' two terms and of the whole numbers (none where the terms come
// ready), for a CTA of its own or one of a pair.
constexpr int value_bytes(bool pair) { return (pair ? 2 : 4) * kBox; }
constexpr int raw_bytes(bool pair, bool ready) {
  return ready ? 0 : kSlice * kTile / (pair ? 2 : 1);
}
constexpr int kMaxSlots = 6;
constexpr int kBars = 3 * kMaxSlots + 5;
constexpr int kSmemLimit = 232448;
constexpr int kRingBytes = kSmemLimit - 1024 - 8 * kBars - 16;
constexpr int kTmemCols = 512;
constexpr int kTileValues = kTile * kTile;
constexpr int kSms = 152;  // that the rows are shared out for, whatever the device: a GB300's

struct WeightArgs {
  int64_t rows, width;
  int32_t dim, row_bytes;
  const uint8_t* x;
  int64_t x_stride;
  int32_t ta;
  bool pair, ready;
  int32_t slices;             // of all rows
  int32_t tiles_j, tiles_i;   // of the output, along width and dim
  int32_t splits, per_split;  // shares of the rows, slices of one
  int32_t chain;
  float* partial;             // [split][tile][kTileValues], as the threads hold them
  float* bias_partial;        // [split][4][width], or null
  void* out;
  int64_t out_stride;
  float* dbias;
  int32_t slots, slot_bytes;
  int32_t* status;
};

// full[s] (the TMA has brought slot s), ready[s] (both terms are written), empty[s] (nobody
// reads it any more); done[d] / taken[d] of the accumulators; drained, when the MMA warp
// gives up.
struct WeightBars {
  uint32_t base;
  __device__ uint32_t at(int i) const { return base + 8u * (uint32_t)i; }
  __device__ uint32_t full(int s) const { return at(s); }
  __device__ uint32_t ready(int s) const { return at(kMaxSlots + s); }
  __device__ uint32_t empty(int s) const { return at(2 * kMaxSlots + s); }
  __device__ uint32_t done(int d) const { return at(3 * kMaxSlots + d); }
  __device__ uint32_t taken(int d) const { return at(3 * kMaxSlots + 2 + d); }
  __device__ uint32_t drained() const { return at(3 * kMaxSlots + 4); }
};

// kReady: the scaled whole numbers' terms are copied like the gradient's.
// kPair: two CTAs have 256 x 128 of the output, each the gradient's columns and the output of
// its half and both terms of half of the whole numbers.
template <bool kPair, bool kReady>
__global__ void __launch_bounds__(kThreads, 1)
weight_kernel(const __grid_constant__ CUtensorMap grad_map,
              const __grid_constant__ CUtensorMap x_map, const WeightArgs a) {
  grid_dep_wait();
  static_assert(kPair || !kReady, "many tiles");
  constexpr uint32_t kIdesc = idesc_16bit(true, true, kPair ? 2 * kTile : kTile, 2 * kTile);
  constexpr int kValueBytes = value_bytes(kPair), kRawBytes = raw_bytes(kPair, kReady);
  const uint32_t rank = kPair ? cluster_rank() : 0;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  uint64_t* bars = (uint64_t*)(smem + a.slots * a.slot_bytes);
  uint32_t* tmem_slot = (uint32_t*)(bars + kBars);
  const WeightBars bar = {smem_addr(bars)};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // this CTA's tile and share
  const int64_t tiles = (int64_t)a.tiles_j * a.tiles_i;
  constexpr int kGroup = kPair ? 2 : 1;
  const int64_t item = blockIdx.x / kGroup, groups = tiles / kGroup;
  const int64_t split = item / groups, group = item % groups;
  const int32_t tile_i = (int32_t)(group % a.tiles_i);
  const int64_t tile_j = group / a.tiles_i * kGroup + rank, tile = tile_j * a.tiles_i + tile_i;
  const int64_t j0 = tile_j * kTile;
  const int32_t i0 = tile_i * kTile;
  const int32_t k0 = (int32_t)split * a.per_split, k1 = min(k0 + a.per_split, a.slices);
  const bool bias = a.bias_partial && tile_i == 0;
  if (warp == kMmaWarp) {
    if constexpr (kPair)
      tmem_alloc_pair(tmem_slot, kTmemCols);
    else
      tmem_alloc(tmem_slot, kTmemCols);
  }
  if (tid == 0) {
    for (int s = 0; s < kMaxSlots; ++s) {
      mbar_init(bar.full(s), 1);
      mbar_init(bar.ready(s), (kReady ? 1 : kConvertWarps) * kGroup);
      mbar_init(bar.empty(s), 1 + (bias ? kEpilogueWarps : 0));
    }
    for (int d = 0; d < 2; ++d) {
      mbar_init(bar.done(d), 1);
      mbar_init(bar.taken(d), kEpilogueWarps * kGroup);
    }
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
  const uint32_t ring_at = smem_addr(smem);
  // in a slot: the gradient's terms, the scaled whole numbers', the whole numbers
  const uint32_t value_off = (uint32_t)(a.ta * kGradBytes), raw_off = value_off + kValueBytes;
  bool ok = true;
  Ring ring;

  if (warp == kProducerWarp) {
    if (lane == 0) {
      int64_t issued = 0;
      for (int32_t k = k0; k < k1; ++k) {
        const int s = ring.slot;
        if (!ring.first && !mbar_wait(bar.empty(s), ring.parity ^ 1u)) {
          ok = false;
          break;
        }
        const uint32_t at = ring_at + (uint32_t)(s * a.slot_bytes);
        mbar_expect(bar.full(s), (uint32_t)(a.ta * kGradBytes + (kReady ? kValueBytes : kRawBytes)));
        // Past the last row a term's slice runs into the next term, which is finite there
        // and meets zeros.
        for (int p = 0; p < a.ta; ++p)
          for (int b = 0; b < 2; ++b)
            tma_load(at + (uint32_t)(p * kGradBytes + b * kBox), &grad_map,
                     (int32_t)(j0 + b * 64), (int32_t)(p * a.rows + (int64_t)k * kSlice),
                     bar.full(s));
        if constexpr (kReady) {  // boxes of 64 columns of each term
          constexpr int kBoxes = kValueBytes / 2 / kBox;
          for (int b = 0; b < 2 * kBoxes; ++b)
            tma_load(at + value_off + (uint32_t)(b * kBox), &x_map,
                     i0 + (int32_t)rank * (kTile / 2) + b % kBoxes * 64,
                     (int32_t)((b / kBoxes * (int64_t)a.slices + k) * kSlice), bar.full(s));
        } else {
          tma_load(at + raw_off, &x_map, i0 + (int32_t)rank * (kTile / 2),
                   (int32_t)((int64_t)k * kSlice), bar.full(s));
        }
        ring.next(a.slots);
        ++issued;
      }
      if (kPair && ok) {  // the other CTA's last arrivals here land before this one may leave
        for (int s = 0; ok && s < a.slots; ++s) {
          ok = ring.first || mbar_wait(bar.empty(ring.slot), ring.parity ^ 1u);
          ring.next(a.slots);
        }
      }
      if (!ok) {  // the copies in flight land before the CTA may leave
        Ring r;
        for (int64_t i = 0; i < issued; ++i, r.next(a.slots))
          if (i + a.slots >= issued) mbar_wait(bar.full(r.slot), r.parity);
      }
    }
  } else if (warp == kMmaWarp) {
    // the whole warp goes through the loop, so that its addresses are the same for all lanes and
    // stay in uniform registers, as the products take them
    if (rank == 0) {
      const bool lead = elect_one();
      const auto multiply = [](uint32_t d, uint64_t x, uint64_t y, uint32_t more) {
        if constexpr (kPair)
          mma_16bit_pair(d, x, y, kIdesc, more);
        else
          mma_16bit(d, x, y, kIdesc, more);
      };
      const auto commit = [](uint32_t b) {
        if constexpr (kPair)
          mma_commit_pair(b);
        else
          mma_commit(b);
      };
      Ring acc;
      for (int32_t c0 = k0; ok && c0 < k1; c0 += a.chain) {
        const int d = acc.slot;
        if (!acc.first && !__all_sync(0xffffffffu, mbar_wait(bar.taken(d), acc.parity ^ 1u))) {
          ok = false;
          break;
        }
        tcgen05_fence_after();
        const uint32_t to = tmem + (uint32_t)(d * 2 * kTile);
        uint32_t accumulate = 0;
        for (int32_t k = c0; k < min(c0 + a.chain, k1); ++k) {
          const int s = ring.slot;
          // what is ready is full as well
          if (!__all_sync(0xffffffffu, mbar_wait(bar.ready(s), ring.parity))) {
            ok = false;
            break;
          }
          tcgen05_fence_after();
          const uint32_t at = ring_at + (uint32_t)(s * a.slot_bytes);
          const int64_t left = a.rows - (int64_t)k * kSlice;
          const int n = left < kSlice ? (int)((left + 15) / 16) : kSlice / 16;
          // descriptors are sums of constants: one thread issues all products
          const uint64_t g0 = operand_desc_mn(at, kBox), v0 = operand_desc_mn(at + value_off, kBox);
          if (lead) {
#pragma unroll
            for (int i = 0; i < kSlice / 16; ++i) {
              if (i >= n) break;
              multiply(to, g0 + (uint64_t)(i * 128), v0 + (uint64_t)(i * 128),
                       accumulate | (uint32_t)(i > 0));
              if (a.ta > 1)
                multiply(to, g0 + (uint64_t)(i * 128 + (kGradBytes >> 4)), v0 + (uint64_t)(i * 128),
                         1);
              if (a.ta > 2)
                multiply(to, g0 + (uint64_t)(i * 128 + 2 * (kGradBytes >> 4)),
                         v0 + (uint64_t)(i * 128), 1);
            }
            commit(bar.empty(s));
          }
          __syncwarp();
          accumulate = 1;
          ring.next(a.slots);
        }
        if (!ok) break;
        if (lead) commit(bar.done(d));
        __syncwarp();
        acc.next(2);
      }
      if (!ok) {  // the products in flight end before the tensor memory is freed
        if (lead) commit(bar.drained());
        mbar_wait(bar.drained(), 0);
      }
    }
  } else if (warp >= kConvertWarp0 && kReady) {
    // one warp tells the pair's first CTA of this one's slices
    if (warp == kConvertWarp0) {
      for (int32_t k = k0; k < k1; ++k) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar.full(ring.slot), ring.parity))) {
          ok = false;
          break;
        }
        if (lane == 0) tell(bar.ready(ring.slot));
        ring.next(a.slots);
      }
    }
  } else if (warp >= kConvertWarp0) {
    // a thread to 64 values of a row (32 of a pair's): neighbouring threads to neighbouring
    // rows, whose pieces lie in different banks
    constexpr int kPieces = kPair ? 2 : 4;  // of 16 whole numbers
    const int t = tid - 32 * kConvertWarp0, half = t >> 6, r = t & 63;
    const auto scale_of = [&](int32_t k) {
      const int64_t row = (int64_t)k * kSlice + r;
      return k < k1 && row < a.rows
                 ? __ldg((const float*)(a.x + row * a.x_stride + a.row_bytes - 4)) : 0.f;
    };
    float next = scale_of(k0);
    for (int32_t k = k0; k < k1; ++k) {
      const int s = ring.slot;
      const float scale = next;
      next = scale_of(k + 1);
      if (!__all_sync(0xffffffffu, mbar_wait(bar.full(s), ring.parity))) {
        ok = false;
        break;
      }
      uint8_t* slot = smem + s * a.slot_bytes;
      const uint8_t* from = slot + raw_off + r * (raw_bytes(kPair, false) / kSlice);
      // a box of 64 values for each half, or one for both; behind them the second terms'
      uint8_t* to = slot + value_off + (kPair ? 0 : half * kBox) + r * 128;
      const int first = kPair ? 4 * half : 0;  // piece of 8 values of the box
      const Int8TermScale s2(scale);
      uint4 w[kPieces];
#pragma unroll
      for (int c = 0; c < kPieces; ++c) {
        const int piece = half * kPieces + c;  // as the TMA's swizzle of 64 or 128 bytes has it
        w[c] = *(const uint4*)(from + ((piece ^ (kPair ? (r >> 1) & 3 : r & 7)) << 4));
      }
      const auto write_terms = [&](auto brief) {
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
          uint2 hi[4], lo[4];
          int8_terms4<brief>(w[c].x, s2, hi[0], lo[0]);
          int8_terms4<brief>(w[c].y, s2, hi[1], lo[1]);
          int8_terms4<brief>(w[c].z, s2, hi[2], lo[2]);
          int8_terms4<brief>(w[c].w, s2, hi[3], lo[3]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = ((first + 2 * c + h) ^ (r & 7)) << 4;
            *(uint4*)(to + at) =
                make_uint4(hi[2 * h].x, hi[2 * h].y, hi[2 * h + 1].x, hi[2 * h + 1].y);
            *(uint4*)(to + kValueBytes / 2 + at) =
                make_uint4(lo[2 * h].x, lo[2 * h].y, lo[2 * h + 1].x, lo[2 * h + 1].y);
          }
        }
      };
      // once for all of a warp's rows: 786,432 x 128 to 256 takes 21 us more by a choice for each
      // four values
      if (__all_sync(0xffffffffu, s2.brief))
        write_terms(std::true_type());
      else
        write_terms(std::false_type());
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) tell(bar.ready(s));
      ring.next(a.slots);
    }
  } else {
    constexpr int kHalf = kTile / 2;
    // both terms' sums of 128 columns, or of a pair's first 64 and then of its second
    constexpr int kTerms = kPair ? kHalf : kTile;  // from a column's first sum to its second
    const uint32_t lanes_at = tmem + ((uint32_t)((warp & 3) * 32) << 16) +
                              (uint32_t)((warp >> 2) * (kPair ? kTile : kHalf));
    float total[kHalf];
#pragma unroll
    for (int e = 0; e < kHalf; ++e) total[e] = 0.f;
    // of the bias, a warp has two columns to a lane and a quarter of a slice's rows
    float column[2] = {0.f, 0.f};
    const int box = warp & 1, rows0 = (warp >> 1) * (kSlice / 4);
    Ring acc;
    for (int32_t c0 = k0; ok && c0 < k1; c0 += a.chain) {
      if (bias) {
        for (int32_t k = c0; k < min(c0 + a.chain, k1); ++k) {
          const int s = ring.slot;
          if (!__all_sync(0xffffffffu, mbar_wait(bar.full(s), ring.parity))) {
            ok = false;
            break;
          }
          // a row's 16-byte pieces as the TMA's swizzle has them; rows past the last are zeros,
          // or the next term's, which only ever follow terms of their own
          const uint8_t* from = smem + s * a.slot_bytes + box * kBox + (lane & 3) * 4;
          const int64_t left = a.rows - (int64_t)k * kSlice - rows0;
          for (int p = 0; p < a.ta; ++p)
#pragma unroll
            for (int r = 0; r < kSlice / 4; ++r) {
              const uint32_t v = *(const uint32_t*)(from + p * kGradBytes + (rows0 + r) * 128 +
                                                    (((lane >> 2) ^ (r & 7)) << 4));
              if (r < left) {
                column[0] += __uint_as_float(v << 16);
                column[1] += __uint_as_float(v & 0xffff0000u);
              }
            }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar.empty(s));
          ring.next(a.slots);
        }
        if (!ok) break;
      }
      const int d = acc.slot;
      if (!__all_sync(0xffffffffu, mbar_wait(bar.done(d), acc.parity))) {
        ok = false;
        break;
      }
      tcgen05_fence_after();
#pragma unroll
      for (int c = 0; c < 2 * kHalf; c += 32) {  // the leading bits' sums, then the rest's
        uint32_t v[32];
        tmem_load32(lanes_at + (uint32_t)(d * 2 * kTile + c % kHalf + c / kHalf * kTerms), v);
#pragma unroll
        for (int e = 0; e < 32; ++e) total[c % kHalf + e] += __uint_as_float(v[e]);
      }
      tcgen05_fence_before();
      __syncwarp();
      if (lane == 0) tell(bar.taken(d));
      acc.next(2);
    }
    float4* to = (float4*)(a.partial + (split * tiles + tile) * kTileValues) + warp * 16 * 32;
#pragma unroll
    for (int c = 0; c < kHalf / 4; ++c)
      to[c * 32 + lane] = make_float4(total[4 * c], total[4 * c + 1], total[4 * c + 2],
                                      total[4 * c + 3]);
    if (bias) {  // four quarters' sums of a column, added up with the shares'
      const int64_t j = j0 + box * 64 + lane * 2;
      float* to_bias = a.bias_partial + (split * 4 + (warp >> 1)) * a.width;
      if (j < a.width) to_bias[j] = column[0];
      if (j + 1 < a.width) to_bias[j + 1] = column[1];
    }
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

// Both terms of the scaled whole numbers, dpad to a row, zeros past the last row up to a
// whole slice, one matrix after the other.
constexpr int kValuesThreads = 256;
struct ValuesArgs {
  const uint8_t* x;
  int64_t stride, rows, padded;  // rows of x, and of a term
  int32_t row_bytes, groups;     // groups of 8 columns to a row of dpad
  uint32_t inv_groups;
  __nv_bfloat16* out;
};
__global__ void __launch_bounds__(kValuesThreads)
terms_kernel(const ValuesArgs a) {
  const FlatRows flat(blockIdx.x, a.groups, a.inv_groups);
#pragma unroll
  for (int u = 0; u < kFlat / kValuesThreads; ++u) {
    int64_t row;
    uint32_t g;
    flat.at(threadIdx.x + u * kValuesThreads, &row, &g);
    if (row >= a.padded) continue;
    uint2 hi[2] = {}, lo[2] = {};
    if (row < a.rows) {
      const uint8_t* from = a.x + row * a.stride;
      const Int8TermScale s2(__ldg((const float*)(from + a.row_bytes - 4)));
      const uint2 w = __ldg((const uint2*)(from + g * 8));
      int8_terms4<false>(w.x, s2, hi[0], lo[0]);
      int8_terms4<false>(w.y, s2, hi[1], lo[1]);
    }
    const int64_t at = row * a.groups + g;  // in 16 bytes; columns past dim are not looked at
    ((uint4*)a.out)[at] = make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y);
    ((uint4*)a.out)[a.padded * a.groups + at] = make_uint4(lo[0].x, lo[0].y, lo[1].x, lo[1].y);
  }
}

// The shares' tiles added up: 32 rows of 64 / kDeal columns of a tile to a CTA, each value's
// shares dealt out to kDeal threads, whose sums are added in order.  The CTAs behind the tiles'
// have the bias.
constexpr int kJoinThreads = 512;
template <typename TOut, int kDeal>
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const WeightArgs a) {
  grid_dep_wait();
  constexpr int kQuads = 16 / kDeal, kParts = 8 * kDeal;  // of four columns; CTAs to a tile
  constexpr int kCols = 4 * kQuads;
  __shared__ float4 sums[kDeal][kQuads][33];
  const int64_t tiles = (int64_t)a.tiles_j * a.tiles_i;
  if (blockIdx.x >= tiles * kParts) {  // 32 columns, their shares dealt out to the warps
    float* part_sums = (float*)sums;
    const int64_t j = (blockIdx.x - tiles * kParts) * 32 + (threadIdx.x & 31);
    float sum = 0.f;
    if (j < a.width) {
#pragma unroll 4
      for (int s = threadIdx.x >> 5; s < 4 * a.splits; s += kJoinThreads / 32)
        sum += a.bias_partial[(int64_t)s * a.width + j];
    }
    part_sums[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || j >= a.width) return;
    for (int w = 1; w < kJoinThreads / 32; ++w) sum += part_sums[w * 32 + threadIdx.x];
    a.dbias[j] = sum;
    return;
  }
  const int lane = threadIdx.x & 31, quad = (threadIdx.x >> 5) % kQuads;
  const int deal = (threadIdx.x >> 5) / kQuads;
  const int64_t tile = blockIdx.x / kParts;
  const int part = blockIdx.x % kParts, warp = part / kDeal, c = part % kDeal * kQuads + quad;
  const float4* from = (const float4*)(a.partial + tile * kTileValues) + (warp * 16 + c) * 32 + lane;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = deal; s < a.splits; s += kDeal) {
    const float4 p = from[(int64_t)s * tiles * (kTileValues / 4)];
    v.x += p.x;
    v.y += p.y;
    v.z += p.z;
    v.w += p.w;
  }
  sums[deal][quad][lane] = v;
  __syncthreads();
  // a row's columns to neighbouring threads
#pragma unroll
  for (int t = threadIdx.x; t < 32 * kCols; t += kJoinThreads) {
    const int r = t / kCols, i_in = t % kCols;
    const int64_t j = tile / a.tiles_i * kTile + (warp & 3) * 32 + r;
    const int32_t i = (int32_t)(tile % a.tiles_i) * kTile + (warp >> 2) * 64 +
                      part % kDeal * kCols + i_in;
    if (j >= a.width || i >= a.dim) continue;
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < kDeal; ++s) sum += ((const float*)&sums[s][i_in / 4][r])[i_in % 4];
    ((TOut*)a.out)[j * a.out_stride + i] = from_f32<TOut>(sum);
  }
}

// How the rows are shared out, and the workspace: partial tiles, partial biases, and the
// gradient's terms where it cannot be taken as it is.
struct WeightSpace {
  bool pair, ready;
  int64_t slices, tiles_j, tiles_i, splits, per_split, wpad, dpad, bias, grad, values, bytes;
  WeightSpace(int64_t rows, int64_t width, int64_t dim, int32_t dtype, bool direct) {
    slices = ceil_div(rows, kSlice);
    // Pairs where there are two tiles: 786,432 rows of 128 to 256 columns 102 us, 130 by CTAs of
    // their own, 8192 of 2048 to 4096 232 and 250; with half a pair idle, 100,000 of 300 to 600
    // 118 and 126.
    pair = width > kTile;
    tiles_j = pair ? ceil_div(width, 2 * kTile) * 2 : 1;
    tiles_i = ceil_div(dim, kTile);
    wpad = ceil_div(width, 8) * 8;
    const int64_t tiles = tiles_j * tiles_i;
    // one CTA to an SM, or a pair to two: shares so that the last turn is as full as the others
    splits = 1;
    if (tiles > 0 && slices > 0) {
      double best = 0;
      for (int64_t s = 1; s <= slices && s * tiles <= 8 * kSms + tiles; ++s) {
        const int64_t per = ceil_div(slices, s), used = ceil_div(slices, per);
        // a share costs some slices' time besides, for its start and its partial tile
        const double turns = (double)(ceil_div(used * tiles, kSms) * (per + 6));
        if (s == 1 || turns < best) {
          best = turns;
          splits = used;
        }
      }
    }
    per_split = slices ? ceil_div(slices, splits) : 0;
    bias = ceil_div(splits * tiles * kTileValues * 4, 256) * 256;
    grad = bias + ceil_div(splits * width * 16, 256) * 256;
    values = grad + (direct ? 0 : ceil_div(grad_terms(dtype) * rows * wpad * 2, 256) * 256);
    dpad = ceil_div(dim, 8) * 8;
    // The scaled whole numbers made once, before, where many tiles share them and the products
    // of a slice take least: 8192 rows of 2048 to 4096 columns, bfloat16, 232 us and 267 by each
    // tile's own convert warps, 4096 x 256 to 4096 25.2 and 25.9.  Below, what they have to write
    // and read costs more: 100,000 x 128 to 1024 61 and 55, 600 x 1024 to 4096 27.8 and 27.2;
    // with a gradient of two terms 8192 x 2048 to 4096 384 and 379.
    ready = dtype == AGNES_BF16 && tiles_j >= 16 && rows >= 4096;
    bytes = rows > 0 && width > 0 ? values + (ready ? 2 * slices * kSlice * dpad * 2 : 0) : 0;
  }
  void shape(WeightArgs& a) const {
    a.pair = pair;
    a.ready = ready;
    a.slices = (int32_t)slices;
    a.tiles_j = (int32_t)tiles_j;
    a.tiles_i = (int32_t)tiles_i;
    a.splits = (int32_t)splits;
    a.per_split = (int32_t)per_split;
  }
};

template <typename TOut>
cudaError_t launch_weight(WeightArgs a, const void* grad, int64_t grad_stride, bool direct,
                          __nv_bfloat16* values, int device, cudaStream_t st) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return cudaErrorNotSupported;
  CUtensorMap grad_map, x_map;
  const int64_t padded = (int64_t)a.slices * kSlice, groups = ceil_div(a.dim, 8);
  if (!map_rows(encode, &grad_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, grad, a.width, a.ta * a.rows,
                grad_stride, 64, kSlice, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !(a.ready ? map_rows(encode, &x_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, values, a.dim,
                           2 * padded, groups * 16, 64, kSlice, CU_TENSOR_MAP_SWIZZLE_128B)
                : map_rows(encode, &x_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.x, a.dim, a.rows,
                           a.x_stride, a.pair ? kTile / 2 : kTile, kSlice,
                           a.pair ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B)))
    return cudaErrorInvalidValue;
  if (a.ready) {
    const ValuesArgs v = {a.x, a.x_stride, a.rows, padded, a.row_bytes, (int32_t)groups,
                          flat_inverse(groups), values};
    terms_kernel<<<(unsigned)ceil_div(padded * groups, kFlat), kValuesThreads, 0, st>>>(v);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const auto kernel = a.ready  ? weight_kernel<true, true>
                      : a.pair ? weight_kernel<true, false>
                               : weight_kernel<false, false>;
  static OncePerDevice once[3];
  cudaError_t e = once[a.pair + a.ready].run(device, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
  });
  if (e != cudaSuccess) return e;
  a.chain = a.ta == 1 ? 5 : a.ta == 2 ? 2 : 1;  // some 16 to 20 products of 16
  a.slot_bytes = a.ta * kGradBytes + value_bytes(a.pair) + raw_bytes(a.pair, a.ready);
  const int slots = kRingBytes / a.slot_bytes;
  a.slots = slots < kMaxSlots ? slots : kMaxSlots;
  const size_t smem = (size_t)kSmemLimit - kRingBytes + (size_t)a.slots * a.slot_bytes;
  const int64_t tiles = (int64_t)a.tiles_j * a.tiles_i;
  const dim3 grid((unsigned)(tiles * a.splits));
  const unsigned cluster = a.pair ? 2u : 1u;
  // the call's first kernel where nothing had to be made of its operands: what is before it on the
  // stream is another call's
  const bool first = direct && !a.ready;
  e = first ? launch_cluster(false, kernel, grid, (unsigned)kThreads, smem, cluster, st, grad_map,
                             x_map, a)
            : launch_next_cluster(kernel, dim3(grid), (unsigned)kThreads, smem, cluster, st,
                                  grad_map, x_map, a);
  if (e != cudaSuccess) return e;
  // Few shares: more values to a CTA; many: more threads to a value.  In the other way the
  // gradient of 8192 rows of 2048 to 4096 columns (2 shares) takes 22 us more, that of 20,000
  // rows of 128 to 128 (as many shares as SMs) 23.7 us and not 11.4.
  const bool few = a.splits <= 8;
  const int64_t ctas = tiles * (few ? 8 : 32) + (a.dbias ? ceil_div(a.width, 32) : 0);
  return launch_next(few ? join_kernel<TOut, 1> : join_kernel<TOut, 4>, dim3((unsigned)ctas),
                     (unsigned)kJoinThreads, 0, st, a);
}

}  // namespace

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_int8_linear_grad_weight_workspace(int64_t rows, int64_t width, int64_t dim,
                                                     int32_t grad_dtype, int32_t direct,
                                                     int64_t* bytes) {
  const char* op = "agnes_int8_linear_grad_weight_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(product_check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(check_direct(op, grad_dtype, direct));
  *bytes = WeightSpace(rows, width, dim, grad_dtype, direct).bytes;
  return AGNES_OK;
}

agnes_status agnes_int8_linear_grad_weight(const void* grad, int32_t grad_dtype,
                                           int64_t grad_stride, int64_t rows, int64_t width,
                                           const void* x, int64_t x_stride, int64_t dim, void* out,
                                           int32_t out_dtype, int64_t out_stride, float* dbias,
                                           void* workspace, int64_t workspace_bytes,
                                           int32_t* status, void* cuda_stream) {
  const char* op = "agnes_int8_linear_grad_weight";
  OP_TRY(product_check_sizes(op, rows, width, dim));
  OP_TRY(op_float_type(op, "grad", grad_dtype));
  OP_TRY(op_float_type(op, "out", out_dtype));
  OP_TRY(product_check_step(op, "grad", rows, width, grad_stride));
  OP_TRY(int8_check_stride(op, "x", rows, dim, x_stride));
  OP_TRY(product_check_step(op, "out", width, dim, out_stride));
  if (width == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "out", out, &device));
  OP_TRY(op_aligned(op, "out", out, float_size(out_dtype)));
  if (dbias) {
    OP_TRY(op_on_device(op, "dbias", dbias, device));
    OP_TRY(op_aligned(op, "dbias", dbias, 4));
  }
  if (rows > 0) {
    OP_TRY(op_on_device(op, "grad", grad, device));
    OP_TRY(op_on_device(op, "x", x, device));
    OP_TRY(op_aligned(op, "grad", grad, float_size(grad_dtype)));
    OP_TRY(op_aligned(op, "x", x, 16));
  }
  OP_TRY(op_status(op, status, device));
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const int64_t out_step = width > 1 ? out_stride : dim;
  if (rows == 0) {  // sums over no rows
    DeviceGuard dg(device);
    if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
    const size_t size = (size_t)float_size(out_dtype);
    OP_TRY(op_launched(op, cudaMemset2DAsync(out, (size_t)out_step * size, 0, (size_t)dim * size,
                                             (size_t)width, st)));
    return dbias ? op_launched(op, cudaMemsetAsync(dbias, 0, (size_t)width * 4, st)) : AGNES_OK;
  }
  const int64_t step = rows > 1 ? grad_stride : width;
  const bool direct = takes_grad(grad, grad_dtype, rows > 1 ? grad_stride : 0);
  const WeightSpace space(rows, width, dim, grad_dtype, direct);
  OP_TRY(product_check_workspace(op, workspace, workspace_bytes, space.bytes, device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const void* a = grad;
  int64_t a_stride = rows > 1 ? step * 2 : space.wpad * 2;
  if (!direct) {
    __nv_bfloat16* terms = (__nv_bfloat16*)((uint8_t*)workspace + space.grad);
    OP_TRY(op_launched(op, split_grad(grad, grad_dtype, step, rows, width, terms, space.wpad, st)));
    a = terms;
    a_stride = space.wpad * 2;
  }
  WeightArgs w = {};
  w.rows = rows;
  w.width = width;
  w.dim = (int32_t)dim;
  w.x = (const uint8_t*)x;
  w.x_stride = rows > 1 ? x_stride : int8_row_bytes(dim);
  w.row_bytes = (int32_t)int8_row_bytes(dim);
  w.ta = direct ? 1 : grad_terms(grad_dtype);
  w.partial = (float*)workspace;
  w.bias_partial = dbias ? (float*)((uint8_t*)workspace + space.bias) : nullptr;
  w.out = out;
  w.out_stride = out_step;
  w.dbias = dbias;
  w.status = status;
  space.shape(w);
  return op_launched(op, with_float_type(out_dtype, [&](auto t) {
    return launch_weight<typename decltype(t)::type>(
        w, a, a_stride, direct, (__nv_bfloat16*)((uint8_t*)workspace + space.values), device, st);
  }));
}

}  // extern "C"
