// embedding.cu -- rows of a learned embedding table, scaled, for a list of node
// ids, and the gradient of that lookup to the table (include/agnes_ops.h).
//
//   out[t] = scale * table[ids[t]]          d[v] = scale * sum_{ids[t] = v} grad[t]
//
// The gradient sorts the tokens by id, so that each row's tokens are adjacent,
// and sums them without atomics: cut into chunks of equal length, whatever the
// ids' distribution, a chunk writes the rows that lie within it and leaves its
// part of a row that spans chunks in the workspace; a last kernel joins those.
#include <type_traits>

#include "ops_common.cuh"

namespace agnes {

namespace {

// ---- lookup -----------------------------------------------------------------

constexpr int kLookupThreads = 256;
constexpr int kLookupItems = 4;  // vectors per thread, loaded before the first is stored
static_assert(kLookupThreads * kLookupItems == kFlat, "a block's vectors");

// A block takes kFlat vectors of kVec elements of the output in order.  vpr:
// vectors per row.
template <typename TIn, typename TOut, typename Id, int kVec>
__global__ void __launch_bounds__(kLookupThreads)
lookup_kernel(const TIn* __restrict__ table, int64_t rows, int64_t table_stride, int32_t vpr,
              uint32_t inv_vpr, const Id* __restrict__ ids, int64_t n, float scale,
              TOut* __restrict__ out, int64_t out_stride, int32_t* status) {
  const FlatRows flat(blockIdx.x, vpr, inv_vpr);
  int64_t token[kLookupItems], id[kLookupItems];
  uint32_t col[kLookupItems];
#pragma unroll
  for (int u = 0; u < kLookupItems; ++u) {
    flat.at(threadIdx.x + u * kLookupThreads, &token[u], &col[u]);
    id[u] = token[u] < n ? (int64_t)__ldg(ids + token[u]) : -1;
  }
  Vec<TIn, kVec> x[kLookupItems];
#pragma unroll
  for (int u = 0; u < kLookupItems; ++u) {
    if (id[u] >= 0 && id[u] < rows)
      x[u] = *(const Vec<TIn, kVec>*)(table + id[u] * table_stride + (int64_t)col[u] * kVec);
    else
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[u].v[e] = from_f32<TIn>(0.f);
  }
#pragma unroll
  for (int u = 0; u < kLookupItems; ++u) {
    if (token[u] >= n) continue;
    const bool real = id[u] >= 0 && id[u] < rows;
    Vec<TOut, kVec> y;
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      y.v[e] = from_f32<TOut>(real ? to_f32(x[u].v[e]) * scale : 0.f);
    *(Vec<TOut, kVec>*)(out + token[u] * out_stride + (int64_t)col[u] * kVec) = y;
    if (id[u] >= rows && col[u] == 0) op_flag(status, AGNES_OP_BAD_INDEX);
  }
}

// Rows that no wide vector divides (dim of 8 or more, the output contiguous): the output
// is one run of 16-byte vectors, each from one row or from the end of one and the start
// of the next, and the table's elements are loaded one by one, sixteen on their way to a
// thread.  (Element by element in the output too, four on their way: 498,000 fp16 rows of
// 301 363 us, now 183.)
template <typename TIn, typename TOut, typename Id>
__global__ void __launch_bounds__(kLookupThreads)
lookup_flat_kernel(const TIn* __restrict__ table, int64_t rows, int64_t table_stride, int32_t dim,
                   uint32_t inv_dim, const Id* __restrict__ ids, int64_t n, float scale,
                   TOut* __restrict__ out, int32_t* status) {
  constexpr int kN = 16 / sizeof(TOut);                        // elements of a vector
  constexpr int kVecs = 16 / kN;                               // vectors at a time
  constexpr int kTurns = kFlatRun / (kLookupThreads * 16);
  const FlatRun flat(blockIdx.x, dim, inv_dim);
  const int64_t total = n * dim;
#pragma unroll 1
  for (int turn = 0; turn < kTurns; ++turn) {
    TIn x[kVecs][kN];
    int valid[kVecs];  // a bit for each element that has a row
    int64_t at[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const uint32_t i = (uint32_t)(((turn * kVecs + v) * kLookupThreads + threadIdx.x) * kN);
      int64_t row;
      uint32_t col;
      flat.at(i, &row, &col);
      at[v] = (int64_t)blockIdx.x * kFlatRun + i;
      const int left = (int)(dim - col);  // elements of this row
      const int64_t id0 = row < n ? (int64_t)__ldg(ids + row) : -1;
      const int64_t id1 = left < kN && row + 1 < n ? (int64_t)__ldg(ids + row + 1) : -1;
      const bool real0 = id0 >= 0 && id0 < rows, real1 = id1 >= 0 && id1 < rows;
      if (id0 >= rows && col < kN) op_flag(status, AGNES_OP_BAD_INDEX);
      const TIn* p0 = table + id0 * table_stride + col;
      const TIn* p1 = table + id1 * table_stride - left;
      valid[v] = 0;
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        const bool real = e < left ? real0 : real1;
        x[v][e] = from_f32<TIn>(0.f);
        if (real) x[v][e] = (e < left ? p0 : p1)[e];
        valid[v] |= (int)real << e;
      }
    }
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      Vec<TOut, kN> y;
#pragma unroll
      for (int e = 0; e < kN; ++e)
        y.v[e] = from_f32<TOut>(valid[v] >> e & 1 ? to_f32(x[v][e]) * scale : 0.f);
      if (at[v] + kN <= total) {
        *(Vec<TOut, kN>*)(out + at[v]) = y;
      } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
          if (at[v] + e < total) out[at[v] + e] = y.v[e];
      }
    }
  }
}

// ---- the stable sort of the tokens by id -------------------------------------
//
// Least significant digit first, kDigits at most 2^kMaxBits, three launches a
// pass: each CTA counts the digits of its run of tokens; the counts of one
// digit are scanned over the CTAs; each CTA puts its tokens in their places,
// in order.  Keys are ids in [0, rows), and `rows` for the tokens that select
// none.

constexpr int kSortThreads = 256;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 8;
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kSmallTile = kSortThreads * 16;  // where one CTA sorts them all
constexpr int kMaxBits = 9;
constexpr int kMaxDigits = 1 << kMaxBits;
constexpr int kSortMaxCtas = 608;

template <typename Id>
__device__ __forceinline__ uint32_t key_of(Id id, int64_t rows, int32_t* status) {
  if (id < 0) return (uint32_t)rows;
  if ((int64_t)id >= rows) {
    op_flag(status, AGNES_OP_BAD_INDEX);
    return (uint32_t)rows;
  }
  return (uint32_t)id;
}

// What the gradient of a table without rows has to do: every id that selects a row is past
// its end.
template <typename Id>
__global__ void __launch_bounds__(kSortThreads)
any_id_kernel(const Id* __restrict__ ids, int64_t n, int32_t* status) {
  const int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x;
  if (__syncthreads_or(i < n && ids[i] >= 0) && threadIdx.x == 0)
    op_flag(status, AGNES_OP_BAD_INDEX);
}

// Where a pass reads its keys: the caller's ids (the first pass), or the last
// pass's.
template <typename Id>
struct FromIds {
  const Id* ids;
  int64_t rows;
  int32_t* status;
  __device__ uint32_t key(int64_t i) const { return key_of(__ldg(ids + i), rows, status); }
  __device__ int32_t token(int64_t i) const { return (int32_t)i; }
};
struct FromPass {
  const uint32_t* keys;
  const int32_t* tokens;
  __device__ uint32_t key(int64_t i) const { return keys[i]; }
  __device__ int32_t token(int64_t i) const { return tokens[i]; }
};

struct Run {
  int64_t begin, end;
};

// CTA b's run of tokens: whole tiles.
__device__ __forceinline__ Run run_of(int64_t n, int b, int ctas) {
  const int64_t tiles = (n + kSortTile - 1) / kSortTile;
  const int64_t lo = tiles * b / ctas * kSortTile, hi = tiles * (b + 1) / ctas * kSortTile;
  return {lo, hi < n ? hi : n};
}

// counts[digit * ctas + cta]
template <typename Src>
__global__ void __launch_bounds__(kSortThreads)
sort_count_kernel(Src src, int64_t n, int shift, int digits, int32_t* __restrict__ counts) {
  grid_dep_wait();
  let_next_start();
  __shared__ int32_t hist[kMaxDigits];
  for (int d = threadIdx.x; d < digits; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  const Run run = run_of(n, blockIdx.x, gridDim.x);
  for (int64_t base = run.begin; base < run.end; base += kSortTile) {
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
      const int64_t i = base + u * kSortThreads + threadIdx.x;
      const bool in = i < run.end;
      if (in) atomicAdd(hist + ((src.key(i) >> shift) & (uint32_t)(digits - 1)), 1);
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads)
    counts[(int64_t)d * gridDim.x + blockIdx.x] = hist[d];
}

// A warp per digit: its counts become their exclusive prefix over the CTAs, and
// totals[digit] their sum.  A lane takes neighbouring CTAs' counts, all on their way at
// once.
constexpr int kScanItems = kSortMaxCtas / 32;
static_assert(kSortMaxCtas % 32 == 0, "whole lanes");

__global__ void __launch_bounds__(256)
sort_scan_kernel(int32_t* __restrict__ counts, int ctas, int digits, int32_t* __restrict__ totals) {
  grid_dep_wait();
  let_next_start();
  const int d = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (d >= digits) return;
  int32_t* row = counts + (int64_t)d * ctas;
  const int per = (ctas + 31) / 32, first = lane_id() * per;
  int32_t v[kScanItems], sum = 0;
#pragma unroll
  for (int j = 0; j < kScanItems; ++j) v[j] = j < per && first + j < ctas ? row[first + j] : 0;
#pragma unroll
  for (int j = 0; j < kScanItems; ++j) sum += v[j];
  const int32_t incl = warp_incl_scan(sum);
  int32_t at = incl - sum;
#pragma unroll
  for (int j = 0; j < kScanItems; ++j) {
    if (j < per && first + j < ctas) row[first + j] = at;
    at += v[j];
  }
  if (lane_id() == 31) totals[d] = incl;
}

struct alignas(16) SortSmem {
  int32_t warp_hist[kSortWarps][kMaxDigits];
  int32_t base[kMaxDigits];   // where the next token of each digit goes
  int32_t delta[kMaxDigits];  // from a token's place in its tile to where it goes
  int32_t warp_total[kSortWarps];
};

// base[d] = the exclusive prefix over the digits of total(d), plus extra(d).  A thread
// has digits 2 t and 2 t + 1.
constexpr int kThreadDigits = kMaxDigits / kSortThreads;
static_assert(kThreadDigits == 2, "two digits to a thread");

template <typename Total, typename Extra>
__device__ __forceinline__ void digit_bases(SortSmem& s, int digits, Total total, Extra extra) {
  const int t = threadIdx.x, d = 2 * t;
  const bool in = d < digits;  // an even number
  const int32_t first = in ? total(d) : 0, second = in ? total(d + 1) : 0;
  const int32_t more = in ? extra(d) : 0, more2 = in ? extra(d + 1) : 0;
  const int32_t incl = warp_incl_scan(first + second);
  if (lane_id() == 31) s.warp_total[t >> 5] = incl;
  __syncthreads();
  int32_t before = incl - first - second;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) before += w < t >> 5 ? s.warp_total[w] : 0;
  if (in) {
    s.base[d] = before + more;
    s.base[d + 1] = before + first + more2;
  }
}

// The lanes with this lane's digit, by a ballot for each of its bits.
__device__ __forceinline__ unsigned same_digit(int digit, int bits) {
  unsigned peers = __ballot_sync(0xffffffffu, digit >= 0);
  for (int b = 0; b < bits; ++b) {
    const bool set = (digit >> b) & 1;
    const unsigned with = __ballot_sync(0xffffffffu, set);
    peers &= set ? with : ~with;
  }
  return peers;
}

// The places of a tile's tokens among themselves, sorted by digit, in order: warp w
// holds tokens w * 32 * kItems + u * 32 + lane.  s.delta: what leads from there to where
// the digit's tokens go; s.base moves on by the tile's counts.  All threads take part; a
// token out of the run has digit -1.
template <int kItems>
__device__ __forceinline__ void tile_places(SortSmem& s, int bits, const int (&digit)[kItems],
                                            int32_t (&place)[kItems]) {
  const int warp = threadIdx.x >> 5, digits = 1 << bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads)
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) s.warp_hist[w][d] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const unsigned peers = same_digit(digit[u], bits);
    int32_t old = 0;
    if (digit[u] >= 0) old = s.warp_hist[warp][digit[u]];
    place[u] = old + __popc(peers & ((1u << lane_id()) - 1u));
    __syncwarp();
    if (digit[u] >= 0 && lane_id() == __ffs(peers) - 1)
      s.warp_hist[warp][digit[u]] = old + __popc(peers);
    __syncwarp();
  }
  __syncthreads();
  const int d = 2 * threadIdx.x;
  const bool in = d < digits;  // an even number
  int2 c[kSortWarps], sum = make_int2(0, 0);
  if (in) {
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      c[w] = *(const int2*)&s.warp_hist[w][d];
      sum.x += c[w].x;
      sum.y += c[w].y;
    }
  }
  const int32_t incl = warp_incl_scan(sum.x + sum.y);
  if (lane_id() == 31) s.warp_total[warp] = incl;
  __syncthreads();
  int32_t before = incl - sum.x - sum.y;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) before += w < warp ? s.warp_total[w] : 0;
  if (in) {
    int2 at = make_int2(before, before + sum.x);
    const int2 base = *(const int2*)&s.base[d];
    *(int2*)&s.delta[d] = make_int2(base.x - at.x, base.y - at.y);
    *(int2*)&s.base[d] = make_int2(base.x + sum.x, base.y + sum.y);
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      *(int2*)&s.warp_hist[w][d] = at;
      at.x += c[w].x;
      at.y += c[w].y;
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kItems; ++u)
    if (digit[u] >= 0) place[u] += s.warp_hist[warp][digit[u]];
}

template <typename Src>
__global__ void __launch_bounds__(kSortThreads)
sort_place_kernel(Src src, int64_t n, int shift, int bits, const int32_t* __restrict__ counts,
                  const int32_t* __restrict__ totals, uint32_t* __restrict__ keys,
                  int32_t* __restrict__ tokens) {
  grid_dep_wait();
  let_next_start();
  __shared__ SortSmem s;
  // a tile's tokens in the order of their digits, so that those of one digit are stored
  // side by side
  __shared__ uint2 sorted[kSortTile];
  const int digits = 1 << bits;
  digit_bases(s, digits, [&](int d) { return totals[d]; },
              [&](int d) { return counts[(int64_t)d * gridDim.x + blockIdx.x]; });
  const Run run = run_of(n, blockIdx.x, gridDim.x);
  const int first = (threadIdx.x >> 5) * 32 * kSortItems + lane_id();
  for (int64_t base = run.begin; base < run.end; base += kSortTile) {
    uint32_t key[kSortItems];
    int32_t token[kSortItems], place[kSortItems];
    int digit[kSortItems];
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
      const int64_t i = base + first + u * 32;
      const bool in = i < run.end;
      key[u] = in ? src.key(i) : 0;
      token[u] = in ? src.token(i) : 0;
      digit[u] = in ? (int)(key[u] >> shift) & (digits - 1) : -1;
    }
    __syncthreads();  // the bases, and the last tile's places, have been read
    tile_places(s, bits, digit, place);
#pragma unroll
    for (int u = 0; u < kSortItems; ++u)
      if (digit[u] >= 0) sorted[place[u]] = make_uint2(key[u], (uint32_t)token[u]);
    __syncthreads();
    const int count = (int)min((int64_t)kSortTile, run.end - base);
    for (int i = threadIdx.x; i < count; i += kSortThreads) {
      const uint2 e = sorted[i];
      const int32_t to = i + s.delta[(e.x >> shift) & (uint32_t)(digits - 1)];
      keys[to] = e.x;
      tokens[to] = (int32_t)e.y;
    }
  }
}

constexpr int kMinChunk = 32;
constexpr int kRunChunks = 128;  // chunks whose ranks one CTA counts
static_assert(kSmallTile <= kMinChunk * kRunChunks, "the small sort's tokens are one run");

// Tokens per chunk where one CTA sorts them: fewer where there are few, so that their
// rows are summed by more warps, but always one run of chunks.
__host__ __device__ inline int small_chunk(int64_t n) {
  return n <= 8 * kRunChunks ? 8 : n <= 16 * kRunChunks ? 16 : kMinChunk;
}

// Up to kSmallTile tokens in one CTA, every pass in shared memory; with rank_of and
// heads, what count_heads_kernel finds, too (one run of chunks of small_chunk(n)).
template <typename Id, int kSmallItems>
__global__ void __launch_bounds__(kSortThreads)
sort_small_kernel(FromIds<Id> src, int n, int passes, int bits, uint32_t* __restrict__ keys,
                  int32_t* __restrict__ tokens, int32_t* __restrict__ rank_of,
                  int32_t* __restrict__ heads) {
  extern __shared__ __align__(16) uint8_t small_smem[];
  SortSmem& s = *(SortSmem*)small_smem;
  uint32_t* skey = (uint32_t*)(small_smem + sizeof(SortSmem));
  int32_t* stoken = (int32_t*)(skey + kSmallTile);
  const int first = (threadIdx.x >> 5) * 32 * kSmallItems + lane_id();
  const int digits = 1 << bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) s.base[d] = 0;
  uint32_t key[kSmallItems];
  int32_t token[kSmallItems], place[kSmallItems];
#pragma unroll
  for (int u = 0; u < kSmallItems; ++u) {
    const int i = first + u * 32;
    key[u] = i < n ? src.key(i) : 0;
    token[u] = i;
  }
  for (int p = 0; p < passes; ++p) {
    int digit[kSmallItems];
#pragma unroll
    for (int u = 0; u < kSmallItems; ++u)
      digit[u] = first + u * 32 < n ? (int)(key[u] >> (p * bits)) & (digits - 1) : -1;
    tile_places(s, bits, digit, place);
#pragma unroll
    for (int u = 0; u < kSmallItems; ++u) {
      if (digit[u] < 0) continue;
      skey[place[u]] = key[u];
      stoken[place[u]] = token[u];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSmallItems; ++u) {
      const int i = first + u * 32;
      if (i < n) {
        key[u] = skey[i];
        token[u] = stoken[i];
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < kSmallItems; ++u) {
    const int i = first + u * 32;
    if (i < n) {
      keys[i] = key[u];
      tokens[i] = token[u];
    }
  }
  if (!heads) return;
  // s.base: the ids that begin in each chunk
  const int chunk = small_chunk(n), chunks = (n + chunk - 1) / chunk, each = 32 / chunk;
  for (int g = threadIdx.x >> 5; g * 32 < n; g += kSortWarps) {  // 32 tokens, `each` chunks
    const int i = g * 32 + lane_id();
    const uint32_t k = i < n ? skey[i] : 0;
    const bool head = i < n && k < (uint32_t)src.rows && (i == 0 || skey[i - 1] != k);
    const unsigned heads_here = __ballot_sync(0xffffffffu, head);
    if (lane_id() < each)
      s.base[g * each + lane_id()] =
          __popc(heads_here >> (lane_id() * chunk) & (0xffffffffu >> (32 - chunk)));
  }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  int32_t before = 0;
  for (int c0 = 0; c0 < chunks; c0 += 32) {
    const int c = c0 + lane_id();
    const int32_t count = c < chunks ? s.base[c] : 0;
    const int32_t incl = warp_incl_scan(count);
    if (c < chunks) rank_of[c] = before + incl - count;
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane_id() == 0) heads[0] = before;
}
constexpr size_t kSmallSmem = sizeof(SortSmem) + 8 * kSmallTile;

// ---- sums over the sorted tokens ----------------------------------------------

constexpr int kSumThreads = 256;
constexpr uint32_t kPastChunk = 0xffffffffu;  // no id
constexpr int32_t kNoPart = -1, kAllOfIt = -2;  // instead of a row

// rank_of[c] = the number of distinct ids that begin in the chunks of c's run before
// c; heads[r] = those that begin in run r.  A warp to a chunk.
__global__ void __launch_bounds__(1024)
count_heads_kernel(const uint32_t* __restrict__ keys, int64_t n, uint32_t rows, int32_t chunk,
                   int64_t chunks, int32_t* __restrict__ rank_of, int32_t* __restrict__ heads) {
  grid_dep_wait();
  let_next_start();
  __shared__ int32_t count[kRunChunks], warp_total[4];
  const int warp = threadIdx.x >> 5, lane = lane_id();
  const int64_t c0 = (int64_t)blockIdx.x * kRunChunks;
  for (int c = warp; c < kRunChunks; c += 32) {
    const int64_t lo = min(n, (c0 + c) * chunk), hi = min(n, lo + chunk);
    int32_t mine = 0;
    for (int64_t i = lo + lane; i < hi; i += 32) {
      const uint32_t k = keys[i];
      mine += k < rows && (i == 0 || keys[i - 1] != k);
    }
    mine = warp_sum(mine);
    if (lane == 0) count[c] = mine;
  }
  __syncthreads();
  const int t = threadIdx.x;
  int32_t incl = 0, mine = 0;
  if (t < kRunChunks) {
    mine = count[t];
    incl = warp_incl_scan(mine);
    if (lane == 31) warp_total[warp] = incl;
  }
  __syncthreads();
  if (t >= kRunChunks) return;
  for (int w = 0; w < warp; ++w) incl += warp_total[w];
  if (c0 + t < chunks) rank_of[c0 + t] = incl - mine;
  if (t == kRunChunks - 1) heads[blockIdx.x] = incl;
}

struct SumArgs {
  const uint32_t* keys;
  const int32_t* tokens;
  int64_t n;
  uint32_t rows;
  int32_t dim;
  const void* grad;
  int64_t grad_stride;
  float scale;
  void* out;
  // the compact form (null: dense, row v of `out` is d[v])
  const int32_t* heads;  // per run of kRunChunks chunks: ids that begin in it
  int32_t runs;
  int32_t* out_ids;
  int32_t* count;
  int32_t* rank_of;  // per chunk: ids that begin in its run before it
  // per chunk: which row of `out` its part 1 belongs to, kNoPart, or kAllOfIt where the
  // whole chunk is in the middle of a row
  int32_t* row_of;
  // a chunk's part of the row that it begins within (which = 0) and of the row that
  // it ends within (1): partial[(2 * chunk + which) * part_dim ..]
  float* partial;
  int32_t part_dim;    // dim up to a multiple of 4
  int32_t chunk;       // tokens per chunk
  int64_t chunks;

  __device__ float* part(int64_t c, int which) const {
    return partial + (2 * c + which) * part_dim;
  }
  __device__ uint32_t first_key(int64_t c) const { return keys[c * chunk]; }
};

// The sum of heads[0 .. limit) for this CTA, and of all of them.
__device__ __forceinline__ void prefix_of_heads(const int32_t* heads, int runs, int limit,
                                                int32_t* before, int32_t* all) {
  __shared__ int32_t sum[2][kSumThreads / 32];
  int32_t b = 0, a = 0;
  for (int i = threadIdx.x; i < runs; i += kSumThreads) {
    const int32_t h = heads[i];
    a += h;
    b += i < limit ? h : 0;
  }
  a = warp_sum(a);
  b = warp_sum(b);
  if (lane_id() == 0) {
    sum[0][threadIdx.x >> 5] = b;
    sum[1][threadIdx.x >> 5] = a;
  }
  __syncthreads();
  a = b = 0;
#pragma unroll
  for (int w = 0; w < kSumThreads / 32; ++w) {
    b += sum[0][w];
    a += sum[1][w];
  }
  *before = b;
  *all = a;
}

// A group of kLanes lanes sums a chunk's rows for kLanes * kVec * kCols columns.
// blockIdx.y: which columns.  Each lane holds the key and place of one token of this
// round of kLanes tokens and of the next round; kDepth rows are on their way at any
// time.  Rows that are loaded two bytes at a time are asked for in L2 when their token
// is known (498,000 fp16 rows of 301: 238 us, 271 without); others are not, as whole
// 128-byte lines come that are partly not theirs or not there any more when they are
// used (1.17M of 128: 221 us, 237 with; 234,000 fp32 rows of 640: 252 and 306).
//
// Bound by instructions as much as by memory, so a token costs as few as possible:
// where rows begin is a mask, found for a round at once; an address is one multiply
// and add; lanes and tokens without a value load a valid one and store nothing.  Warps
// hide the loads' latency better than rows in flight: with two rows each and six CTAs an
// SM (three for ten columns a lane) this kernel takes 108 us of 1.0M fp16 rows of 128
// over 10M nodes and 70 of 300,001 x 301 bf16; with four rows and as many CTAs as the
// registers allow 118 and 76.
template <typename TIn, typename TOut, int kVec, int kCols, int kLanes>
__global__ void __launch_bounds__(kSumThreads, kCols > 4 ? 3 : 6) sum_kernel(SumArgs a) {
  grid_dep_wait();
  let_next_start();
  constexpr int kGroups = kSumThreads / kLanes;
  constexpr int kDepth = 2;
  constexpr int kTileCols = kLanes * kVec * kCols;
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const int shift = threadIdx.x % 32 / kLanes * kLanes;  // of the group within its warp
  const unsigned lanes = kLanes == 32 ? 0xffffffffu : ((1u << (kLanes & 31)) - 1u) << shift;
  const int64_t chunk = (int64_t)blockIdx.x * kGroups + group;
  const int64_t lo = min(a.n, chunk * a.chunk), hi = min(a.n, lo + a.chunk);
  const int32_t tile_col = blockIdx.y * kTileCols, col0 = tile_col + lane * kVec;
  const uint32_t in_bytes = (uint32_t)(a.grad_stride * (int64_t)sizeof(TIn));
  const uint32_t out_bytes = (uint32_t)(a.dim * (int32_t)sizeof(TOut));
  const char* in[kCols];
#pragma unroll
  for (int c = 0; c < kCols; ++c) {
    const int32_t col = col0 + c * kLanes * kVec;
    in[c] = (const char*)a.grad + (int64_t)(col < a.dim ? col : 0) * (int64_t)sizeof(TIn);
  }
  char* const out = (char*)a.out + (int64_t)col0 * (int64_t)sizeof(TOut);
  const int32_t tile_bytes = min(kTileCols, a.dim - tile_col) * (int32_t)sizeof(TIn);

  // The key and token of place i for this lane; a token without a row to read (past
  // the chunk, or padding) becomes token 0, whose row is read and not used.
  const auto fetch = [&](int64_t i, uint32_t& k, uint32_t& token) {
    k = i < hi ? a.keys[i] : kPastChunk;
    token = k < a.rows ? (uint32_t)a.tokens[i] : 0u;
    if (k >= a.rows) return;
    const char* row = (const char*)a.grad + (uint64_t)token * in_bytes +
                      (int64_t)tile_col * (int64_t)sizeof(TIn);
    if constexpr (kVec == 1)
      for (int32_t b = 0; b < tile_bytes; b += 128)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(row + b));
  };
  // before the ranks: the chain from a token to its row is the longest
  uint32_t held_key, next_key, held_token, next_token;
  fetch(lo + lane, held_key, held_token);
  fetch(lo + kLanes + lane, next_key, next_token);
  uint32_t rank = 0;  // of the next row to begin, among the distinct ids
  if (a.heads) {
    int32_t before, all;
    prefix_of_heads(a.heads, a.runs, (int)((int64_t)blockIdx.x * kGroups / kRunChunks), &before,
                    &all);
    if (chunk < a.chunks) rank = before + a.rank_of[chunk];
    if (blockIdx.y == 0) {  // the ids and zeros past the last row, the CTAs' shares in turn
      const int64_t share = (a.n - all + gridDim.x - 1) / gridDim.x;
      const int64_t p0 = min(a.n, all + share * blockIdx.x), p1 = min(a.n, p0 + share);
      for (int64_t i = p0 + threadIdx.x; i < p1; i += kSumThreads) a.out_ids[i] = -1;
      if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = all;
      Vec<TOut, kVec> z;
#pragma unroll
      for (int e = 0; e < kVec; ++e) z.v[e] = from_f32<TOut>(0.f);
      Vec<TOut, kVec>* to = (Vec<TOut, kVec>*)((TOut*)a.out + p0 * a.dim);
      const int64_t vecs = (p1 - p0) * (a.dim / kVec);
      for (int64_t i = threadIdx.x; i < vecs; i += kSumThreads) to[i] = z;
    }
  }
  if (lo >= hi) return;
  uint32_t key = __shfl_sync(lanes, held_key, 0, kLanes);
  const auto leave = [&](int32_t what) {
    if (blockIdx.y == 0 && lane == 0) a.row_of[chunk] = what;
  };
  if (key >= a.rows) {  // padding only
    leave(kNoPart);
    return;
  }
  const bool goes_on = hi < a.n && a.keys[hi] == a.keys[hi - 1];  // past the chunk
  bool spans = lo > 0 && a.keys[lo - 1] == key;  // the current row began in an earlier chunk

  float acc[kCols][kVec];
  const auto clear = [&] {
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
      for (int e = 0; e < kVec; ++e) acc[c][e] = 0.f;
  };
  const auto put_row = [&](uint32_t row) {
    char* to = out + (uint64_t)row * out_bytes;
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      if (col0 + c * kLanes * kVec >= a.dim) break;
      Vec<TOut, kVec> y;
#pragma unroll
      for (int e = 0; e < kVec; ++e) y.v[e] = from_f32<TOut>(acc[c][e] * a.scale);
      *(Vec<TOut, kVec>*)(to + c * kLanes * kVec * (int)sizeof(TOut)) = y;
    }
  };
  const auto put_part = [&](int which) {
    constexpr int kN = kVec < 4 ? kVec : 4;
    float* p = a.part(chunk, which);
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      const int32_t col = col0 + c * kLanes * kVec;
      if (col >= a.dim) break;
#pragma unroll
      for (int h = 0; h < kVec / kN; ++h) {
        Vec<float, kN> y;
#pragma unroll
        for (int e = 0; e < kN; ++e) y.v[e] = acc[c][h * kN + e];
        *(Vec<float, kN>*)(p + col + h * kN) = y;
      }
    }
  };
  Vec<TIn, kVec> x[kDepth][kCols];
  const auto load = [&](uint32_t token, Vec<TIn, kVec>(&to)[kCols]) {
#pragma unroll
    for (int c = 0; c < kCols; ++c)
      to[c] = *(const Vec<TIn, kVec>*)(in[c] + (uint64_t)token * in_bytes);
  };
  // The places of a round where a key begins, as a mask; a compact row's id is put
  // down where it begins.
  const auto begins = [&](uint32_t k, uint32_t before_round) {
    uint32_t before = __shfl_up_sync(lanes, k, 1, kLanes);
    if (lane == 0) before = before_round;
    const bool begin = k != before;
    const unsigned mask = (__ballot_sync(lanes, begin) >> shift);
    if (a.heads && blockIdx.y == 0 && begin && k < a.rows)
      a.out_ids[rank + __popc(mask & ((1u << lane) - 1u))] = (int32_t)k;
    return mask;
  };
#pragma unroll
  for (int d = 0; d < kDepth; ++d) load(__shfl_sync(lanes, held_token, d, kLanes), x[d]);
  unsigned mask = begins(held_key, spans ? key : kPastChunk);
  uint32_t row = a.heads ? rank : key;  // of the output; a spanning row's is not used
  if (!spans) ++rank;
  mask &= ~1u;  // the first row has begun
  clear();
  const int32_t count = (int32_t)(hi - lo);
#pragma unroll 1
  for (int32_t j = 0; j < count; j += kDepth) {
    const int at0 = j % kLanes;  // a round is a multiple of kDepth
    if (at0 == 0 && j > 0) {
      const uint32_t before = __shfl_sync(lanes, held_key, kLanes - 1, kLanes);
      held_key = next_key;
      held_token = next_token;
      mask = begins(held_key, before);
      fetch(lo + j + kLanes + lane, next_key, next_token);
    }
    const uint32_t source = at0 + kDepth < kLanes ? held_token : next_token;
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (d > 0 && j + d >= count) break;
      if ((mask >> (at0 + d)) & 1u) {
        if (spans)
          put_part(0);
        else
          put_row(row);
        spans = false;
        clear();
        key = __shfl_sync(lanes, held_key, at0 + d, kLanes);
        if (key >= a.rows) {  // the rest is padding
          leave(kNoPart);
          return;
        }
        row = a.heads ? rank : key;
        ++rank;
      }
#pragma unroll
      for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int e = 0; e < kVec; ++e) acc[c][e] += to_f32(x[d][c].v[e]);
      load(__shfl_sync(lanes, source, (at0 + kDepth + d) % kLanes, kLanes), x[d]);
    }
  }
  if (spans)
    put_part(0);
  else if (goes_on)
    put_part(1);
  else
    put_row(row);
  leave(!goes_on ? kNoPart : spans ? kAllOfIt : (int32_t)row);
}

// Rows that span chunks.  Such a row has part 1 of the chunk in which it begins and
// part 0 of each later one.  Where kFold chunks from a multiple of kFold on are all
// within one row, their parts are first summed into the first one's (fold_kernel),
// so that a row of any length has few parts left.
constexpr int kFold = 64;
constexpr int kJoinCols = 128;  // columns per CTA, four to a lane

__device__ __forceinline__ void add4(float4& s, const float4& x) {
  s.x += x.x;
  s.y += x.y;
  s.z += x.z;
  s.w += x.w;
}

// The sum over i in [first, count) in steps of `step` of item(i)'s four columns.
template <typename Item>
__device__ __forceinline__ float4 sum_items(int64_t first, int64_t count, int step, Item item) {
  constexpr int kAhead = 8;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  int64_t i = first;
  for (; i + (kAhead - 1) * step < count; i += kAhead * step) {
    float4 x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = *(const float4*)item(i + u * step);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) add4(s, x[u]);
  }
  for (; i < count; i += step) add4(s, *(const float4*)item(i));
  return s;
}

constexpr int kFoldThreads = 256;

__global__ void __launch_bounds__(kFoldThreads) fold_kernel(SumArgs a) {
  grid_dep_wait();
  let_next_start();
  __shared__ float4 part[kFoldThreads / 32][32];
  const int64_t c0 = (int64_t)blockIdx.x * kFold;
  if (c0 == 0 || c0 + kFold > a.chunks) return;
  const uint32_t key = a.keys[c0 * a.chunk - 1];
  if (key >= a.rows || a.first_key(c0 + kFold - 1) != key) return;
  const int warp = threadIdx.x >> 5;
  const int32_t col = blockIdx.y * kJoinCols + lane_id() * 4;
  const bool in = col < a.part_dim;
  if (in)
    part[warp][lane_id()] = sum_items(warp, kFold, kFoldThreads / 32,
                                      [&](int64_t i) { return a.part(c0 + i, 0) + col; });
  __syncthreads();
  if (warp == 0 && in) {
    float4 s = part[0][lane_id()];
    for (int w = 1; w < kFoldThreads / 32; ++w) add4(s, part[w][lane_id()]);
    *(float4*)(a.part(c0, 0) + col) = s;
  }
}

// The parts of the row that begins in chunk `own` and goes on to chunk `last`.
struct Parts {
  int64_t own, last, count;
  int64_t fold0, folds;  // the first folded chunk, and how many runs of kFold

  __device__ Parts() {}
  __device__ Parts(int64_t own_, int64_t last_) : own(own_), last(last_) {
    fold0 = (own + kFold) / kFold * kFold;  // the first multiple of kFold past own
    folds = last + 1 > fold0 ? (last + 1 - fold0) / kFold : 0;
    count = last - own + 1 - folds * (kFold - 1);
  }
  __device__ const float* at(const SumArgs& a, int64_t i) const {
    if (i == 0) return a.part(own, 1);
    int64_t c = own + i;
    if (folds > 0 && c > fold0) {
      const int64_t f = c - fold0;  // folded runs count as one
      c = f < folds ? fold0 + f * kFold : fold0 + folds * kFold + (f - folds);
    }
    return a.part(c, 0);
  }
};

// Few warps to a CTA: those without a row leave early (128 threads: the join of 1.0M
// tokens 13 us, 512: 19).
constexpr int kJoinThreads = 128;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kJoinAlone = 32;  // parts that a warp sums by itself

// A warp for each chunk in which a row begins that goes on past it; the CTA
// together where the row has many parts.
template <typename TOut>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(SumArgs a) {
  grid_dep_wait();
  let_next_start();
  __shared__ Parts all[kJoinWarps];
  __shared__ int64_t row_of[kJoinWarps];
  __shared__ float4 part[kJoinWarps][32];
  const int warp = threadIdx.x >> 5, lane = lane_id();
  const int64_t chunk = (int64_t)blockIdx.x * kJoinWarps + warp;
  const int32_t col = blockIdx.y * kJoinCols + lane * 4;
  const auto put = [&](int64_t row, const float4& s) {
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < a.dim) ((TOut*)a.out)[row * a.dim + col + e] = from_f32<TOut>(v[e] * a.scale);
  };
  int64_t many = -1;  // the row, where the CTA sums it
  Parts parts;
  const int32_t row = chunk < a.chunks ? a.row_of[chunk] : kNoPart;
  if (row >= 0) {
    // the last chunk of the row: the first after this one that it does not fill
    int64_t last = chunk + 1;
    const int64_t c = last + lane;
    const unsigned ends =
        __ballot_sync(0xffffffffu, c >= a.chunks || a.row_of[c] != kAllOfIt);
    if (ends) {
      last += __ffs(ends) - 1;
    } else {  // a long row: the last chunk that begins with its key
      const uint32_t key = a.first_key(last);
      int64_t end = a.chunks;
      while (end - last > 1) {
        const int64_t mid = (last + end) / 2;
        if (a.first_key(mid) == key)
          last = mid;
        else
          end = mid;
      }
    }
    parts = Parts(chunk, last);
    if (parts.count > kJoinAlone)
      many = row;
    else if (col < a.part_dim)
      put(row, sum_items(0, parts.count, 1, [&](int64_t i) { return parts.at(a, i) + col; }));
  }
  if (lane == 0) {
    row_of[warp] = many;
    all[warp] = parts;
  }
  if (!__syncthreads_or(many >= 0)) return;
  for (int o = 0; o < kJoinWarps; ++o) {
    const int64_t row = row_of[o];
    if (row < 0) continue;
    const Parts p = all[o];
    if (col < a.part_dim)
      part[warp][lane] =
          sum_items(warp, p.count, kJoinWarps, [&](int64_t i) { return p.at(a, i) + col; });
    __syncthreads();
    if (warp == 0 && col < a.part_dim) {
      float4 s = part[0][lane];
      for (int w = 1; w < kJoinWarps; ++w) add4(s, part[w][lane]);
      put(row, s);
    }
    __syncthreads();
  }
}

// ---- host ------------------------------------------------------------------

constexpr int64_t kMaxTokens = 0x7fffffff;
constexpr int64_t kMaxCells = 1ll << 40;
constexpr int64_t kMaxDim = 1 << 22;  // its column tiles fit a grid's second dimension
constexpr int kMaxChunks = 65536;

struct GradPlan {
  int64_t chunk, chunks;
  size_t keys[2], tokens[2], counts, totals, heads, rank_of, row_of, partial, bytes;
};

GradPlan grad_plan(int64_t n, int64_t dim) {
  GradPlan p;
  p.chunk = ceil_div(ceil_div(n, kMaxChunks), kMinChunk) * kMinChunk;
  if (p.chunk < kMinChunk) p.chunk = kMinChunk;
  if (n <= kSmallTile) p.chunk = small_chunk(n);
  p.chunks = ceil_div(n, p.chunk);
  size_t at = 0;
  const auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)((bytes + 255) / 256 * 256);
    return here;
  };
  for (int i = 0; i < 2; ++i) {
    p.keys[i] = take(4 * n);
    p.tokens[i] = take(4 * n);
  }
  p.counts = take(4ll * kMaxDigits * kSortMaxCtas);
  p.totals = take(4 * kMaxDigits);
  p.heads = take(4 * ceil_div(p.chunks, kRunChunks));
  p.rank_of = take(4 * p.chunks);
  p.row_of = take(4 * p.chunks);
  p.partial = take(8 * p.chunks * (ceil_div(dim, 4) * 4));
  p.bytes = at;
  return p;
}

template <typename Id>
cudaError_t sort_tokens(const Id* ids, int64_t n, int64_t rows, uint8_t* ws, const GradPlan& p,
                        int32_t* status, int32_t* heads, int device, cudaStream_t st, int* result) {
  int bits = 1;
  while ((1ll << bits) <= rows) ++bits;  // keys 0 .. rows
  const int passes = (int)ceil_div(bits, kMaxBits);
  const int pass_bits = (int)ceil_div(bits, passes);
  const int digits = 1 << pass_bits;
  const FromIds<Id> ids_src{ids, rows, status};
  const auto keys = [&](int i) { return (uint32_t*)(ws + p.keys[i]); };
  const auto tokens = [&](int i) { return (int32_t*)(ws + p.tokens[i]); };
  if (n <= kSmallTile) {
    const auto run = [&](auto items) {
      constexpr int kItems = decltype(items)::value;
      static OncePerDevice once;
      const cudaError_t e = once.run(device, [] {
        return cudaFuncSetAttribute(sort_small_kernel<Id, kItems>,
                                    cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallSmem);
      });
      if (e != cudaSuccess) return e;
      sort_small_kernel<Id, kItems><<<1, kSortThreads, kSmallSmem, st>>>(
          ids_src, (int)n, passes, pass_bits, keys(0), tokens(0), (int32_t*)(ws + p.rank_of),
          heads);
      return cudaGetLastError();
    };
    *result = 0;
    if (n <= 4 * kSortThreads) return run(std::integral_constant<int, 4>());
    if (n <= 8 * kSortThreads) return run(std::integral_constant<int, 8>());
    return run(std::integral_constant<int, 16>());
  }
  const int64_t tiles = ceil_div(n, kSortTile);
  const int num_sms = op_num_sms(device);
  int ctas = 4 * num_sms < kSortMaxCtas ? 4 * num_sms : kSortMaxCtas;
  if (tiles < ctas) ctas = (int)tiles;
  int32_t* counts = (int32_t*)(ws + p.counts);
  int32_t* totals = (int32_t*)(ws + p.totals);
  cudaError_t e = cudaSuccess;
  for (int pass = 0; pass < passes && e == cudaSuccess; ++pass) {
    const int shift = pass * pass_bits, to = pass & 1;
    const FromPass from{keys(to ^ 1), tokens(to ^ 1)};
    if (pass == 0) {
      // after whatever the caller's stream ran before
      sort_count_kernel<<<ctas, kSortThreads, 0, st>>>(ids_src, n, shift, digits, counts);
      e = cudaGetLastError();
    } else {
      e = launch_next(sort_count_kernel<FromPass>, ctas, kSortThreads, 0, st, from, n, shift,
                      digits, counts);
    }
    if (e == cudaSuccess)
      e = launch_next(sort_scan_kernel, (digits + 7) / 8, 256, 0, st, counts, ctas, digits, totals);
    if (e != cudaSuccess) break;
    if (pass == 0)
      e = launch_next(sort_place_kernel<FromIds<Id>>, ctas, kSortThreads, 0, st, ids_src, n, shift,
                      pass_bits, counts, totals, keys(to), tokens(to));
    else
      e = launch_next(sort_place_kernel<FromPass>, ctas, kSortThreads, 0, st, from, n, shift,
                      pass_bits, counts, totals, keys(to), tokens(to));
    *result = to;
  }
  return e;
}

template <typename TIn, typename TOut, int kVec, int kCols, int kLanes>
cudaError_t launch_sum(SumArgs a, int32_t* heads, cudaStream_t st) {
  constexpr int kGroups = kSumThreads / kLanes;
  const int64_t ctas = ceil_div(a.chunks, kGroups);
  const int64_t cols = ceil_div(a.dim, kLanes * kVec * kCols);
  if (heads) {
    a.heads = heads;
    a.runs = (int32_t)ceil_div(a.chunks, kRunChunks);
    if (a.n > kSmallTile) {  // else the sort has counted them
      const cudaError_t e = launch_next(count_heads_kernel, (unsigned)a.runs, 1024, 0, st, a.keys,
                                        a.n, a.rows, a.chunk, a.chunks, a.rank_of, heads);
      if (e != cudaSuccess) return e;
    }
  }
  cudaError_t e = launch_next(sum_kernel<TIn, TOut, kVec, kCols, kLanes>,
                              dim3((unsigned)ctas, (unsigned)cols), kSumThreads, 0, st, a);
  const unsigned join_cols = (unsigned)ceil_div(a.dim, kJoinCols);
  if (e == cudaSuccess && a.chunks >= 2 * kFold)  // a whole run after the first
    e = launch_next(fold_kernel, dim3((unsigned)(a.chunks / kFold), join_cols), kFoldThreads, 0, st,
                    a);
  if (e == cudaSuccess && a.chunks > 1)
    e = launch_next(join_kernel<TOut>, dim3((unsigned)ceil_div(a.chunks, kJoinWarps), join_cols),
                    kJoinThreads, 0, st, a);
  return e;
}

// A warp to a row where the row has 32 columns or more: half a warp to a row has
// the two halves end their rows at different tokens, one after the other (1.0M fp16
// rows of 128, the whole gradient at the time: 4 columns a lane 258 us, 8 a lane in half
// a warp 265).  More columns a lane where a row is longer: of vectors of one or two
// elements 1, 2, 5 or 10, whichever is the first that covers the row (10 covers 301 single
// elements; lanes past the row's end load its first column and store nothing), of wider
// ones 1, 2 or 3.  What is longer takes several column tiles, each with a pass of its own
// over the tokens, of wide vectors with one column a lane (not measured against more).
template <typename TIn, typename TOut, int kVec>
cudaError_t launch_sum_lanes(const SumArgs& a, int32_t* heads, cudaStream_t st) {
  if constexpr (kVec > 1) {
    if (a.dim < 32 * kVec) return launch_sum_lanes<TIn, TOut, kVec / 2>(a, heads, st);
  } else {
    if (a.dim <= 4) return launch_sum<TIn, TOut, 1, 1, 4>(a, heads, st);
    if (a.dim <= 16) return launch_sum<TIn, TOut, 1, 1, 16>(a, heads, st);
  }
  const int64_t need = ceil_div(a.dim, 32 * kVec);  // columns a lane
  if constexpr (kVec <= 2) {
    if (need > 5) return launch_sum<TIn, TOut, kVec, 10, 32>(a, heads, st);
    if (need > 2) return launch_sum<TIn, TOut, kVec, 5, 32>(a, heads, st);
    if (need > 1) return launch_sum<TIn, TOut, kVec, 2, 32>(a, heads, st);
  } else {
    if (need == 2) return launch_sum<TIn, TOut, kVec, 2, 32>(a, heads, st);
    if (need == 3) return launch_sum<TIn, TOut, kVec, 3, 32>(a, heads, st);
  }
  return launch_sum<TIn, TOut, kVec, 1, 32>(a, heads, st);
}

// f(constant) for the widest vector of 8, 4, 2 or 1 elements (16 bytes at most of
// either type) that divides the rows and to which both arrays are aligned.
template <typename TA, typename TB, typename F>
cudaError_t with_vector(int64_t dim, const void* a, int64_t a_stride, const void* b,
                        int64_t b_stride, F&& f) {
  constexpr int kWide = 16 / (sizeof(TA) > sizeof(TB) ? sizeof(TA) : sizeof(TB));
  const auto fits = [&](int64_t v) {
    return dim % v == 0 && aligned_rows(a, a_stride * (int64_t)sizeof(TA), v * sizeof(TA)) &&
           aligned_rows(b, b_stride * (int64_t)sizeof(TB), v * sizeof(TB));
  };
  if (fits(kWide)) return f(std::integral_constant<int, kWide>());
  if constexpr (kWide > 4)
    if (fits(4)) return f(std::integral_constant<int, 4>());
  if (fits(2)) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}

// The checks that the lookup and the gradient share.
agnes_status check_embedding(const char* op, int64_t rows, int64_t dim, int64_t n,
                             int32_t ids_bits) {
  if (rows < 0 || n < 0 || dim < 1)
    return op_error(AGNES_EINVAL, "%s: rows %lld, dim %lld, n %lld", op, (long long)rows,
                    (long long)dim, (long long)n);
  if (rows > kMaxTokens || n > kMaxTokens || dim > kMaxDim || (n && dim > kMaxCells / n) ||
      (rows && dim > kMaxCells / rows))
    return op_error(AGNES_ERANGE, "%s: rows %lld, dim %lld, n %lld are too large", op,
                    (long long)rows, (long long)dim, (long long)n);
  return op_index_bits(op, "ids", ids_bits);
}

struct GradCall {
  const char* op;
  const void* grad;
  int32_t grad_dtype;
  int64_t grad_stride;
  const void* ids;
  int32_t ids_bits;
  int64_t n, rows, dim;
  float scale;
  void* out;
  int32_t out_dtype;
  int32_t* out_ids;  // the compact form's, with count
  int32_t* count;
  void* workspace;
  int64_t workspace_bytes;
  int32_t* status;
  cudaStream_t st;
};

// The dense gradient of a table without rows: nothing to write, ids past its end to report.
agnes_status report_ids(const GradCall& c) {
  const char* op = c.op;
  if (c.n == 0 || !c.status) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "ids", c.ids, &device));
  OP_TRY(op_aligned(op, "ids", c.ids, c.ids_bits / 8));
  OP_TRY(op_status(op, c.status, device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  return op_launched(op, with_index_type(c.ids_bits, [&](auto id) {
    using Id = typename decltype(id)::type;
    any_id_kernel<Id><<<(unsigned)ceil_div(c.n, kSortThreads), kSortThreads, 0, c.st>>>(
        (const Id*)c.ids, c.n, c.status);
    return cudaGetLastError();
  }));
}

agnes_status embedding_grad(const GradCall& c, bool compact) {
  const char* op = c.op;
  OP_TRY(check_embedding(op, c.rows, c.dim, c.n, c.ids_bits));
  OP_TRY(op_float_type(op, "grad", c.grad_dtype));
  OP_TRY(op_float_type(op, "out", c.out_dtype));
  if (c.n > 0 && c.grad_stride < c.dim)
    return op_error(AGNES_EINVAL, "%s: grad_stride %lld is below dim %lld", op,
                    (long long)c.grad_stride, (long long)c.dim);
  if (c.n > 1 && c.grad_stride * float_size(c.grad_dtype) > 0xffffffffll)
    return op_error(AGNES_ERANGE, "%s: grad_stride %lld is too large", op,
                    (long long)c.grad_stride);
  const int64_t out_rows = compact ? c.n : c.rows;
  int device = -1;
  if (compact) {
    OP_TRY(op_device_of(op, "count", c.count, &device));
    OP_TRY(op_aligned(op, "count", c.count, 4));
  } else if (out_rows == 0) {
    return report_ids(c);
  } else {
    OP_TRY(op_device_of(op, "out", c.out, &device));
  }
  if (out_rows > 0) {
    OP_TRY(op_on_device(op, "out", c.out, device));
    OP_TRY(op_aligned(op, "out", c.out, float_size(c.out_dtype)));
  }
  OP_TRY(op_status(op, c.status, device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  if (c.n == 0) {
    cudaError_t e;
    if (compact)
      e = cudaMemsetAsync(c.count, 0, 4, c.st);
    else
      e = cudaMemsetAsync(c.out, 0, (size_t)(c.rows * c.dim * float_size(c.out_dtype)), c.st);
    return op_launched(op, e);
  }
  OP_TRY(op_on_device(op, "grad", c.grad, device));
  OP_TRY(op_aligned(op, "grad", c.grad, float_size(c.grad_dtype)));
  OP_TRY(op_on_device(op, "ids", c.ids, device));
  OP_TRY(op_aligned(op, "ids", c.ids, c.ids_bits / 8));
  if (compact) {
    OP_TRY(op_on_device(op, "out_ids", c.out_ids, device));
    OP_TRY(op_aligned(op, "out_ids", c.out_ids, 4));
  }
  OP_TRY(op_on_device(op, "workspace", c.workspace, device));
  OP_TRY(op_aligned(op, "workspace", c.workspace, 256));
  const GradPlan p = grad_plan(c.n, c.dim);
  if (c.workspace_bytes < (int64_t)p.bytes)
    return op_error(AGNES_EINVAL, "%s: a workspace of %lld bytes, %lld are needed", op,
                    (long long)c.workspace_bytes, (long long)p.bytes);
  uint8_t* ws = (uint8_t*)c.workspace;
  int32_t* heads = compact ? (int32_t*)(ws + p.heads) : nullptr;
  int which = 0;
  if (!compact) {  // before the kernels, which then follow one another
    const cudaError_t e =
        cudaMemsetAsync(c.out, 0, (size_t)(c.rows * c.dim * float_size(c.out_dtype)), c.st);
    if (e != cudaSuccess) return op_launched(op, e);
  }
  cudaError_t e = with_index_type(c.ids_bits, [&](auto id) {
    using Id = typename decltype(id)::type;
    return sort_tokens((const Id*)c.ids, c.n, c.rows, ws, p, c.status, heads, device, c.st,
                       &which);
  });
  if (e != cudaSuccess) return op_launched(op, e);
  SumArgs a = {};
  a.keys = (const uint32_t*)(ws + p.keys[which]);
  a.tokens = (const int32_t*)(ws + p.tokens[which]);
  a.n = c.n;
  a.rows = (uint32_t)c.rows;
  a.dim = (int32_t)c.dim;
  a.grad = c.grad;
  a.grad_stride = c.n > 1 ? c.grad_stride : c.dim;
  a.scale = c.scale;
  a.out = c.out;
  a.out_ids = c.out_ids;
  a.count = c.count;
  a.rank_of = (int32_t*)(ws + p.rank_of);
  a.row_of = (int32_t*)(ws + p.row_of);
  a.partial = (float*)(ws + p.partial);
  a.part_dim = (int32_t)(ceil_div(c.dim, 4) * 4);
  a.chunk = (int32_t)p.chunk;
  a.chunks = p.chunks;
  e = with_float_type(c.grad_dtype, [&](auto tin) {
    return with_float_type(c.out_dtype, [&](auto tout) {
      using TIn = typename decltype(tin)::type;
      using TOut = typename decltype(tout)::type;
      return with_vector<TIn, TOut>(c.dim, c.grad, c.grad_stride, c.out, c.dim, [&](auto v) {
        return launch_sum_lanes<TIn, TOut, decltype(v)::value>(a, heads, c.st);
      });
    });
  });
  return op_launched(op, e);
}

}  // namespace

}  // namespace agnes

using namespace agnes;

extern "C" {

agnes_status agnes_embedding_lookup(const void* table, int32_t table_dtype, int64_t rows,
                                    int64_t table_stride, int64_t dim, const void* ids,
                                    int32_t ids_bits, int64_t n, float scale, void* out,
                                    int32_t out_dtype, int64_t out_stride, int32_t* status,
                                    void* cuda_stream) {
  const char* op = "agnes_embedding_lookup";
  OP_TRY(check_embedding(op, rows, dim, n, ids_bits));
  OP_TRY(op_float_type(op, "table", table_dtype));
  OP_TRY(op_float_type(op, "out", out_dtype));
  if ((rows > 1 && table_stride < dim) || (n > 1 && out_stride < dim))
    return op_error(AGNES_EINVAL, "%s: table_stride %lld or out_stride %lld is below dim %lld", op,
                    (long long)table_stride, (long long)out_stride, (long long)dim);
  if (n == 0) return AGNES_OK;
  int device = -1;
  OP_TRY(op_device_of(op, "out", out, &device));
  if (rows > 0) OP_TRY(op_on_device(op, "table", table, device));
  OP_TRY(op_on_device(op, "ids", ids, device));
  OP_TRY(op_aligned(op, "table", table, float_size(table_dtype)));
  OP_TRY(op_aligned(op, "out", out, float_size(out_dtype)));
  OP_TRY(op_aligned(op, "ids", ids, ids_bits / 8));
  OP_TRY(op_status(op, status, device));
  DeviceGuard dg(device);
  if (!dg.ok()) return op_error(AGNES_ECUDA, "%s: cudaSetDevice(%d) failed", op, device);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = with_float_type(table_dtype, [&](auto tin) {
    return with_float_type(out_dtype, [&](auto tout) {
      using TIn = typename decltype(tin)::type;
      using TOut = typename decltype(tout)::type;
      return with_vector<TIn, TOut>(dim, table, table_stride, out, out_stride, [&](auto v) {
        constexpr int kVec = decltype(v)::value;
        // a vector of 4 bytes or less: the output as one run, where it can be
        if (kVec * sizeof(TOut) <= 4 && dim >= 8 && (n == 1 || out_stride == dim) &&
            (uintptr_t)out % 16 == 0) {
          const int64_t blocks = ceil_div(n * dim, kFlatRun);
          return with_index_type(ids_bits, [&](auto id) {
            using Id = typename decltype(id)::type;
            lookup_flat_kernel<TIn, TOut, Id><<<(unsigned)blocks, kLookupThreads, 0, st>>>(
                (const TIn*)table, rows, table_stride, (int32_t)dim, flat_inverse(dim),
                (const Id*)ids, n, scale, (TOut*)out, status);
            return cudaGetLastError();
          });
        }
        const int64_t vpr = dim / kVec, blocks = ceil_div(n * vpr, kFlat);  // 2^30 at most
        return with_index_type(ids_bits, [&](auto id) {
          using Id = typename decltype(id)::type;
          lookup_kernel<TIn, TOut, Id, kVec><<<(unsigned)blocks, kLookupThreads, 0, st>>>(
              (const TIn*)table, rows, table_stride, (int32_t)vpr, flat_inverse(vpr),
              (const Id*)ids, n, scale, (TOut*)out, out_stride, status);
          return cudaGetLastError();
        });
      });
    });
  });
  return op_launched(op, e);
}

agnes_status agnes_embedding_grad(const void* grad, int32_t grad_dtype, int64_t grad_stride,
                                  const void* ids, int32_t ids_bits, int64_t n, int64_t rows,
                                  int64_t dim, float scale, void* out, int32_t out_dtype,
                                  void* workspace, int64_t workspace_bytes, int32_t* status,
                                  void* cuda_stream) {
  return embedding_grad({"agnes_embedding_grad", grad, grad_dtype, grad_stride, ids, ids_bits, n,
                         rows, dim, scale, out, out_dtype, nullptr, nullptr, workspace,
                         workspace_bytes, status, (cudaStream_t)cuda_stream},
                        false);
}

agnes_status agnes_embedding_grad_rows(const void* grad, int32_t grad_dtype, int64_t grad_stride,
                                       const void* ids, int32_t ids_bits, int64_t n, int64_t rows,
                                       int64_t dim, float scale, int32_t* out_ids, void* out,
                                       int32_t out_dtype, int32_t* count, void* workspace,
                                       int64_t workspace_bytes, int32_t* status,
                                       void* cuda_stream) {
  return embedding_grad({"agnes_embedding_grad_rows", grad, grad_dtype, grad_stride, ids, ids_bits,
                         n, rows, dim, scale, out, out_dtype, out_ids, count, workspace,
                         workspace_bytes, status, (cudaStream_t)cuda_stream},
                        true);
}

agnes_status agnes_embedding_grad_workspace(int64_t n, int64_t dim, int64_t* bytes) {
  const char* op = "agnes_embedding_grad_workspace";
  if (!bytes) return op_error(AGNES_EINVAL, "%s: bytes is NULL", op);
  OP_TRY(check_embedding(op, 0, dim, n, 32));
  *bytes = (int64_t)grad_plan(n, dim).bytes;
  return AGNES_OK;
}

}  // extern "C"
