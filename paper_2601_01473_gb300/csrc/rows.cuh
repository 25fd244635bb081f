// rows.cuh -- rows of a matrix that groups of threads hold in registers: who has which
// columns, loads and stores, reductions over a group.
//
// A group of `lanes` threads (a power of two up to 1024) has a row.  In vectors of kVec
// elements (16 bytes at most an access), vector i of a thread starts at column
// (i * lanes + lane) * kVec, so neighbouring threads' accesses are side by side; with
// kVec = 1 that holds for single elements, for rows that no vector divides.  A CTA has
// 256 threads, or a group's if that is more.
#pragma once

#include "ops_common.cuh"

namespace agnes {

constexpr int kRowThreads = 256;
constexpr int kRowLanesMax = 1024;

// How a launch spreads its rows.
struct RowShape {
  int32_t lanes;   // threads to a row
  int32_t groups;  // rows of a CTA at a time
  unsigned threads() const { return (unsigned)(lanes * groups); }
};

// For rows of `cols` columns, `per_thread` of them to a thread.
inline RowShape row_shape(int64_t cols, int per_thread) {
  int32_t lanes = 1;
  while (lanes < kRowLanesMax && (int64_t)lanes * per_thread < cols) lanes *= 2;
  return {lanes, lanes < kRowThreads ? kRowThreads / lanes : 1};
}

template <typename T, int kVec>
__device__ __forceinline__ void load_vec(const T* p, float* v) {
  constexpr int kN = kVec * sizeof(T) > 16 ? 16 / sizeof(T) : kVec;
#pragma unroll
  for (int h = 0; h < kVec / kN; ++h) {
    const Vec<T, kN> x = ((const Vec<T, kN>*)p)[h];
#pragma unroll
    for (int e = 0; e < kN; ++e) v[h * kN + e] = to_f32(x.v[e]);
  }
}

template <typename T, int kVec>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
  constexpr int kN = kVec * sizeof(T) > 16 ? 16 / sizeof(T) : kVec;
#pragma unroll
  for (int h = 0; h < kVec / kN; ++h) {
    Vec<T, kN> x;
#pragma unroll
    for (int e = 0; e < kN; ++e) x.v[e] = from_f32<T>(v[h * kN + e]);
    ((Vec<T, kN>*)p)[h] = x;
  }
}

// A thread's kPer vectors of a row, of which it has those before column `dim`.
template <int kVec, int kPer>
struct RowPart {
  static constexpr int kElems = kVec * kPer;
  int32_t lanes, lane, dim;

  __device__ int32_t col(int i) const { return (i * lanes + lane) * kVec; }

  // zeros past the end, or where there is no row
  template <typename T>
  __device__ void load(const T* row, bool valid, float (&v)[kElems]) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (valid && col(i) < dim) {
        load_vec<T, kVec>(row + col(i), v + i * kVec);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[i * kVec + e] = 0.f;
      }
    }
  }
  template <typename T>
  __device__ void store(T* row, bool valid, const float (&v)[kElems]) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (valid && col(i) < dim) store_vec<T, kVec>(row + col(i), v + i * kVec);
  }
  // elements past the end hold zeros or what a row's arithmetic made of them
  __device__ bool has(int i) const { return col(i) < dim; }
};

struct SumOp {
  using type = float;
  static __device__ float identity() { return 0.f; }
  static __device__ float of(float a, float b) { return a + b; }
};
struct MaxBits {  // of magnitudes as bit patterns, which order as the numbers do
  using type = uint32_t;
  static __device__ uint32_t identity() { return 0u; }
  static __device__ uint32_t of(uint32_t a, uint32_t b) { return max(a, b); }
};

// Shared memory of the reductions: two sets in turn, so that one barrier is enough (the
// next but one writes where everybody has read).
struct RowScratch {
  uint32_t words[2][3][32];
};

// v[k] over the threads of each group, for all of them; kN values at once, 3 at most.
// Every thread of the CTA takes part.  The order of a sum depends on `lanes` alone.
template <typename Op, int kN>
__device__ __forceinline__ void group_reduce(typename Op::type (&v)[kN], int lanes,
                                             RowScratch* scratch, int& turn) {
  static_assert(kN <= 3, "RowScratch");
  const int first = lanes < 32 ? lanes / 2 : 16;
  for (int d = first; d > 0; d >>= 1) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = Op::of(v[k], __shfl_xor_sync(0xffffffffu, v[k], d));
  }
  if (lanes <= 32) return;
  using V = typename Op::type;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = lanes >> 5;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < kN; ++k) *(V*)&scratch->words[turn][k][warp] = v[k];
  }
  __syncthreads();
  const int from = warp & ~(warps - 1);
#pragma unroll
  for (int k = 0; k < kN; ++k)
    v[k] = lane < warps ? *(const V*)&scratch->words[turn][k][from + lane] : Op::identity();
  for (int d = warps / 2; d > 0; d >>= 1) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = Op::of(v[k], __shfl_xor_sync(0xffffffffu, v[k], d));
  }
  // lanes past `warps` reduced identities among themselves
#pragma unroll
  for (int k = 0; k < kN; ++k) v[k] = __shfl_sync(0xffffffffu, v[k], 0);
  turn ^= 1;
}

}  // namespace agnes
