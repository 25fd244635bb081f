// rows.cuh -- rows of a matrix that groups of threads hold in registers: who has which
// columns, loads and stores, reductions over a group.
//
// A group of `lanes` threads (a power of two up to 1024) has a row.  In vectors of kVec
// elements (16 bytes at most an access), vector i of a thread starts at column
// (i * lanes + lane) * kVec, so neighbouring threads' accesses are side by side; with
// kVec = 1 that holds for single elements, for rows that no vector divides.  A CTA has
// 256 threads, or a group's if that is more.
#pragma once

#include <type_traits>

#include "ops_common.cuh"

namespace agnes {

constexpr int kRowThreads = 256;
constexpr int kRowLanesMax = 1024;

// How a launch spreads its rows.
struct RowShape {
  int32_t lanes, log_lanes;  // threads to a row
  int32_t groups;            // rows of a CTA at a time
  unsigned threads() const { return (unsigned)(lanes * groups); }
};

// For rows of `cols` columns, `per_thread` of them to a thread, `most` threads at most.
inline RowShape row_shape(int64_t cols, int per_thread, int most = kRowLanesMax) {
  RowShape s = {1, 0, 0};
  while (s.lanes < most && (int64_t)s.lanes * per_thread < cols) {
    s.lanes *= 2;
    ++s.log_lanes;
  }
  s.groups = s.lanes < kRowThreads ? kRowThreads / s.lanes : 1;
  return s;
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
  // vector i
  template <typename T>
  __device__ void store_one(T* row, bool valid, int i, const float* v) const {
    if (valid && col(i) < dim) store_vec<T, kVec>(row + col(i), v);
  }
  // Whether no thread has anything of vector i on: for single elements, of which a row rarely
  // fills all that a thread could take.
  __device__ bool beyond(int i) const { return kVec == 1 && i * lanes >= dim; }
  // elements past the end hold zeros or what a row's arithmetic made of them
  __device__ bool has(int i) const { return col(i) < dim; }
};

// A thread's part of a row as it lies in memory: two 16-bit values to a register.
template <typename T, int kVec, int kPer>
struct RowRegs {
  static constexpr int kWords = kVec * sizeof(T) / 4;
  uint32_t w[kPer][kWords];

  __device__ void load(const RowPart<kVec, kPer>& part, const T* row, bool valid) {
    constexpr int kPiece = kWords < 4 ? kWords : 4;  // words to an access
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll
      for (int h = 0; h < kWords; h += kPiece) {
        Vec<uint32_t, kPiece> v = {};
        if (valid && part.has(i))
          v = ((const Vec<uint32_t, kPiece>*)(row + part.col(i)))[h / kPiece];
#pragma unroll
        for (int e = 0; e < kPiece; ++e) w[i][h + e] = v.v[e];
      }
    }
  }
  // vector i
  __device__ void get(int i, float* f) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) f[e] = __uint_as_float(w[i][e]);
    } else if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
      for (int e = 0; e < kWords; ++e) {
        const float2 v = __half22float2(*(const __half2*)&w[i][e]);
        f[2 * e] = v.x;
        f[2 * e + 1] = v.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kWords; ++e) {
        f[2 * e] = __uint_as_float(w[i][e] << 16);
        f[2 * e + 1] = __uint_as_float(w[i][e] & 0xffff0000u);
      }
    }
  }
  // The largest magnitude, as the bits of a float.
  __device__ uint32_t top() const {
    uint32_t most = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < kWords; ++e) most = max(most, w[i][e] & 0x7fffffffu);
      return most;
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < kWords; ++e) most = __vmaxu2(most, w[i][e] & 0x7fff7fffu);
      const uint16_t bits = (uint16_t)max(most & 0xffffu, most >> 16);
      return __float_as_uint(to_f32(*(const T*)&bits));
    }
  }
  // Keeps the values as they are across this point, instead of what was made of them.
  __device__ void pin() {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int e = 0; e < kWords; ++e) asm volatile("" : "+r"(w[i][e]));
  }
};
// Single elements, for rows that no vector divides.
template <typename T, int kPer>
struct RowRegs<T, 1, kPer> {
  float v[kPer];

  __device__ void load(const RowPart<1, kPer>& part, const T* row, bool valid) {
    part.load(row, valid, v);
  }
  __device__ void get(int i, float* f) const { f[0] = v[i]; }
  __device__ uint32_t top() const {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
    return most;
  }
  __device__ void pin() {}
};

// Rows that no vector divides, of a contiguous matrix: a CTA's rows are one run of memory, which
// goes through shared memory in 16-byte pieces.  A run keeps its place within a piece there, so
// pieces lie as in memory.  (Single elements from and to memory keep 16 KB of an SM's loads on
// their way at most.)
constexpr int64_t staged_bytes(int64_t bytes) { return (bytes + 15) / 16 * 16 + 16; }

// Where a run that starts at p has its first byte in its buffer.
__device__ __forceinline__ int stage_offset(const void* p) { return (int)((uintptr_t)p & 15); }

// Starts the copies of `bytes` from p on to `buffer` (16-byte aligned); only [lo, hi) is read.
// stage_wait() ends them, for the whole CTA.
__device__ __forceinline__ void stage_in(uint8_t* buffer, const void* p, int64_t bytes,
                                         const void* lo, const void* hi) {
  const uint8_t* first = (const uint8_t*)p - stage_offset(p);
  const int pieces = (int)((bytes + stage_offset(p) + 15) / 16);
  for (int i = threadIdx.x; i < pieces; i += blockDim.x) {
    const uint8_t* at = first + (int64_t)i * 16;
    uint8_t* to = buffer + i * 16;
    if (at >= (const uint8_t*)lo && at + 16 <= (const uint8_t*)hi) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                       (uint32_t)__cvta_generic_to_shared(to)),
                   "l"(at)
                   : "memory");
    } else {
      for (int b = 0; b < 16; ++b)
        if (at + b >= (const uint8_t*)lo && at + b < (const uint8_t*)hi) to[b] = at[b];
    }
  }
}
__device__ __forceinline__ void stage_wait() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
}

// A run of `bytes` from `buffer` to p on, after a barrier.
__device__ __forceinline__ void stage_out(const uint8_t* buffer, void* p, int64_t bytes) {
  const int offset = stage_offset(p), end = (int)(bytes + offset);
  uint8_t* first = (uint8_t*)p - offset;
  for (int i = threadIdx.x; i * 16 < end; i += blockDim.x) {
    if (i * 16 >= offset && i * 16 + 16 <= end) {
      ((uint4*)first)[i] = ((const uint4*)buffer)[i];
    } else {
      for (int b = i * 16; b < i * 16 + 16; ++b)
        if (b >= offset && b < end) first[b] = buffer[b];
    }
  }
}

// How many batches of `groups` rows a CTA that stages them takes: some 48 KB of them, as a CTA
// loads, works and stores in turn, but not fewer CTAs than the device runs at a time.
inline int32_t stage_batches(int64_t rows, int32_t groups, int64_t row_bytes, int sms) {
  const int64_t fit = 49152 / (groups * row_bytes), share = rows / (groups * (int64_t)sms * 4);
  const int64_t n = fit < share ? fit : share;
  return n < 1 ? 1 : (int32_t)n;
}

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
  uint32_t words[2][4][32];
};

// v[k] over the threads of each group, for all of them; kN values at once, 4 at most.
// Every thread of the CTA takes part.  The order of a sum depends on `lanes` alone; kLanes
// is that number where it is known, or 0.
template <typename Op, int kLanes = 0, int kN>
__device__ __forceinline__ void group_reduce(typename Op::type (&v)[kN], int lanes,
                                             RowScratch* scratch, int& turn) {
  static_assert(kN <= 4, "RowScratch");
  using V = typename Op::type;
  const auto step = [&](int d) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = Op::of(v[k], __shfl_xor_sync(0xffffffffu, v[k], d));
  };
  if constexpr (kLanes > 0) {
    static_assert(kLanes <= 32, "within a warp");
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) step(d);
    return;
  }
  if (lanes < 32) {
    for (int d = lanes / 2; d > 0; d >>= 1) step(d);
    return;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) step(d);
  if (lanes == 32) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = lanes >> 5;
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < kN; ++k) *(V*)&scratch->words[turn][k][warp] = v[k];
  }
  __syncthreads();
  const int from = warp & ~(warps - 1);
#pragma unroll
  for (int k = 0; k < kN; ++k) v[k] = *(const V*)&scratch->words[turn][k][from + (lane & (warps - 1))];
  for (int d = warps / 2; d > 0; d >>= 1) step(d);
  turn ^= 1;
}

}  // namespace agnes
