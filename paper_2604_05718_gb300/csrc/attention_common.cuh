// What the attention kernels share: where a sequence's rows are, which tile a
// work item is, and the scores' arithmetic.
//
// Sequences are packed, and their lengths are known on the device only.  Tiles
// of T rows are numbered without a plan: sequence b's begin at number
// floor(off[b] / T) + b.  That leaves it floor(off[b + 1] / T) + 1 - floor(off[b] / T)
// numbers, which is at least ceil(n / T); the one that may be left over is idle.
#pragma once

#include "attention.h"
#include "common.cuh"
#include "norm_rows.cuh"

namespace mpm {
namespace attn {

using norm::from_f32;
using norm::to_f32;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// What the rounding of a value to T leaves, rounded to T (0 where it overflowed).
template <typename T>
__device__ __forceinline__ T rest_of(float v) {
  const float r = v - to_f32(from_f32<T>(v));
  return from_f32<T>(isfinite(r) ? r : 0.f);
}

struct Span {
  int64_t lo;
  int n;
};
// Rows of sequence b, within the buffer whatever the offsets say.
__device__ __forceinline__ Span span_of(const int64_t* __restrict__ off, int b, int64_t rows) {
  if (off == nullptr) return {0, static_cast<int>(rows)};
  int64_t lo = __ldg(off + b), hi = __ldg(off + b + 1);
  lo = lo < 0 ? 0 : lo > rows ? rows : lo;
  hi = hi < lo ? lo : hi > rows ? rows : hi;
  return {lo, static_cast<int>(hi - lo)};
}
// Rows that belong to sequences.
__device__ __forceinline__ int64_t live_rows(const int64_t* __restrict__ off, int batch, int64_t rows) {
  if (off == nullptr) return rows;
  const int64_t n = __ldg(off + batch);
  return n < 0 ? 0 : n > rows ? rows : n;
}

template <int T>
__host__ __device__ __forceinline__ int64_t tile_slots(const int64_t* off, int batch, int64_t rows) {
  return off == nullptr ? (rows + T - 1) / T : rows / T + batch;
}
struct Tile {
  int image;   // -1: idle
  int first;   // first row of the tile within the sequence
  Span rows;   // the sequence's rows
};
__device__ __forceinline__ Tile tile_of(const int64_t* __restrict__ off, int batch, int64_t rows, int64_t slot, int T) {
  int b = 0;
  int64_t t = slot;
  if (off != nullptr) {
    int lo = 0, hi = batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (__ldg(off + mid) / T + mid <= slot) lo = mid; else hi = mid - 1;
    }
    b = lo;
    t = slot - (__ldg(off + b) / T + b);
  }
  const Span s = span_of(off, b, rows);
  if (t < 0 || t * T >= s.n) return {-1, 0, s};
  return {b, static_cast<int>(t * T), s};
}
template <int T>
__device__ __forceinline__ Tile tile_of(const int64_t* __restrict__ off, int batch, int64_t rows, int64_t slot) {
  return tile_of(off, batch, rows, slot, T);
}

// Tiles [begin, end) of `tiles` that part `split` of `splits` takes.
struct Part {
  int begin, end;
};
__device__ __forceinline__ Part part_of(int tiles, int split, int splits) {
  if (splits == 1) return {0, tiles};
  const int per = tiles / splits, extra = tiles % splits;
  const int begin = split * per + (split < extra ? split : extra);
  return {begin, begin + per + (split < extra ? 1 : 0)};
}

// By the threads of one block of a launch, or of one of its warps: reports offsets
// that are not 0 = off[0] <= .. <= off[batch] <= rows.
__device__ __forceinline__ void check_offsets(const int64_t* __restrict__ off, int batch, int64_t rows, int32_t* status,
                                              int first, int step) {
  if (off == nullptr || status == nullptr) return;
  for (int b = first; b <= batch; b += step) {
    const int64_t v = __ldg(off + b);
    const bool bad = b == 0 ? v != 0 : v < __ldg(off + b - 1);
    if (bad || (b == batch && v > rows)) report(status, MPM_ERR_DEVICE_CHECK, b);
  }
}
__device__ __forceinline__ void check_offsets(const int64_t* __restrict__ off, int batch, int64_t rows, int32_t* status) {
  check_offsets(off, batch, rows, status, threadIdx.x, blockDim.x);
}

}  // namespace attn
}  // namespace mpm
