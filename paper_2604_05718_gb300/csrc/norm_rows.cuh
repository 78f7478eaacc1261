// What the forward and the backward block_norm kernels share: how a row is
// spread over threads, its loads and stores, and sums over it.
#pragma once

#include "block_launch.h"
#include "common.cuh"

namespace mpm {
namespace norm {

// A row belongs to a group of W warps.  Each thread holds C chunks of eight
// of its columns; chunk c of warp w covers columns [256 (c W + w), + 256).
// Within it a lane takes eight neighbours (VEC: one or two 16-byte accesses)
// or, where rows are not 16-byte aligned, every 32nd column, so that a warp's
// accesses are whole 64- or 128-byte runs all the same.
template <bool VEC>
__device__ __forceinline__ int first_column(int chunk, int lane) {
  return chunk * kNormWarpCols + (VEC ? lane * 8 : lane);
}
// Column i of a chunk whose first column is col.
template <bool VEC>
__device__ __forceinline__ int column(int col, int i) {
  return VEC ? col + i : col + 32 * i;
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight values of a row as pairs: the kernels' arithmetic is on pairs, which
// Blackwell issues as one instruction.
struct F8 {
  float2 p[4];
};
__device__ __forceinline__ float2 pair(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ F8 all8(float v) { return {{pair(v), pair(v), pair(v), pair(v)}}; }

__device__ __forceinline__ F8 widen(uint4 r) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  F8 v;
#pragma unroll
  for (int k = 0; k < 4; ++k) v.p[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
  return v;
}
__device__ __forceinline__ F8 join(float4 a, float4 b) {
  return {{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}

// Eight columns of a row of tokens; zeros outside the row.
template <typename T, bool VEC>
__device__ __forceinline__ F8 load8(const T* __restrict__ row, int col, int dim) {
  if constexpr (VEC) {
    // Zeros as they lie in memory: selecting among widened values would take twice the instructions.
    if constexpr (sizeof(T) == 2) {
      uint4 r = make_uint4(0, 0, 0, 0);
      if (col < dim) r = ld_stream(reinterpret_cast<const uint4*>(row + col));
      return widen(r);
    } else {
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
      if (col < dim) {
        const float4* p = reinterpret_cast<const float4*>(row + col);
        a = __ldcs(p);
        b = __ldcs(p + 1);
      }
      return join(a, b);
    }
  } else {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + 32 * i < dim ? to_f32(row[col + 32 * i]) : 0.f;
    return {{make_float2(v[0], v[1]), make_float2(v[2], v[3]), make_float2(v[4], v[5]), make_float2(v[6], v[7])}};
  }
}

// Eight columns of a parameter vector (kept in the caches); `otherwise` where it is absent.
template <bool VEC>
__device__ __forceinline__ F8 param8(const float* __restrict__ p, int col, int dim, float otherwise) {
  if (p == nullptr) return all8(otherwise);
  if constexpr (VEC) {
    if (col >= dim) return all8(0.f);
    const float4* q = reinterpret_cast<const float4*>(p + col);
    return join(__ldg(q), __ldg(q + 1));
  } else {
    return load8<float, false>(p, col, dim);
  }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* __restrict__ row, int col, int dim, const F8& v) {
  if constexpr (VEC) {
    if (col >= dim) return;
    if constexpr (sizeof(T) == 2) {
      uint4 r;
      __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(v.p[k].x, v.p[k].y);
      st_stream(reinterpret_cast<uint4*>(row + col), r);
    } else {
      float4* p = reinterpret_cast<float4*>(row + col);
      __stcs(p, make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y));
      __stcs(p + 1, make_float4(v.p[2].x, v.p[2].y, v.p[3].x, v.p[3].y));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + 32 * i < dim) row[col + 32 * i] = from_f32<T>(i & 1 ? v.p[i / 2].y : v.p[i / 2].x);
  }
}

// 1 for the columns inside the row, 0 for the others (a factor, so that pairs stay pairs).
template <bool VEC>
__device__ __forceinline__ F8 mask8(int col, int dim) {
  if constexpr (VEC) {
    return all8(col < dim ? 1.f : 0.f);
  } else {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + 32 * i < dim ? 1.f : 0.f;
    return {{make_float2(v[0], v[1]), make_float2(v[2], v[3]), make_float2(v[4], v[5]), make_float2(v[6], v[7])}};
  }
}

// Vectors in shared memory, eight columns a thread, without bank conflicts:
// chunk, half of the eight, thread of the row.
struct SharedVector {
  float4* v;
  int threads, at;
  __device__ __forceinline__ F8 get(int c) const { return join(v[2 * c * threads + at], v[(2 * c + 1) * threads + at]); }
  __device__ __forceinline__ void set(int c, const F8& f) const {
    v[2 * c * threads + at] = make_float4(f.p[0].x, f.p[0].y, f.p[1].x, f.p[1].y);
    v[(2 * c + 1) * threads + at] = make_float4(f.p[2].x, f.p[2].y, f.p[3].x, f.p[3].y);
  }
};
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// The sum over a row held by the W warps of a group, the same in every thread.
// MULTI = false: one warp, no shared memory.  `sh` holds 2 x W floats of the
// group; the two halves alternate, so that one barrier a sum is enough: a
// warp writes a half again only after the next sum's barrier, which every
// warp reaches after it has read this one.
template <bool MULTI>
struct RowSum {
  float* sh;
  int warps, warp, barrier, turn;
  __device__ __forceinline__ float operator()(float a) {
    float v = warp_sum(a);
    if constexpr (MULTI) {
      float* half = sh + (turn & 1) * warps;
      ++turn;
      if ((threadIdx.x & 31) == 0) half[warp] = v;
      asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(warps * 32) : "memory");
      v = half[0];
      for (int w = 1; w < warps; ++w) v += half[w];
    }
    return v;
  }
};

// Two values summed over a warp: lanes 0 to 15 get the sum of the first, the
// others of the second.  They trade values first, so that both take six
// shuffles instead of ten.
__device__ __forceinline__ float warp_sums(const float (&v)[2]) {
  const bool hi = (threadIdx.x & 16) != 0;
  float s = (hi ? v[1] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? v[0] : v[1], 16);
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  return s;
}

// The same over the W warps of a group, both sums to every thread.  `sh` holds
// 2 x W pairs; its halves alternate as in RowSum.
template <bool MULTI>
struct PairSum {
  float2* sh;
  int warps, warp, barrier, turn;
  __device__ __forceinline__ void operator()(float (&v)[2]) {
    const float s = warp_sums(v);
    if constexpr (MULTI) {
      const int lane = threadIdx.x & 31;
      float2* half = sh + (turn & 1) * warps;
      ++turn;
      if (lane % 16 == 0) (lane == 0 ? half[warp].x : half[warp].y) = s;
      asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(warps * 32) : "memory");
      float2 t = half[0];
      for (int w = 1; w < warps; ++w) {
        t.x += half[w].x;
        t.y += half[w].y;
      }
      v[0] = t.x;
      v[1] = t.y;
    } else {
      v[0] = __shfl_sync(0xFFFFFFFFu, s, 0);
      v[1] = __shfl_sync(0xFFFFFFFFu, s, 16);
    }
  }
};

// Rows in use: those of the images, or all.
__device__ __forceinline__ int64_t used_rows(const int64_t* offsets, int batch, int64_t rows) {
  if (offsets == nullptr) return rows;
  const int64_t n = __ldg(offsets + batch);
  return n < 0 ? 0 : (n < rows ? n : rows);
}

// Offsets that are not 0 = off[0] <= ... <= off[batch] <= rows are reported.
__device__ __forceinline__ void check_offsets(const int64_t* offsets, int batch, int64_t rows, int32_t* status) {
  if (offsets == nullptr || status == nullptr || blockIdx.x != 0) return;
  for (int b = threadIdx.x; b <= batch; b += blockDim.x) {
    const int64_t v = __ldg(offsets + b);
    if ((b == 0 && v != 0) || (b > 0 && v < __ldg(offsets + b - 1)) || v > rows)
      report(status, MPM_ERR_DEVICE_CHECK, b);
  }
}

}  // namespace norm
}  // namespace mpm
