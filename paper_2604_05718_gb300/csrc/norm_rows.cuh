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
// In a vector chunk all eight columns lie inside the row or none does (dim is a multiple of 8).
template <bool VEC>
__device__ __forceinline__ bool inside(int col, int i, int dim) {
  return column<VEC>(col, VEC ? 0 : i) < dim;
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void widen(uint4 r, float (&v)[8]) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = __bfloat1622float2(h[k]);
    v[2 * k] = f.x;
    v[2 * k + 1] = f.y;
  }
}

// Eight columns of a row of tokens; zeros outside the row.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* __restrict__ row, int col, int dim, float (&v)[8]) {
  if constexpr (VEC) {
    if (col >= dim) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else if constexpr (sizeof(T) == 2) {
      widen(ld_stream(reinterpret_cast<const uint4*>(row + col)), v);
    } else {
      const uint4 a = ld_stream(reinterpret_cast<const uint4*>(row + col));
      const uint4 b = ld_stream(reinterpret_cast<const uint4*>(row + col) + 1);
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + 32 * i < dim ? to_f32(row[col + 32 * i]) : 0.f;
  }
}

// Eight columns of a parameter vector (kept in the caches); `otherwise` where it is absent.
template <bool VEC>
__device__ __forceinline__ void param8(const float* __restrict__ p, int col, int dim, float otherwise,
                                       float (&v)[8]) {
  if (p == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = otherwise;
  } else if constexpr (VEC) {
    if (col < dim) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p + col));
      const float4 b = __ldg(reinterpret_cast<const float4*>(p + col) + 1);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + 32 * i < dim ? __ldg(p + col + 32 * i) : 0.f;
  }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* __restrict__ row, int col, int dim, const float (&v)[8]) {
  if constexpr (VEC) {
    if (col >= dim) return;
    if constexpr (sizeof(T) == 2) {
      uint4 r;
      __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      st_stream(reinterpret_cast<uint4*>(row + col), r);
    } else {
      uint4* p = reinterpret_cast<uint4*>(row + col);
      st_stream(p, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
      st_stream(p + 1, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + 32 * i < dim) row[col + 32 * i] = from_f32<T>(v[i]);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Sums over a row held by the W warps of a group, the same in every thread.
// MULTI = false: one warp, no shared memory.  `sh` holds 2 x W float2 of the
// group; the two halves alternate, so that one barrier a sum is enough: a
// warp writes a half again only after the next sum's barrier, which every
// warp reaches after it has read this one.
template <bool MULTI>
struct RowSum {
  float2* sh;
  int warps, warp, barrier, turn;
  __device__ __forceinline__ float2 operator()(float a, float b) {
    float2 v = make_float2(warp_sum(a), warp_sum(b));
    if constexpr (MULTI) {
      float2* half = sh + (turn & 1) * warps;
      ++turn;
      if ((threadIdx.x & 31) == 0) half[warp] = v;
      asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(warps * 32) : "memory");
      v = half[0];
      for (int w = 1; w < warps; ++w) {
        v.x += half[w].x;
        v.y += half[w].y;
      }
    }
    return v;
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
