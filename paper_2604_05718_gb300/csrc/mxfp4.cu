// Tokens to MXFP4 and back (mxfp4.cuh has the layout).
//
// A block's scale is 2^(floor(log2 amax) - 2), 2 being E2M1's largest
// exponent, and at least 2^-127; elements are rounded to nearest, ties to
// even, and saturate at 6.  All of it is exact but the one rounding: the
// scale comes from amax's exponent bits, and scaling is by a power of two.
// A block with a NaN or an infinity has no scale: it is stored as the scale
// code of NaN, and all of its elements read back as NaN.
//
// Bound: HBM (bf16: 2 bytes an element in, 17/32 out).  A block of threads
// takes whole scale tiles (128 rows x 128 columns): half a warp spans the
// tile's columns, eight elements a lane, and a thread has the loads of its
// eight rows in flight.  Rows and columns of a thread are then constants of
// the loop; walking all rows' elements with running indexes was bound by
// those instructions (65536 x 768 bf16: 46 us; tiles 24).
#include <string.h>

#include "common.cuh"
#include "mxfp4.cuh"

namespace mpm {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 8;                                           // elements a thread takes of a row
constexpr int kTileCols = mx::kBlock * mx::kTileBlocks;
constexpr int kLanes = kTileCols / kUnit;                          // lanes that span a tile's columns
constexpr int kRowsAtOnce = kThreads / kLanes;
constexpr int kRows = mx::kTileRows / kRowsAtOnce;                 // rows of a tile that a thread takes
static_assert(kLanes == 16 && kRows == 8, "half a warp per row");

// Eight elements of a row, as they lie in memory.
template <typename T>
struct Unit {
  uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Unit<T> load_unit(const T* p, int left, bool vec) {
  Unit<T> u;
  if (vec && left >= kUnit) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) u.w[i] = ld_stream(reinterpret_cast<const uint4*>(p) + i);
  } else {
    T e[kUnit];
#pragma unroll
    for (int i = 0; i < kUnit; ++i) e[i] = i < left ? p[i] : T(0.f);
    memcpy(&u, e, sizeof(u));
  }
  return u;
}
// The largest magnitude's bits, as those of a float.
__device__ __forceinline__ uint32_t top_bits(const Unit<__nv_bfloat16>& u) {
  const uint32_t w[4] = {u.w[0].x, u.w[0].y, u.w[0].z, u.w[0].w};
  uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
  for (int i = 1; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
  return max(m << 16, m & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t top_bits(const Unit<float>& u) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w[4] = {u.w[i].x, u.w[i].y, u.w[i].z, u.w[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, w[j] & 0x7FFFFFFFu);
  }
  return m;
}
__device__ __forceinline__ void widen(const Unit<__nv_bfloat16>& u, float (&v)[kUnit]) {
  const uint32_t w[4] = {u.w[0].x, u.w[0].y, u.w[0].z, u.w[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen(const Unit<float>& u, float (&v)[kUnit]) { memcpy(v, &u, sizeof(u)); }

// Eight E2M1 codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t encode8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

// Eight codes to bf16 pairs, times 2^(c - 127).  A code's exponent and
// mantissa bits in the place of bf16's last exponent bits and first mantissa
// bit are the value times 2^-126 (E2M1's subnormal 0.5 as bf16's), so one
// multiplication makes it the value and another scales it: both are exact
// (bf16 reaches down to 2^-133), or overflow as fp32 would.
__device__ __forceinline__ void decode8(uint32_t codes, int c, __nv_bfloat162 (&v)[4]) {
  const __nv_bfloat162 up = __bfloat162bfloat162(__ushort_as_bfloat16(253 << 7));  // 2^126
  const uint16_t unit = c == mx::kNanScale ? 0x7FFF : c > 0 ? static_cast<uint16_t>(c << 7) : 0x0040;
  const __nv_bfloat162 by = __bfloat162bfloat162(__ushort_as_bfloat16(unit));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = codes >> (8 * i);
    const uint32_t t = (b & 0xFu) | ((b & 0xF0u) << 12);
    const uint32_t bits = ((t & 0x00070007u) << 6) | ((t & 0x00080008u) << 12);
    v[i] = __hmul2_rn(__hmul2_rn(*reinterpret_cast<const __nv_bfloat162*>(&bits), up), by);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_kernel(QuantizeArgs a, bool vec, int64_t scale_tiles) {
  wait_for_previous_grid();
  allow_next_grid();
  const int tiles_k = mx::scale_tiles(a.dim), pitch = mx::code_pitch(a.dim);
  const int lane = threadIdx.x % kLanes, first = threadIdx.x / kLanes;
  for (int64_t tile = blockIdx.x; tile < scale_tiles; tile += gridDim.x) {
    const int64_t row_tile = tile / tiles_k;
    const int col = static_cast<int>(tile - row_tile * tiles_k) * kTileCols + lane * kUnit;
    const int64_t row0 = row_tile * mx::kTileRows + first;
    const T* x = static_cast<const T*>(a.x) + row0 * a.stride + col;
    Unit<T> u[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      u[i] = load_unit(x + i * kRowsAtOnce * a.stride, row0 + i * kRowsAtOnce < a.rows ? a.dim - col : 0, vec);
    uint8_t* codes = a.codes + row0 * pitch + col / 2;
    uint8_t* scales = a.scales + tile * mx::kTileBytes + lane / 4;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      // The four lanes of a block.
      uint32_t top = top_bits(u[i]);
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      // What a block that is not finite holds as codes does not matter: its scale makes it NaN.
      const bool finite = top < 0x7F800000u;
      const int code = finite ? max(static_cast<int>(top >> 23) - 2, 0) : mx::kNanScale;
      const float by = finite ? __uint_as_float(static_cast<uint32_t>(254 - code) << 23) : 0.f;
      float v[kUnit];
      widen(u[i], v);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[j] *= by;
      if (row0 + i * kRowsAtOnce < a.rows && col / 2 < pitch)
        *reinterpret_cast<uint32_t*>(codes + i * kRowsAtOnce * static_cast<int64_t>(pitch)) = encode8(v);
      const int r = first + i * kRowsAtOnce;
      if (lane % 4 == 0) scales[(r % 32) * 16 + (r / 32) * 4] = static_cast<uint8_t>(code);
    }
  }
}

// Eight values of a row where all of them lie inside it and 16-byte aligned.
__device__ __forceinline__ void store_unit(__nv_bfloat16* p, const __nv_bfloat162 (&v)[4]) {
  st_stream(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(v));
}
__device__ __forceinline__ void store_unit(float* p, const __nv_bfloat162 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = __bfloat1622float2(v[2 * i]), b = __bfloat1622float2(v[2 * i + 1]);
    __stcs(reinterpret_cast<float4*>(p) + i, make_float4(a.x, a.y, b.x, b.y));
  }
}

// VEC: rows of 16-byte aligned values.  Otherwise a row's values (bf16 holds
// them all) cross over in shared memory, so that a half warp stores 16
// neighbours at a time: 50000 x 769 bf16 in 30 us, 122 with a lane's eight
// values stored one by one.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(DequantizeArgs a, int64_t scale_tiles) {
  wait_for_previous_grid();
  allow_next_grid();
  __shared__ __align__(16) __nv_bfloat16 rows[VEC ? 1 : kRowsAtOnce][VEC ? 8 : kTileCols + 8];
  const int tiles_k = mx::scale_tiles(a.dim), pitch = mx::code_pitch(a.dim);
  const int lane = threadIdx.x % kLanes, first = threadIdx.x / kLanes;
  for (int64_t tile = blockIdx.x; tile < scale_tiles; tile += gridDim.x) {
    const int64_t row_tile = tile / tiles_k;
    const int col0 = static_cast<int>(tile - row_tile * tiles_k) * kTileCols, col = col0 + lane * kUnit;
    const int64_t row0 = row_tile * mx::kTileRows + first;
    const uint8_t* codes = a.codes + row0 * pitch + col / 2;
    const uint8_t* scales = a.scales + tile * mx::kTileBytes + lane / 4;
    T* out = static_cast<T*>(a.out) + row0 * a.stride + col;
    uint32_t code[kRows];
    int scale[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = first + i * kRowsAtOnce;
      const bool in = row0 + i * kRowsAtOnce < a.rows && col < a.dim;
      code[i] = in ? __ldcs(reinterpret_cast<const uint32_t*>(codes + i * kRowsAtOnce * static_cast<int64_t>(pitch))) : 0u;
      scale[i] = in ? __ldg(scales + (r % 32) * 16 + (r / 32) * 4) : 0;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      __nv_bfloat162 v[4];
      decode8(code[i], scale[i], v);
      T* to = out + i * kRowsAtOnce * a.stride;
      if constexpr (VEC) {
        if (row0 + i * kRowsAtOnce < a.rows && col + kUnit <= a.dim) {
          store_unit(to, v);
          continue;
        }
        if (row0 + i * kRowsAtOnce < a.rows) {
#pragma unroll
          for (int j = 0; j < kUnit; ++j)
            if (col + j < a.dim) to[j] = j & 1 ? T(__high2float(v[j / 2])) : T(__low2float(v[j / 2]));
        }
      } else {
        __nv_bfloat16* mine = rows[first];
        __syncwarp();  // the row before has been read
        *reinterpret_cast<uint4*>(mine + lane * kUnit) = *reinterpret_cast<const uint4*>(v);
        __syncwarp();
        if (row0 + i * kRowsAtOnce < a.rows) {
          T* row = to - lane * kUnit;
#pragma unroll
          for (int j = 0; j < kUnit; ++j) {
            const int c = j * kLanes + lane;
            if (col0 + c < a.dim) row[c] = T(__bfloat162float(mine[c]));
          }
        }
      }
    }
  }
}

template <typename Args>
int tile_grid(const Args& a, int per_sm, int num_sms, int64_t* tiles) {
  *tiles = mx::row_tiles(a.rows) * mx::scale_tiles(a.dim);
  const int64_t most = static_cast<int64_t>(num_sms) * per_sm;
  return static_cast<int>(*tiles < most ? *tiles : most);
}

template <typename T>
cudaError_t quantize(const QuantizeArgs& a, bool vec, int num_sms, cudaStream_t stream) {
  static const int per_sm = resident_per_sm(quantize_kernel<T>, kThreads, 8);
  int64_t tiles;
  const int grid = tile_grid(a, per_sm, num_sms, &tiles);
  return launch_dependent(quantize_kernel<T>, dim3(grid), dim3(kThreads), 0, stream, a, vec, tiles);
}

template <typename T, bool VEC>
cudaError_t dequantize(const DequantizeArgs& a, int num_sms, cudaStream_t stream) {
  static const int per_sm = resident_per_sm(dequantize_kernel<T, VEC>, kThreads, 8);
  int64_t tiles;
  const int grid = tile_grid(a, per_sm, num_sms, &tiles);
  return launch_dependent(dequantize_kernel<T, VEC>, dim3(grid), dim3(kThreads), 0, stream, a, tiles);
}

}  // namespace

cudaError_t launch_mxfp4_quantize(const QuantizeArgs& a, bool bf16, bool vec, int num_sms, cudaStream_t stream) {
  return bf16 ? quantize<__nv_bfloat16>(a, vec, num_sms, stream) : quantize<float>(a, vec, num_sms, stream);
}

cudaError_t launch_mxfp4_dequantize(const DequantizeArgs& a, bool bf16, bool vec, int num_sms, cudaStream_t stream) {
  if (bf16)
    return vec ? dequantize<__nv_bfloat16, true>(a, num_sms, stream) : dequantize<__nv_bfloat16, false>(a, num_sms, stream);
  return vec ? dequantize<float, true>(a, num_sms, stream) : dequantize<float, false>(a, num_sms, stream);
}

}  // namespace mpm
