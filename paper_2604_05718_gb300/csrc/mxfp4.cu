// Tokens to MXFP4 and back (mxfp4.cuh has the layout).
//
// A block's scale is 2^(floor(log2 amax) - 2), 2 being E2M1's largest
// exponent, and at least 2^-127; elements are rounded to nearest, ties to
// even, and saturate at 6.  All of it is exact but the one rounding: the
// scale comes from amax's exponent bits, and scaling is by a power of two.
// A block with a NaN or an infinity has no scale: it is stored as the scale
// code of NaN, and all of its elements read back as NaN.
//
// Bound: HBM (bf16: 2 bytes an element in, 17/32 out).  A thread takes eight
// elements of a row, four neighbouring lanes make up a block, and a thread
// has four such loads in flight.
#include "common.cuh"
#include "mxfp4.cuh"

namespace mpm {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 8;      // elements a thread takes at a time
constexpr int kUnroll = 4;
// Units of one scale tile's columns: rows are walked in whole tiles, so that padding scales are written too.
constexpr int kTileUnits = mx::kBlock * mx::kTileBlocks / kUnit;

// Place of a thread in the units of all rows, advanced without divisions.
struct Walk {
  int64_t row;
  int unit;
  __device__ __forceinline__ void advance(int64_t rows, int units, int per_row) {
    row += rows;
    unit += units;
    if (unit >= per_row) {
      unit -= per_row;
      ++row;
    }
  }
};

template <typename T>
__device__ __forceinline__ float as_f32(T v);
template <>
__device__ __forceinline__ float as_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float as_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ void load_unit(const T* p, int left, bool vec, float (&v)[kUnit]) {
  if (vec && left >= kUnit) {
    if constexpr (sizeof(T) == 2) {
      const uint4 r = ld_stream(reinterpret_cast<const uint4*>(p));
      const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
      const uint4 a = ld_stream(reinterpret_cast<const uint4*>(p)), b = ld_stream(reinterpret_cast<const uint4*>(p) + 1);
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kUnit; ++i) v[i] = i < left ? as_f32(p[i]) : 0.f;
  }
}

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

__device__ __forceinline__ void decode8(uint32_t codes, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

__device__ __forceinline__ float scale_value(int code) {
  return __uint_as_float(code == mx::kNanScale ? 0x7FFFFFFFu : code > 0 ? static_cast<uint32_t>(code) << 23 : 0x00400000u);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_kernel(QuantizeArgs a, bool vec, int64_t padded_rows, int64_t step_rows,
                                                            int step_units) {
  wait_for_previous_grid();
  allow_next_grid();
  const int tiles = mx::scale_tiles(a.dim), per_row = tiles * kTileUnits, pitch = mx::code_pitch(a.dim);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  Walk at{first / per_row, static_cast<int>(first % per_row)};
  // Rows are whole numbers of 16 units: a block's four lanes leave the loop together.
  while (at.row < padded_rows) {
    Walk unit[kUnroll];
    float v[kUnroll][kUnit];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      unit[u] = at;
      const int col = at.unit * kUnit;
      load_unit(static_cast<const T*>(a.x) + (at.row < a.rows ? at.row * a.stride + col : 0),
                at.row < a.rows ? a.dim - col : 0, vec, v[u]);
      at.advance(step_rows, step_units, per_row);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7FFFFFFFu);
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const bool finite = top < 0x7F800000u;
      const int exponent = static_cast<int>(top >> 23);
      const int code = finite ? max(exponent - 2, 0) : mx::kNanScale;
      const float by = finite ? __uint_as_float(static_cast<uint32_t>(254 - code) << 23) : 0.f;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) v[u][i] = finite ? v[u][i] * by : 0.f;
      const Walk w = unit[u];
      if (w.row < a.rows && w.unit * 4 < pitch)
        *reinterpret_cast<uint32_t*>(a.codes + w.row * pitch + w.unit * 4) = encode8(v[u]);
      if ((w.unit & 3) == 0 && w.row < padded_rows)
        a.scales[mx::scale_byte(w.row, w.unit >> 2, tiles)] = static_cast<uint8_t>(code);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(DequantizeArgs a, bool vec, int64_t step_rows, int step_units) {
  wait_for_previous_grid();
  allow_next_grid();
  const int tiles = mx::scale_tiles(a.dim), per_row = (a.dim + kUnit - 1) / kUnit, pitch = mx::code_pitch(a.dim);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  Walk at{first / per_row, static_cast<int>(first % per_row)};
  while (at.row < a.rows) {
    Walk unit[kUnroll];
    uint32_t codes[kUnroll];
    int scale[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      unit[u] = at;
      const bool in = at.row < a.rows;
      codes[u] = in ? __ldcs(reinterpret_cast<const uint32_t*>(a.codes + at.row * pitch + at.unit * 4)) : 0u;
      scale[u] = in ? __ldg(a.scales + mx::scale_byte(at.row, at.unit >> 2, tiles)) : 0;
      at.advance(step_rows, step_units, per_row);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const Walk w = unit[u];
      if (w.row >= a.rows) break;
      float v[kUnit];
      decode8(codes[u], v);
      const float by = scale_value(scale[u]);
#pragma unroll
      for (int i = 0; i < kUnit; ++i) v[i] *= by;
      const int col = w.unit * kUnit;
      T* out = static_cast<T*>(a.out) + w.row * a.stride + col;
      if (vec && col + kUnit <= a.dim) {
        if constexpr (sizeof(T) == 2) {
          uint4 r;
          __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          st_stream(reinterpret_cast<uint4*>(out), r);
        } else {
          __stcs(reinterpret_cast<float4*>(out), make_float4(v[0], v[1], v[2], v[3]));
          __stcs(reinterpret_cast<float4*>(out) + 1, make_float4(v[4], v[5], v[6], v[7]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
          if (col + i < a.dim) {
            if constexpr (sizeof(T) == 2) out[i] = __float2bfloat16_rn(v[i]);
            else out[i] = v[i];
          }
      }
    }
  }
}

// Grid and the step of a grid-wide stride, in rows and units.
struct Plan {
  int grid;
  int64_t step_rows;
  int step_units;
};
Plan plan_of(int64_t rows, int per_row, int per_sm, int num_sms) {
  const int64_t want = (rows * per_row + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  const int64_t most = static_cast<int64_t>(num_sms) * per_sm;
  const int grid = static_cast<int>(want < most ? want : most);
  const int64_t step = static_cast<int64_t>(grid) * kThreads;
  return {grid, step / per_row, static_cast<int>(step % per_row)};
}

template <typename T>
cudaError_t quantize(const QuantizeArgs& a, bool vec, int num_sms, cudaStream_t stream) {
  static const int per_sm = resident_per_sm(quantize_kernel<T>, kThreads, 8);
  const int64_t padded = mx::row_tiles(a.rows) * mx::kTileRows;
  const Plan p = plan_of(padded, mx::scale_tiles(a.dim) * kTileUnits, per_sm, num_sms);
  return launch_dependent(quantize_kernel<T>, dim3(p.grid), dim3(kThreads), 0, stream, a, vec, padded, p.step_rows,
                          p.step_units);
}

template <typename T>
cudaError_t dequantize(const DequantizeArgs& a, bool vec, int num_sms, cudaStream_t stream) {
  static const int per_sm = resident_per_sm(dequantize_kernel<T>, kThreads, 8);
  const Plan p = plan_of(a.rows, (a.dim + kUnit - 1) / kUnit, per_sm, num_sms);
  return launch_dependent(dequantize_kernel<T>, dim3(p.grid), dim3(kThreads), 0, stream, a, vec, p.step_rows, p.step_units);
}

}  // namespace

cudaError_t launch_mxfp4_quantize(const QuantizeArgs& a, bool bf16, bool vec, int num_sms, cudaStream_t stream) {
  return bf16 ? quantize<__nv_bfloat16>(a, vec, num_sms, stream) : quantize<float>(a, vec, num_sms, stream);
}

cudaError_t launch_mxfp4_dequantize(const DequantizeArgs& a, bool bf16, bool vec, int num_sms, cudaStream_t stream) {
  return bf16 ? dequantize<__nv_bfloat16>(a, vec, num_sms, stream) : dequantize<float>(a, vec, num_sms, stream);
}

}  // namespace mpm
