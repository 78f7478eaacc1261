// Rotary positions of several axes: pair p of every head's features, of axis
// a(p), turns by positions[row, a(p)] * frequencies[p] radians.
//
//   (u, v) -> (u cos - v sin, u sin + v cos);  backward: the angle negated
//
// Angles are held in turns, t = position * frequency / 2 pi, with the frequency
// as a sum of two fp32 values: t = position * high rounded, its remainder by one
// fma, and position * low.  The whole turns are dropped before anything is
// rounded, so an angle far out (10^6 turns and more) is as exact as one near 0,
// where position * frequency in fp32 would be off by 0.06 radians at 10^6.  Fp64
// is left to the two products a pair and block; its rate is 1 / 64 of fp32's.
//
// A warp takes a row, or where there are few rows a block does: it puts the row's
// sines and cosines into shared memory once for all heads, and then moves 16
// bytes a lane.  Bound: HBM, every value once in and once out (54208 rows, 24 heads of
// 64, two axes: 56 us, 5.9 TB/s).
#include "attention_common.cuh"

namespace mpm {
namespace {

using namespace attn;

constexpr int kWarps = 8;
constexpr int kAtOnce = 3;  // units of a lane

template <typename T>
struct Vec {
  static constexpr int kSize = 16 / sizeof(T);
  float v[kSize];
};
template <typename T>
__device__ __forceinline__ Vec<T> widen_vec(const uint4& u) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  Vec<T> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      r.v[i] = __uint_as_float(w[i]);
    } else {
      r.v[2 * i] = __uint_as_float(w[i] << 16);
      r.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store_vec(T* p, const Vec<T>& r) {
  uint4 u;
  if constexpr (sizeof(T) == 4) {
    u = make_uint4(__float_as_uint(r.v[0]), __float_as_uint(r.v[1]), __float_as_uint(r.v[2]), __float_as_uint(r.v[3]));
  } else {
    __nv_bfloat162 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(r.v[2 * i], r.v[2 * i + 1]);
    u = *reinterpret_cast<const uint4*>(h);
  }
  *reinterpret_cast<uint4*>(p) = u;
}

__device__ __forceinline__ void turn(float& u, float& v, float2 cs) {
  const float a = u, b = v;
  u = fmaf(a, cs.x, -b * cs.y);
  v = fmaf(a, cs.y, b * cs.x);
}

// A row's work is `heads` times `units`: 16-byte pieces (VEC; with halves a piece
// of either half), or single pairs, then what is left over.
template <typename T, bool VEC, bool HALVES>
__global__ void __launch_bounds__(kWarps * 32) rotary_kernel(const RotaryArgs a, int row_warps) {
  extern __shared__ float2 sm[];
  float2* turns = sm;                                                     // (high, low) of each pair's turns per position
  int* axis = reinterpret_cast<int*>(turns + a.pairs);
  float2* table = reinterpret_cast<float2*>(axis + (a.pairs + 1) / 2 * 2) + threadIdx.x / 32 * a.pairs;  // the row's (cos, sin)
  wait_for_previous_grid();
  allow_next_grid();
  if (blockIdx.x == 0) check_offsets(a.offsets, a.batch, a.rows, a.status);
  for (int p = threadIdx.x; p < a.pairs; p += blockDim.x) {
    const double t = a.frequencies[p] * 0.15915494309189533577;  // 1 / (2 pi)
    const float hi = static_cast<float>(t);
    turns[p] = make_float2(hi, static_cast<float>(t - static_cast<double>(hi)));
    int k = 0;
    for (int i = 1; i < a.axes; ++i) k += p >= a.first_pair[i];
    axis[p] = k;
  }
  __syncthreads();
  constexpr int S = Vec<T>::kSize;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t live = live_rows(a.offsets, a.batch, a.rows);
  const int turned = VEC ? (HALVES ? a.pairs / S : 2 * a.pairs / S) : a.pairs;  // units of a head that turn
  const int rest = VEC ? (a.dim - 2 * a.pairs) / S : a.dim - 2 * a.pairs;       // units that are copied
  const bool in_place = a.out == a.x.p && a.out_row == a.x.row && a.out_head == a.x.head;
  const int units = turned + (in_place ? 0 : rest), all = units * a.heads;
  const int groups = kWarps / row_warps, step = 32 * row_warps, first = warp % row_warps * 32 + lane;
  const int head0 = first / units, u0 = first % units, step_head = step / units, step_u = step % units;
  for (int64_t r = blockIdx.x * static_cast<int64_t>(groups) + warp / row_warps; r < live;
       r += gridDim.x * static_cast<int64_t>(groups)) {
    const T* x = static_cast<const T*>(a.x.p) + r * a.x.row;
    T* y = static_cast<T*>(a.out) + r * a.out_row;
    const T* from[kAtOnce];
    T* to[kAtOnce];
    int unit[kAtOnce];
    uint4 lo[kAtOnce], hi[kAtOnce];
    int head = head0, u = u0;
    auto load = [&](int i) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        unit[k] = i + k * step < all ? u : -1;
        from[k] = x + head * a.x.head;
        to[k] = y + head * a.out_head;
        if constexpr (VEC) {
          if (unit[k] >= turned) {
            lo[k] = *reinterpret_cast<const uint4*>(from[k] + 2 * a.pairs + (u - turned) * S);
          } else if (unit[k] >= 0) {
            lo[k] = *reinterpret_cast<const uint4*>(from[k] + u * S);
            if constexpr (HALVES) hi[k] = *reinterpret_cast<const uint4*>(from[k] + a.pairs + u * S);
          }
        }
        u += step_u;
        head += step_head;
        if (u >= units) {
          u -= units;
          ++head;
        }
      }
    };
    // The row's first units are under way while its sines are found.
    load(first);
    __syncwarp();
    for (int p = lane; p < a.pairs; p += 32) {
      const float at = __ldg(a.positions + r * a.axes + axis[p]);
      const float2 f = turns[p];
      const float t = at * f.x, low = fmaf(at, f.y, fmaf(at, f.x, -t));
      float s, c;
      sincospif(2.f * ((t - rintf(t)) + low), &s, &c);
      table[p] = make_float2(c, a.inverse ? -s : s);
    }
    __syncwarp();
    for (int i = first; i < all; i += kAtOnce * step) {
      if (i != first) load(i);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int n = unit[k];
        if (n < 0) continue;
        if (n >= turned) {
          if constexpr (VEC) *reinterpret_cast<uint4*>(to[k] + 2 * a.pairs + (n - turned) * S) = lo[k];
          else to[k][2 * a.pairs + n - turned] = from[k][2 * a.pairs + n - turned];
        } else if constexpr (VEC && HALVES) {
          Vec<T> v = widen_vec<T>(lo[k]), w = widen_vec<T>(hi[k]);
#pragma unroll
          for (int e = 0; e < S; ++e) turn(v.v[e], w.v[e], table[n * S + e]);
          store_vec(to[k] + n * S, v);
          store_vec(to[k] + a.pairs + n * S, w);
        } else if constexpr (VEC) {
          Vec<T> v = widen_vec<T>(lo[k]);
#pragma unroll
          for (int e = 0; e < S / 2; ++e) turn(v.v[2 * e], v.v[2 * e + 1], table[n * (S / 2) + e]);
          store_vec(to[k] + n * S, v);
        } else {
          const int f = HALVES ? n : 2 * n, g = HALVES ? n + a.pairs : 2 * n + 1;
          float v = to_f32(from[k][f]), w = to_f32(from[k][g]);
          turn(v, w, table[n]);
          to[k][f] = from_f32<T>(v);
          to[k][g] = from_f32<T>(w);
        }
      }
    }
  }
}

template <typename T, bool VEC, bool HALVES>
cudaError_t launch(const RotaryArgs& a, int num_sms, cudaStream_t stream) {
  const size_t smem = a.pairs * sizeof(float2) * (1 + kWarps) + (a.pairs + 1) / 2 * 2 * sizeof(int);
  // A block a row where a warp a row would leave SMs idle.
  const int row_warps = a.rows < int64_t{num_sms} * kWarps ? kWarps : 1;
  const int64_t blocks = (a.rows + kWarps / row_warps - 1) / (kWarps / row_warps), most = int64_t{num_sms} * 8;
  return launch_dependent(rotary_kernel<T, VEC, HALVES>, dim3(static_cast<unsigned>(blocks < most ? blocks : most)),
                          dim3(kWarps * 32), smem, stream, a, row_warps);
}
template <typename T>
cudaError_t launch_type(const RotaryArgs& a, int num_sms, cudaStream_t stream) {
  if (a.vec) return a.halves ? launch<T, true, true>(a, num_sms, stream) : launch<T, true, false>(a, num_sms, stream);
  return a.halves ? launch<T, false, true>(a, num_sms, stream) : launch<T, false, false>(a, num_sms, stream);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  return bf16 ? launch_type<__nv_bfloat16>(a, num_sms, stream) : launch_type<float>(a, num_sms, stream);
}

}  // namespace mpm
