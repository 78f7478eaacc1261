// The norm after an encoder block, its gate, the scaled residual stream and
// the norm before the next block, in one pass over packed tokens:
//
//   u  = (y - m1) r1 w_post + b_post          (u = y without post_weight)
//   x' = alpha x + gate u
//   h  = (x' - m2) r2 w_pre + b_pre
//
// with r = 1 / sqrt(mean((v - m)^2) + eps), m the row's mean (layer norm) or
// 0 (root mean square).  h is computed from x' before x' is rounded to the
// stream's type, so every output is rounded once.
//
// Bound: HBM (y and x in, x' and h out, about 20 flops an element).  A row
// stays in registers between its sums and is read once.  Rows of up to 1024
// features take one warp, whose sums are shuffles; longer ones take a group
// of warps that meet at a named barrier per sum.  The variance is a second
// pass over the registers around the mean, not E[v^2] - m^2.
#include "block_launch.h"
#include "norm_rows.cuh"

namespace mpm {
namespace {

using namespace norm;

constexpr int kThreads = 256;

template <typename TY, typename TX, int C, bool VEC, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : kThreads) block_norm_kernel(NormForward a, int row_warps) {
  wait_for_previous_grid();
  allow_next_grid();
  __shared__ float2 sh[MULTI ? 32 : 1];
  check_offsets(a.offsets, a.batch, a.rows, a.status);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int w = MULTI ? row_warps : 1;
  const int groups = (blockDim.x >> 5) / w, group = warp / w, in_group = warp % w;
  RowSum<MULTI> sum{sh + group * 2 * w, w, in_group, group + 1, 0};
  const int64_t total = used_rows(a.offsets, a.batch, a.rows);
  const int64_t all = static_cast<int64_t>(gridDim.x) * groups, g = static_cast<int64_t>(blockIdx.x) * groups + group;
  // Neighbouring rows to one group: its image changes only now and then.
  const int64_t per = total / all, extra = total % all;
  const int64_t begin = g * per + (g < extra ? g : extra), end = begin + per + (g < extra ? 1 : 0);
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  const bool post = a.post_weight != nullptr, pre = a.pre_weight != nullptr;
  const float* gate = a.gate;
  int image = 0;
  int64_t image_end = INT64_MAX;
  if (gate != nullptr && a.gate_per_image && begin < end) {
    image = find_image(a.offsets, a.batch, begin);
    image_end = __ldg(a.offsets + image + 1);
    gate = a.gate + static_cast<int64_t>(image) * a.dim;
  }
  int col[C];
#pragma unroll
  for (int c = 0; c < C; ++c) col[c] = first_column<VEC>(c * w + in_group, lane);

  for (int64_t row = begin; row < end; ++row) {
    while (row >= image_end && image < a.batch - 1) {
      ++image;
      image_end = __ldg(a.offsets + image + 1);
      gate = a.gate + static_cast<int64_t>(image) * a.dim;
    }
    float u[C][8], x[C][8];
    const TY* yr = static_cast<const TY*>(a.y) + row * a.y_stride;
    const TX* xr = static_cast<const TX*>(a.residual) + row * a.residual_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) load8<TY, VEC>(yr, col[c], a.dim, u[c]);
#pragma unroll
    for (int c = 0; c < C; ++c) load8<TX, VEC>(xr, col[c], a.dim, x[c]);

    // (mean, 1 / deviation) of a row in registers.
    auto statistics = [&](const float(&v)[C][8]) {
      float m = 0.f;
      if (a.layer) {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) s += v[c][i];
        m = sum(s, 0.f).x * inv_dim;
      }
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = inside<VEC>(col[c], i, a.dim) ? v[c][i] - m : 0.f;
          s = fmaf(d, d, s);
        }
      return make_float2(m, 1.f / sqrtf(fmaf(sum(s, 0.f).x, inv_dim, a.eps)));
    };

    float2 s1 = make_float2(0.f, 1.f), s2 = make_float2(0.f, 1.f);
    if (post) s1 = statistics(u);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (post) {
        float wv[8], bv[8];
        param8<VEC>(a.post_weight, col[c], a.dim, 1.f, wv);
        param8<VEC>(a.post_bias, col[c], a.dim, 0.f, bv);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] = fmaf((u[c][i] - s1.x) * s1.y, wv[i], bv[i]);
      }
      float gv[8];
      param8<VEC>(gate, col[c], a.dim, 1.f, gv);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[c][i] = fmaf(gv[i], u[c][i], a.alpha * x[c][i]);
        if (!inside<VEC>(col[c], i, a.dim)) x[c][i] = 0.f;
      }
      store8<TX, VEC>(static_cast<TX*>(a.residual_out) + row * a.dim, col[c], a.dim, x[c]);
    }
    if (pre) {
      s2 = statistics(x);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float wv[8], bv[8];
        param8<VEC>(a.pre_weight, col[c], a.dim, 1.f, wv);
        param8<VEC>(a.pre_bias, col[c], a.dim, 0.f, bv);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = fmaf((x[c][i] - s2.x) * s2.y, wv[i], bv[i]);
        store8<TY, VEC>(static_cast<TY*>(a.h) + row * a.dim, col[c], a.dim, x[c]);
      }
    }
    if (a.stats != nullptr && in_group == 0 && lane == 0) a.stats[row] = make_float4(s1.x, s1.y, s2.x, s2.y);
  }
}

template <typename TY, typename TX, int C, bool VEC, bool MULTI>
cudaError_t launch_instance(const NormForward& a, int row_warps, int num_sms, cudaStream_t stream) {
  const int warps = MULTI ? 16 / row_warps * row_warps : kThreads / 32;
  const int groups = warps / row_warps;
  static const int per_sm = resident_per_sm(block_norm_kernel<TY, TX, C, VEC, MULTI>, MULTI ? 512 : kThreads, 8);
  const int64_t want = (a.rows + groups - 1) / groups, most = static_cast<int64_t>(num_sms) * per_sm;
  const int grid = static_cast<int>(want < most ? want : most);
  return launch_dependent(block_norm_kernel<TY, TX, C, VEC, MULTI>, dim3(grid), dim3(warps * 32), 0, stream, a,
                          row_warps);
}

template <typename TY, typename TX, bool VEC>
cudaError_t launch_types(const NormForward& a, int num_sms, cudaStream_t stream) {
  const int chunks = (a.dim + kNormWarpCols - 1) / kNormWarpCols;
  switch (chunks) {
    case 1: return launch_instance<TY, TX, 1, VEC, false>(a, 1, num_sms, stream);
    case 2: return launch_instance<TY, TX, 2, VEC, false>(a, 1, num_sms, stream);
    case 3: return launch_instance<TY, TX, 3, VEC, false>(a, 1, num_sms, stream);
    case 4: return launch_instance<TY, TX, 4, VEC, false>(a, 1, num_sms, stream);
    default: return launch_instance<TY, TX, 4, VEC, true>(a, (chunks + 3) / 4, num_sms, stream);
  }
}

template <typename TY, typename TX>
cudaError_t launch_vec(const NormForward& a, bool vec, int num_sms, cudaStream_t stream) {
  return vec ? launch_types<TY, TX, true>(a, num_sms, stream) : launch_types<TY, TX, false>(a, num_sms, stream);
}

}  // namespace

cudaError_t launch_block_norm(const NormForward& a, NormTypes types, bool vec, int num_sms, cudaStream_t stream) {
  switch (types) {
    case NormTypes::kF32: return launch_vec<float, float>(a, vec, num_sms, stream);
    case NormTypes::kBf16: return launch_vec<__nv_bfloat16, __nv_bfloat16>(a, vec, num_sms, stream);
    case NormTypes::kBf16StreamF32: return launch_vec<__nv_bfloat16, float>(a, vec, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace mpm
