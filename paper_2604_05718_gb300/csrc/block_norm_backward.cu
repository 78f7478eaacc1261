// Gradients of block_norm (block_norm.cu).  For a row, with n1 and n2 the
// normalised rows of y and of x', dh and dx' the gradients of h and x':
//
//   a  = dh w_pre,   G = dx' + r2 (a - [layer] mean(a) - n2 mean(a n2))
//   dx = alpha G,    du = gate G
//   c  = du w_post,  dy = r1 (c - [layer] mean(c) - n1 mean(c n1))   (dy = du without w_post)
//
// and, summed over rows, d w_pre = dh n2, d b_pre = dh, d w_post = du n1,
// d b_post = du, d gate = u G (over an image's rows for a gate per image).
// n1, u and n2 come from y, x and the four statistics that the forward pass
// kept: x' itself is formed again in fp32, so no rounding of it enters.
//
// Bound: HBM (y, x, dx' and dh in, dy and dx out).  A group of warps keeps
// eight columns a thread of a run of neighbouring rows, with the parameters
// and all five column sums in registers; the sums leave them once, at the end
// of the run (or of an image, for its gate).  Column sums are joined in fixed
// order, first over the groups of a block in shared memory, then over blocks
// by a second kernel: no atomics, the same bits every time.
#include "block_launch.h"
#include "norm_rows.cuh"

namespace mpm {
namespace {

using namespace norm;

constexpr int kMaxBlocks = 160;  // blocks of the row kernel: one per SM
constexpr int kWarps = 16;       // warps of a block, less what does not make up a group
constexpr int kSums = 5;         // column sums: w_pre, b_pre, w_post, b_post, gate per channel

// Chunks of columns a thread holds: one, as long as 16 warps span the row.
__host__ __device__ constexpr int chunks_per_thread(int dim) {
  return dim <= 16 * kNormWarpCols ? 1 : (dim <= 32 * kNormWarpCols ? 2 : 4);
}
__host__ __device__ constexpr int warps_per_row(int dim) {
  return (dim + kNormWarpCols * chunks_per_thread(dim) - 1) / (kNormWarpCols * chunks_per_thread(dim));
}

// The run of rows of group g out of `all`, sizes one apart at most.
struct Run {
  int64_t begin, end;
};
__device__ __forceinline__ Run run_of(int64_t g, int64_t all, int64_t total) {
  const int64_t per = total / all, extra = total % all;
  const int64_t begin = g * per + (g < extra ? g : extra);
  return {begin, begin + per + (g < extra ? 1 : 0)};
}
__device__ __forceinline__ int64_t group_of(int64_t row, int64_t all, int64_t total) {
  const int64_t per = total / all, extra = total % all, long_rows = extra * (per + 1);
  return row < long_rows ? row / (per + 1) : extra + (row - long_rows) / per;
}

// Workspace: column sums [kSums][blocks][dim], then the gate's parts of the
// images that a run shares with an earlier one (head) or a later one (tail).
struct Parts {
  float* sums;
  float* head;
  float* tail;
};
__device__ __forceinline__ Parts parts_of(const NormBackward& a, int blocks, int64_t all) {
  float* sums = a.partial;
  float* head = sums + static_cast<int64_t>(kSums) * blocks * a.dim;
  return {sums, head, head + all * a.dim};
}

template <typename TY, typename TX, int C, bool VEC, bool MULTI>
__global__ void __launch_bounds__(kWarps * 32, 1) block_norm_backward_kernel(NormBackward a, int row_warps) {
  wait_for_previous_grid();
  allow_next_grid();
  extern __shared__ float joined[];  // [dim], when the block holds several groups
  __shared__ float2 sh[MULTI ? 2 * kWarps : 1];
  check_offsets(a.offsets, a.batch, a.rows, a.status);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int w = MULTI ? row_warps : 1;
  const int groups = (blockDim.x >> 5) / w, group = warp / w, in_group = warp % w;
  RowSum<MULTI> sum{sh + group * 2 * w, w, in_group, group + 1, 0};
  const int64_t total = used_rows(a.offsets, a.batch, a.rows);
  const int64_t all = static_cast<int64_t>(gridDim.x) * groups, g = static_cast<int64_t>(blockIdx.x) * groups + group;
  const Run run = run_of(g, all, total);
  const Parts parts = parts_of(a, gridDim.x, all);
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  const bool post = a.post_weight != nullptr, per_image = a.gate != nullptr && a.gate_per_image;

  int col[C];
  float w_pre[C][8], w_post[C][8], b_post[C][8], gate[C][8];
  float s_wpre[C][8], s_bpre[C][8], s_wpost[C][8], s_bpost[C][8], s_gate[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = first_column<VEC>(c * w + in_group, lane);
    param8<VEC>(a.pre_weight, col[c], a.dim, 0.f, w_pre[c]);  // absent: h has no part in the gradients
    param8<VEC>(a.post_weight, col[c], a.dim, 1.f, w_post[c]);
    param8<VEC>(a.post_bias, col[c], a.dim, 0.f, b_post[c]);
    if (!per_image) param8<VEC>(a.gate, col[c], a.dim, 1.f, gate[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) s_wpre[c][i] = s_bpre[c][i] = s_wpost[c][i] = s_bpost[c][i] = s_gate[c][i] = 0.f;
  }

  int image = 0;
  int64_t image_begin = 0, image_end = INT64_MAX;
  auto open_image = [&](int b) {
    image = b;
    image_begin = __ldg(a.offsets + b);
    image_end = __ldg(a.offsets + b + 1);
#pragma unroll
    for (int c = 0; c < C; ++c) param8<VEC>(a.gate + static_cast<int64_t>(b) * a.dim, col[c], a.dim, 0.f, gate[c]);
  };
  // The gate's sum over this run's rows of the image: all of its rows, or a part.
  auto close_image = [&]() {
    float* to = image_begin < run.begin ? parts.head + g * a.dim
                : image_end <= run.end  ? (a.d_gate == nullptr ? nullptr : a.d_gate + static_cast<int64_t>(image) * a.dim)
                                        : parts.tail + g * a.dim;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (to != nullptr) store8<float, VEC>(to, col[c], a.dim, s_gate[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s_gate[c][i] = 0.f;
    }
  };
  if (per_image && run.begin < run.end) open_image(find_image(a.offsets, a.batch, run.begin));

  for (int64_t row = run.begin; row < run.end; ++row) {
    if (row >= image_end && image < a.batch - 1) {
      close_image();
      int b = image + 1;
      while (b < a.batch - 1 && row >= __ldg(a.offsets + b + 1)) ++b;
      open_image(b);
    }
    float y[C][8], x[C][8], dh[C][8], dxo[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      load8<TY, VEC>(static_cast<const TY*>(a.y) + row * a.y_stride, col[c], a.dim, y[c]);
      load8<TX, VEC>(static_cast<const TX*>(a.residual) + row * a.residual_stride, col[c], a.dim, x[c]);
      if (a.d_h != nullptr) {
        load8<TY, VEC>(static_cast<const TY*>(a.d_h) + row * a.d_h_stride, col[c], a.dim, dh[c]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) dh[c][i] = 0.f;
      }
      if (a.d_residual_out != nullptr) {
        load8<TX, VEC>(static_cast<const TX*>(a.d_residual_out) + row * a.d_residual_out_stride, col[c], a.dim,
                       dxo[c]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) dxo[c][i] = 0.f;
      }
    }
    const float4 st = __ldg(a.stats + row);
    float sa = 0.f, san = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n1 = (y[c][i] - st.x) * st.y;
        const float u = fmaf(n1, w_post[c][i], b_post[c][i]);
        const float n2 = (fmaf(gate[c][i], u, a.alpha * x[c][i]) - st.z) * st.w;
        s_bpre[c][i] += dh[c][i];
        s_wpre[c][i] = fmaf(dh[c][i], n2, s_wpre[c][i]);
        const float aw = dh[c][i] * w_pre[c][i];  // zero outside the row: w_pre is
        sa += aw;
        san = fmaf(aw, n2, san);
        x[c][i] = n2;
        dh[c][i] = aw;
        y[c][i] = n1;
      }
    const float2 m2 = sum(sa, san);
    const float mean_a = a.layer ? m2.x * inv_dim : 0.f, mean_an = m2.y * inv_dim;
    float sc = 0.f, scn = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n1 = y[c][i];
        const float grad = fmaf(st.w, dh[c][i] - mean_a - x[c][i] * mean_an, dxo[c][i]);
        s_gate[c][i] = fmaf(grad, fmaf(n1, w_post[c][i], b_post[c][i]), s_gate[c][i]);
        const float du = gate[c][i] * grad;
        s_bpost[c][i] += du;
        s_wpost[c][i] = fmaf(du, n1, s_wpost[c][i]);
        const float cw = inside<VEC>(col[c], i, a.dim) ? du * w_post[c][i] : 0.f;
        sc += cw;
        scn = fmaf(cw, n1, scn);
        dxo[c][i] = a.alpha * grad;
        dh[c][i] = cw;
      }
      store8<TX, VEC>(static_cast<TX*>(a.d_residual) + row * a.dim, col[c], a.dim, dxo[c]);
    }
    if (post) {
      const float2 m1 = sum(sc, scn);
      const float mean_c = a.layer ? m1.x * inv_dim : 0.f, mean_cn = m1.y * inv_dim;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dh[c][i] = st.y * (dh[c][i] - mean_c - y[c][i] * mean_cn);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) store8<TY, VEC>(static_cast<TY*>(a.d_y) + row * a.dim, col[c], a.dim, dh[c]);
  }
  if (per_image && run.begin < run.end) close_image();

  // Column sums of the block's groups, joined in the groups' order.
  auto leave = [&](float(&s)[C][8], int which) {
    float* out = parts.sums + (static_cast<int64_t>(which) * gridDim.x + blockIdx.x) * a.dim;
    for (int k = 0; k < groups; ++k) {
      if (group == k) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if (k > 0) {
            float v[8];
            // Each column belongs to the same lane and warp of every group.
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (inside<VEC>(col[c], i, a.dim)) v[i] = joined[column<VEC>(col[c], i)];
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c][i] += inside<VEC>(col[c], i, a.dim) ? v[i] : 0.f;
          }
          if (k == groups - 1) {
            store8<float, VEC>(out, col[c], a.dim, s[c]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (inside<VEC>(col[c], i, a.dim)) joined[column<VEC>(col[c], i)] = s[c][i];
          }
        }
      }
      if (groups > 1) __syncthreads();
    }
  };
  if (a.d_pre_weight != nullptr) leave(s_wpre, 0);
  if (a.d_pre_bias != nullptr) leave(s_bpre, 1);
  if (a.d_post_weight != nullptr) leave(s_wpost, 2);
  if (a.d_post_bias != nullptr) leave(s_bpost, 3);
  if (a.d_gate != nullptr && !per_image) leave(s_gate, 4);
}

constexpr int kJoinCols = 32, kJoinRows = 16;

// Column sums over blocks, and the gates of images that several runs share.
__global__ void __launch_bounds__(kJoinCols * kJoinRows) block_norm_join_kernel(NormBackward a, int blocks, int groups) {
  wait_for_previous_grid();
  allow_next_grid();
  __shared__ float part[kJoinRows][kJoinCols];
  const int64_t all = static_cast<int64_t>(blocks) * groups;
  const Parts parts = parts_of(a, blocks, all);
  const bool per_image = a.gate != nullptr && a.gate_per_image;
  float* const outs[kSums] = {a.d_pre_weight, a.d_pre_bias, a.d_post_weight, a.d_post_bias,
                              per_image ? nullptr : a.d_gate};
  const int col_blocks = (a.dim + kJoinCols - 1) / kJoinCols;
  const int x = threadIdx.x % kJoinCols, r = threadIdx.x / kJoinCols;
  const int which = blockIdx.x / col_blocks;
  if (which < kSums) {
    if (outs[which] == nullptr) return;
    const int col = blockIdx.x % col_blocks * kJoinCols + x;
    const float* in = parts.sums + static_cast<int64_t>(which) * blocks * a.dim;
    float s = 0.f;
    if (col < a.dim)
      for (int b = r; b < blocks; b += kJoinRows) s += in[static_cast<int64_t>(b) * a.dim + col];
    part[r][x] = s;
    __syncthreads();
    if (r == 0 && col < a.dim) {
      for (int k = 1; k < kJoinRows; ++k) s += part[k][x];
      outs[which][col] = s;
    }
    return;
  }
  const int wide = (a.dim + blockDim.x - 1) / blockDim.x, k = blockIdx.x - kSums * col_blocks;
  const int image = k / wide, col = k % wide * blockDim.x + threadIdx.x;
  if (image >= a.batch || col >= a.dim || a.d_gate == nullptr) return;
  const int64_t total = used_rows(a.offsets, a.batch, a.rows);
  int64_t lo = __ldg(a.offsets + image), hi = __ldg(a.offsets + image + 1);
  lo = lo < 0 ? 0 : lo;
  hi = hi < total ? hi : total;
  float* out = a.d_gate + static_cast<int64_t>(image) * a.dim + col;
  if (hi <= lo) {
    *out = 0.f;
    return;
  }
  const int64_t first = group_of(lo, all, total), last = group_of(hi - 1, all, total);
  if (first == last) return;  // written by its run
  float s = parts.tail[first * a.dim + col];
  for (int64_t g = first + 1; g <= last; ++g) s += parts.head[g * a.dim + col];
  *out = s;
}

int groups_of(int dim) { return kWarps / warps_per_row(dim); }

template <typename TY, typename TX, int C, bool VEC, bool MULTI>
cudaError_t launch_instance(const NormBackward& a, int num_sms, cudaStream_t stream) {
  const int w = warps_per_row(a.dim), groups = groups_of(a.dim);
  const int64_t want = a.rows > 0 ? (a.rows + groups - 1) / groups : 1;  // without rows the sums are still written
  const int most = num_sms < kMaxBlocks ? num_sms : kMaxBlocks;
  const int grid = static_cast<int>(want < most ? want : most);
  const size_t smem = groups > 1 ? sizeof(float) * a.dim : 0;
  cudaError_t e = launch_dependent(block_norm_backward_kernel<TY, TX, C, VEC, MULTI>, dim3(grid), dim3(groups * w * 32),
                                   smem, stream, a, w);
  if (e != cudaSuccess) return e;
  const bool per_image = a.gate != nullptr && a.gate_per_image && a.d_gate != nullptr;
  if (!per_image && a.d_gate == nullptr && a.d_pre_weight == nullptr && a.d_pre_bias == nullptr &&
      a.d_post_weight == nullptr && a.d_post_bias == nullptr)
    return cudaSuccess;
  const int threads = kJoinCols * kJoinRows;
  const int64_t joins = static_cast<int64_t>(kSums) * ((a.dim + kJoinCols - 1) / kJoinCols) +
                        (per_image ? static_cast<int64_t>(a.batch) * ((a.dim + threads - 1) / threads) : 0);
  return launch_dependent(block_norm_join_kernel, dim3(static_cast<unsigned>(joins)), dim3(threads), 0, stream, a, grid,
                          groups);
}

template <typename TY, typename TX, bool VEC>
cudaError_t launch_types(const NormBackward& a, int num_sms, cudaStream_t stream) {
  if (warps_per_row(a.dim) == 1) return launch_instance<TY, TX, 1, VEC, false>(a, num_sms, stream);
  switch (chunks_per_thread(a.dim)) {
    case 1: return launch_instance<TY, TX, 1, VEC, true>(a, num_sms, stream);
    case 2: return launch_instance<TY, TX, 2, VEC, true>(a, num_sms, stream);
    default: return launch_instance<TY, TX, 4, VEC, true>(a, num_sms, stream);
  }
}

template <typename TY, typename TX>
cudaError_t launch_vec(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  return vec ? launch_types<TY, TX, true>(a, num_sms, stream) : launch_types<TY, TX, false>(a, num_sms, stream);
}

}  // namespace

size_t block_norm_workspace_floats(int dim) {
  return static_cast<size_t>(dim) * kMaxBlocks * (kSums + 2 * static_cast<size_t>(groups_of(dim)));
}

cudaError_t launch_block_norm_backward(const NormBackward& a, NormTypes types, bool vec, int num_sms,
                                       cudaStream_t stream) {
  switch (types) {
    case NormTypes::kF32: return launch_vec<float, float>(a, vec, num_sms, stream);
    case NormTypes::kBf16: return launch_vec<__nv_bfloat16, __nv_bfloat16>(a, vec, num_sms, stream);
    case NormTypes::kBf16StreamF32: return launch_vec<__nv_bfloat16, float>(a, vec, num_sms, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace mpm
