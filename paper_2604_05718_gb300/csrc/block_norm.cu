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
//
// A warp's parameters are as many bytes as several rows.  They lie in shared
// memory in the order in which lanes take them (16 bytes a lane, no bank
// conflicts), the norm after the block and the gate folded into two vectors,
// A = gate w_post and B = gate b_post: x' = alpha x + n1 A + B.  What bounds the
// kernel beside HBM is the accesses to them (54208 x 768 bf16, layer norm on both
// sides and a gate per image, 333 MB: 85 us with all five vectors read through
// L1, 64 with the gate alone, 62 folded; 30000 x 1024: 49 to 45).
#include <atomic>

#include "block_launch.h"
#include "norm_rows.cuh"
#include "ptx.cuh"

namespace mpm {
namespace {

using namespace norm;

constexpr int kThreads = 256;
constexpr int kSmShared = 228 * 1024;     // shared memory of an SM
constexpr int kBlockShared = 225 * 1024;  // the most that a block's vectors take

// Blocks that an SM has to hold: the registers a thread may take (80 for 3 blocks, 64 for 4).
__host__ __device__ constexpr int min_blocks(int chunks, bool vec, bool multi) {
  return multi ? 1 : vec ? (chunks == 1 ? 4 : chunks < 4 ? 3 : 2) : chunks < 3 ? 3 : 2;
}
// Rows that a warp takes at once: two where they are short (registers for more warps do more for longer ones).
__host__ __device__ constexpr int rows_at_once(int chunks, bool multi) { return multi || chunks > 1 ? 1 : 2; }

template <typename TY, typename TX, int C, bool VEC, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : kThreads, min_blocks(C, VEC, MULTI))
    block_norm_kernel(NormForward a, int row_warps, int staged_vectors) {
  constexpr int R = rows_at_once(C, MULTI);
  // Rows so long that the vectors have no room in shared memory read them through L1.
  const bool staged = !MULTI || staged_vectors != 0;
  __shared__ float sh[MULTI ? 32 : 1];
  // w_pre and b_pre, then A and B: of the block, or (a gate per image) of each group.
  extern __shared__ __align__(16) float4 vectors[];
  wait_for_previous_grid();
  allow_next_grid();
  check_offsets(a.offsets, a.batch, a.rows, a.status);
  const bool post = a.post_weight != nullptr, pre = a.pre_weight != nullptr;
  const bool per_image = a.gate != nullptr && a.gate_per_image;
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
  const int w = MULTI ? row_warps : 1;
  const int groups = (blockDim.x >> 5) / w, group = warp / w, in_group = warp % w;
  RowSum<MULTI> sum{sh + group * 2 * w, w, in_group, group + 1, 0};
  const int64_t total = used_rows(a.offsets, a.batch, a.rows);
  const int64_t all = static_cast<int64_t>(gridDim.x) * groups, g = static_cast<int64_t>(blockIdx.x) * groups + group;
  // Neighbouring rows to one group: its image changes only now and then.
  const int64_t per = static_cast<uint32_t>(total) / static_cast<uint32_t>(all), extra = total - per * all;
  const int64_t begin = g * per + (g < extra ? g : extra), end = begin + per + (g < extra ? 1 : 0);
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  int col[C];
#pragma unroll
  for (int c = 0; c < C; ++c) col[c] = first_column<VEC>(c * w + in_group, lane);

  const int quads = w * C * kNormWarpCols / 4;  // of one vector
  const auto shared_vector = [&](int k) { return SharedVector{vectors + k * quads, w * 32, in_group * 32 + lane}; };
  const SharedVector w_pre = shared_vector(0), b_pre = shared_vector(1);
  const SharedVector scale = shared_vector(2 + (per_image ? 2 * group : 0)), shift = shared_vector(3 + (per_image ? 2 * group : 0));
  auto fold = [&](const float* gate, int c, F8& A, F8& B) {
    const F8 g8 = param8<VEC>(gate, col[c], a.dim, 1.f);
    A = param8<VEC>(a.post_weight, col[c], a.dim, 1.f);
    B = param8<VEC>(a.post_bias, col[c], a.dim, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      A.p[k] = mul(g8.p[k], A.p[k]);
      B.p[k] = mul(g8.p[k], B.p[k]);
    }
  };
  auto open_gate = [&](const float* gate) {  // each thread reads back its own columns only
#pragma unroll
    for (int c = 0; c < C; ++c) {
      F8 A, B;
      fold(gate, c, A, B);
      scale.set(c, A);
      shift.set(c, B);
    }
  };
  const float* gate = a.gate;
  int image = 0;
  int64_t image_end = INT64_MAX;
  auto open_image = [&](int b) {
    image = b;
    image_end = __ldg(a.offsets + b + 1);
    gate = a.gate + static_cast<int64_t>(b) * a.dim;
    if (staged) open_gate(gate);
  };
  if (staged) {
    if (group == 0) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        w_pre.set(c, param8<VEC>(a.pre_weight, col[c], a.dim, 1.f));
        b_pre.set(c, param8<VEC>(a.pre_bias, col[c], a.dim, 0.f));
      }
      if (!per_image) open_gate(gate);
    }
    __syncthreads();
  }
  if (per_image && begin < end) open_image(find_image(a.offsets, a.batch, begin));

  for (int64_t row = begin; row < end;) {
    if (row >= image_end && image < a.batch - 1) {
      int b = image + 1;
      while (b < a.batch - 1 && row >= __ldg(a.offsets + b + 1)) ++b;
      open_image(b);
    }
    // The last row stands in for one past the run's or the image's end, and is written once.
    int64_t at[R];
    int count = 1;
    at[0] = row;
#pragma unroll
    for (int r = 1; r < R; ++r) {
      const bool more = row + r < end && (row + r < image_end || image == a.batch - 1);
      at[r] = more ? row + r : row;
      count += more ? 1 : 0;
    }
    row += count;
    F8 u[R][C], x[R][C];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        u[r][c] = load8<TY, VEC>(static_cast<const TY*>(a.y) + at[r] * a.y_stride, col[c], a.dim);
#pragma unroll
      for (int c = 0; c < C; ++c)
        x[r][c] = load8<TX, VEC>(static_cast<const TX*>(a.residual) + at[r] * a.residual_stride, col[c], a.dim);
    }

    // Takes the mean out of rows in registers; 1 / deviation and the mean of each.
    auto standardise = [&](F8(&v)[R][C], float2(&s)[R]) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[r].x = 0.f;
      if (a.layer) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float2 t = pair(0.f);
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k) t = add(t, v[r][c].p[k]);
          s[r].x = t.x + t.y;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) s[r].x = sum(s[r].x) * inv_dim;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const F8 in = mask8<VEC>(col[c], a.dim);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[r][c].p[k] = fma(in.p[k], pair(-s[r].x), v[r][c].p[k]);
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float2 t = pair(0.f);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) t = fma(v[r][c].p[k], v[r][c].p[k], t);
        s[r].y = t.x + t.y;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) s[r].y = 1.f / sqrtf(fmaf(sum(s[r].y), inv_dim, a.eps));
    };

    float2 s1[R], s2[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s1[r] = s2[r] = make_float2(0.f, 1.f);
    if (post) standardise(u, s1);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      F8 A, B;
      if (staged) {
        A = scale.get(c);
        B = shift.get(c);
      } else {
        fold(gate, c, A, B);
      }
      // Outside the row u, x and B are zeros, and so is x'.
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          x[r][c].p[k] = fma(mul(u[r][c].p[k], pair(s1[r].y)), A.p[k], fma(pair(a.alpha), x[r][c].p[k], B.p[k]));
        if (r < count) store8<TX, VEC>(static_cast<TX*>(a.residual_out) + at[r] * a.dim, col[c], a.dim, x[r][c]);
      }
    }
    if (pre) {
      standardise(x, s2);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const F8 wv = staged ? w_pre.get(c) : param8<VEC>(a.pre_weight, col[c], a.dim, 1.f);
        const F8 bv = staged ? b_pre.get(c) : param8<VEC>(a.pre_bias, col[c], a.dim, 0.f);
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
          for (int k = 0; k < 4; ++k) x[r][c].p[k] = fma(mul(x[r][c].p[k], pair(s2[r].y)), wv.p[k], bv.p[k]);
          if (r < count) store8<TY, VEC>(static_cast<TY*>(a.h) + at[r] * a.dim, col[c], a.dim, x[r][c]);
        }
      }
    }
    if (a.stats != nullptr && in_group == 0 && lane == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (r < count) a.stats[at[r]] = make_float4(s1[r].x, s1[r].y, s2[r].x, s2[r].y);
    }
  }
}

template <typename TY, typename TX, int C, bool VEC, bool MULTI>
cudaError_t launch_instance(const NormForward& a, int row_warps, int num_sms, cudaStream_t stream) {
  const auto kernel = block_norm_kernel<TY, TX, C, VEC, MULTI>;
  const int warps = MULTI ? 16 / row_warps * row_warps : kThreads / 32;
  const int groups = warps / row_warps;
  static const int by_registers = resident_per_sm(kernel, MULTI ? 512 : kThreads, 8);
  const int owners = a.gate != nullptr && a.gate_per_image ? groups : 1;
  int smem = (2 + 2 * owners) * row_warps * C * kNormWarpCols * static_cast<int>(sizeof(float));
  const int staged = smem <= kBlockShared;
  if (!staged) smem = 0;
  static std::atomic<uint64_t> attr_done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(attr_done.load() & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlockShared);
    if (e != cudaSuccess) return e;
    attr_done.fetch_or(bit);
  }
  const int fit = kSmShared / (smem + 2048);
  const int per_sm = fit < by_registers ? fit : by_registers;
  const int64_t want = (a.rows + groups - 1) / groups, most = static_cast<int64_t>(num_sms) * per_sm;
  const int grid = static_cast<int>(want < most ? want : most);
  return launch_dependent(kernel, dim3(grid), dim3(warps * 32), static_cast<size_t>(smem), stream, a, row_warps, staged);
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
