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
// The gate enters a row as A = gate w_post and B = gate b_post alone, and the
// sums of the rows under one gate follow from two, S1 = sum G n1 and S0 = sum G:
// d w_post += gate S1, d b_post += gate S0, d gate = w_post S1 + b_post S0.
//
// Bound: HBM (y, x, dx' and dh in, dy and dx out).  A group of warps keeps
// eight columns a thread of a run of neighbouring rows, with A, B and the
// column sums in registers; the sums leave them once, at the end of the run
// (or of an image, for its gate).  Column sums are joined in fixed order, first
// over the groups of a block in shared memory, then over blocks by a second
// kernel: no atomics, the same bits every time.
//
// The sums take many registers, so few warps are there to hide the loads.
// Rows that are 16-byte aligned therefore come through a ring in shared
// memory, filled by bulk copies some pairs of rows ahead; two rows are worked
// on at once and share their two barriers.  54208 x 768 bf16, layer norm on
// both sides: BWD0 us from loads in place, BWD1 through the ring.
#include <atomic>

#include "block_launch.h"
#include "norm_rows.cuh"
#include "ptx.cuh"

namespace mpm {
namespace {

using namespace norm;

constexpr int kMaxBlocks = 160;  // blocks of the row kernel: one per SM
constexpr int kSums = 5;         // column sums: w_pre, b_pre, w_post, b_post, gate per channel
constexpr int kMaxRing = 4;      // stages of a group's ring
constexpr uint64_t kWaitNs = 2000000000ull;

// Chunks of columns that a thread holds: one as long as 12 warps span the row
// (168 registers a thread hold the sums and two rows), two as long as 12 warps
// do then, else four in up to 16 warps.
__host__ __device__ constexpr int chunks_per_thread(int dim) {
  return dim <= 12 * kNormWarpCols ? 1 : (dim <= 24 * kNormWarpCols ? 2 : 4);
}
__host__ __device__ constexpr int block_warps(int chunks) { return chunks == 4 ? 16 : 12; }
__host__ __device__ constexpr int warps_per_row(int dim) {
  return (dim + kNormWarpCols * chunks_per_thread(dim) - 1) / (kNormWarpCols * chunks_per_thread(dim));
}
// Shared memory for the rings: what a block may have (227 KB), less the weight in it and 2 KB of barriers and sums.
__host__ __device__ constexpr int ring_bytes(int chunks) {
  return 225 * 1024 - chunks * 2 * block_warps(chunks) * 32 * 16;
}
// Rows that a group works on at once.
__host__ __device__ constexpr int rows_at_once(int chunks) { return chunks == 1 ? 2 : 1; }

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

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   ptx::smem_addr(dst)),
               "l"(src), "r"(bytes), "r"(ptx::smem_addr(bar))
               : "memory");
}

// One stage of a group's ring: R rows of y, x, dh and dx' one after another, and their statistics.
template <typename TY, typename TX, int R>
struct Stage {
  static constexpr int kRowBytes = 2 * sizeof(TY) + 2 * sizeof(TX);
  __host__ __device__ static constexpr int bytes(int dim) { return R * (dim * kRowBytes + 16); }
  uint8_t* base;
  int dim;
  __device__ __forceinline__ TY* y() const { return reinterpret_cast<TY*>(base); }
  __device__ __forceinline__ TY* d_h() const { return y() + R * dim; }
  __device__ __forceinline__ TX* x() const { return reinterpret_cast<TX*>(d_h() + R * dim); }
  __device__ __forceinline__ TX* d_x() const { return x() + R * dim; }
  __device__ __forceinline__ float4* stats() const { return reinterpret_cast<float4*>(d_x() + R * dim); }
};

// n rows of a matrix into a stage: one copy if they lie next to one another.
template <typename T>
__device__ __forceinline__ void load_rows(T* dst, const void* src, int64_t stride, int64_t row, int n, int dim, uint64_t* bar) {
  const T* from = static_cast<const T*>(src) + row * stride;
  if (stride == dim) {
    bulk_load(dst, from, static_cast<uint32_t>(n * dim * sizeof(T)), bar);
  } else {
    for (int i = 0; i < n; ++i) bulk_load(dst + i * dim, from + i * stride, static_cast<uint32_t>(dim * sizeof(T)), bar);
  }
}

// Eight columns of a staged row.
template <typename T>
__device__ __forceinline__ F8 staged8(const T* row, int col, int dim) {
  if (col >= dim) return all8(0.f);
  if constexpr (sizeof(T) == 2) {
    return widen(*reinterpret_cast<const uint4*>(row + col));
  } else {
    const float4* p = reinterpret_cast<const float4*>(row + col);
    return join(p[0], p[1]);
  }
}

// RING: 16-byte aligned rows through shared memory (VEC accesses); otherwise loads of single elements.
template <typename TY, typename TX, int C, bool RING, bool MULTI>
__global__ void __launch_bounds__(block_warps(C) * 32, 1)
    block_norm_backward_kernel(NormBackward a, int row_warps, int ring) {
  constexpr int R = rows_at_once(C), N = 2 * R;
  using S = Stage<TY, TX, R>;
  extern __shared__ __align__(16) uint8_t dynamic[];  // the groups' rings; afterwards float [dim] to join sums in
  __shared__ __align__(16) float sh[2 * block_warps(C) * N];
  // The weight that is used least, out of registers: chunk, half of its eight columns, thread of the row.
  __shared__ float4 pre_weight[C][2][block_warps(C) * 32];
  __shared__ uint64_t full[block_warps(C)][kMaxRing];
  __shared__ int dead;  // a wait ran out: no further one is taken
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int w = MULTI ? row_warps : 1;
  const int groups = (blockDim.x >> 5) / w, group = warp / w, in_group = warp % w;
  if (threadIdx.x == 0) {
    dead = 0;
    if constexpr (RING) {
      for (int k = 0; k < groups; ++k)
        for (int s = 0; s < ring; ++s) ptx::mbar_init(&full[k][s], 1);
      ptx::fence_barrier_init();
    }
  }
  __syncthreads();
  wait_for_previous_grid();
  allow_next_grid();
  check_offsets(a.offsets, a.batch, a.rows, a.status);
  GroupSums<N, MULTI> sum{sh + group * 2 * w * N, w, in_group, group + 1, 0};
  const int64_t total = used_rows(a.offsets, a.batch, a.rows);
  const int64_t all = static_cast<int64_t>(gridDim.x) * groups, g = static_cast<int64_t>(blockIdx.x) * groups + group;
  const Run run = run_of(g, all, total);
  const Parts parts = parts_of(a, gridDim.x, all);
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  const bool post = a.post_weight != nullptr, per_image = a.gate != nullptr && a.gate_per_image;

  // Stage s of the run: rows run.begin + s R .., into slot s % ring.
  auto slot = [&](int64_t s) {
    return S{dynamic + (static_cast<int64_t>(group) * ring + s % ring) * S::bytes(a.dim), a.dim};
  };
  const int64_t stages = (run.end - run.begin + R - 1) / R;
  auto fill = [&](int64_t s) {  // by one thread of the group
    const int64_t row = run.begin + s * R;
    const int n = run.end - row < R ? static_cast<int>(run.end - row) : R;
    uint64_t* bar = &full[group][s % ring];
    const S to = slot(s);
    const uint32_t bytes = n * (a.dim * (sizeof(TY) + sizeof(TX) + (a.d_h != nullptr ? sizeof(TY) : 0) +
                                         (a.d_residual_out != nullptr ? sizeof(TX) : 0)) + 16);
    ptx::mbar_arrive_expect_tx(bar, bytes);
    load_rows<TY>(to.y(), a.y, a.y_stride, row, n, a.dim, bar);
    load_rows<TX>(to.x(), a.residual, a.residual_stride, row, n, a.dim, bar);
    if (a.d_h != nullptr) load_rows<TY>(to.d_h(), a.d_h, a.d_h_stride, row, n, a.dim, bar);
    if (a.d_residual_out != nullptr)
      load_rows<TX>(to.d_x(), a.d_residual_out, a.d_residual_out_stride, row, n, a.dim, bar);
    bulk_load(to.stats(), a.stats + row, n * 16, bar);
  };
  const bool filler = in_group == 0 && lane == 0;
  if constexpr (RING) {
    if (filler)
      for (int64_t s = 0; s < ring && s < stages; ++s) fill(s);
  }

  int col[C];
  F8 scale[C], shift[C];                      // A and B
  F8 s_wpre[C], s_bpre[C], s_one[C], s_n1[C]; // sums of dh n2, dh, G and G n1
  F8 s_wpost[C], s_bpost[C], s_gate[C];       // of the gates closed so far; the last gate's
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = first_column<RING>(c * w + in_group, lane);
    if (group == 0) {
      const F8 v = param8<RING>(a.pre_weight, col[c], a.dim, 0.f);  // absent: h has no part in the gradients
      pre_weight[c][0][in_group * 32 + lane] = make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y);
      pre_weight[c][1][in_group * 32 + lane] = make_float4(v.p[2].x, v.p[2].y, v.p[3].x, v.p[3].y);
    }
    s_wpre[c] = s_bpre[c] = s_one[c] = s_n1[c] = s_wpost[c] = s_bpost[c] = s_gate[c] = all8(0.f);
  }
  __syncthreads();

  // Rows under one gate: between opening and closing it.
  auto open_gate = [&](const float* gate) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const F8 g8 = param8<RING>(gate, col[c], a.dim, 1.f);
      const F8 w8 = param8<RING>(a.post_weight, col[c], a.dim, 1.f), b8 = param8<RING>(a.post_bias, col[c], a.dim, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        scale[c].p[k] = mul(g8.p[k], w8.p[k]);
        shift[c].p[k] = mul(g8.p[k], b8.p[k]);
      }
    }
  };
  auto close_gate = [&](const float* gate) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const F8 g8 = param8<RING>(gate, col[c], a.dim, 1.f);
      const F8 w8 = param8<RING>(a.post_weight, col[c], a.dim, 1.f), b8 = param8<RING>(a.post_bias, col[c], a.dim, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s_wpost[c].p[k] = fma(g8.p[k], s_n1[c].p[k], s_wpost[c].p[k]);
        s_bpost[c].p[k] = fma(g8.p[k], s_one[c].p[k], s_bpost[c].p[k]);
        s_gate[c].p[k] = fma(w8.p[k], s_n1[c].p[k], mul(b8.p[k], s_one[c].p[k]));
      }
      s_n1[c] = s_one[c] = all8(0.f);
    }
  };
  int image = 0;
  int64_t image_begin = 0, image_end = INT64_MAX;
  auto gate_of = [&](int b) { return a.gate + static_cast<int64_t>(b) * a.dim; };
  auto open_image = [&](int b) {
    image = b;
    image_begin = __ldg(a.offsets + b);
    image_end = __ldg(a.offsets + b + 1);
    open_gate(gate_of(b));
  };
  // The gate's gradient over this run's rows of the image: all of its rows, or a part.
  auto close_image = [&]() {
    close_gate(gate_of(image));
    float* to = image_begin < run.begin ? parts.head + g * a.dim
                : image_end <= run.end  ? (a.d_gate == nullptr ? nullptr : a.d_gate + static_cast<int64_t>(image) * a.dim)
                                        : parts.tail + g * a.dim;
    if (to == nullptr) return;
#pragma unroll
    for (int c = 0; c < C; ++c) store8<float, RING>(to, col[c], a.dim, s_gate[c]);
  };
  if (!per_image) open_gate(a.gate);
  else if (run.begin < run.end) open_image(find_image(a.offsets, a.batch, run.begin));

  // Rows lo .. hi - 1 out of the R of stage s, all of them (ALL) or some; `last`: no others of the stage follow.
  auto work = [&](auto all_rows, int64_t s, int64_t lo, int64_t hi, bool last) {
    constexpr bool ALL = decltype(all_rows)::value;
    const int64_t row0 = run.begin + s * R;
    const S in = slot(s);
    auto live = [&](int r) { return ALL || (row0 + r >= lo && row0 + r < hi); };
    F8 y[R][C], x[R][C], dh[R][C];
    float4 st[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if constexpr (!ALL) {  // rows of zeros add nothing to any sum
        st[r] = make_float4(0.f, 1.f, 0.f, 1.f);
#pragma unroll
        for (int c = 0; c < C; ++c) y[r][c] = x[r][c] = all8(0.f);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) dh[r][c] = all8(0.f);
      if (!live(r)) continue;
      const int64_t row = row0 + r;
      if constexpr (RING) {
        st[r] = in.stats()[r];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          y[r][c] = staged8(in.y() + r * a.dim, col[c], a.dim);
          x[r][c] = staged8(in.x() + r * a.dim, col[c], a.dim);
          if (a.d_h != nullptr) dh[r][c] = staged8(in.d_h() + r * a.dim, col[c], a.dim);
        }
      } else {
        st[r] = __ldg(a.stats + row);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          y[r][c] = load8<TY, false>(static_cast<const TY*>(a.y) + row * a.y_stride, col[c], a.dim);
          x[r][c] = load8<TX, false>(static_cast<const TX*>(a.residual) + row * a.residual_stride, col[c], a.dim);
          if (a.d_h != nullptr)
            dh[r][c] = load8<TY, false>(static_cast<const TY*>(a.d_h) + row * a.d_h_stride, col[c], a.dim);
        }
      }
    }
    float v[N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 sa = pair(0.f), san = pair(0.f);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const F8 w_pre = join(pre_weight[c][0][in_group * 32 + lane], pre_weight[c][1][in_group * 32 + lane]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 n1 = mul(add(y[r][c].p[k], pair(-st[r].x)), pair(st[r].y));
          const float2 xo = fma(n1, scale[c].p[k], fma(pair(a.alpha), x[r][c].p[k], shift[c].p[k]));
          const float2 n2 = mul(add(xo, pair(-st[r].z)), pair(st[r].w));
          const float2 d = dh[r][c].p[k], aw = mul(d, w_pre.p[k]);  // zero outside the row: dh is
          s_bpre[c].p[k] = add(s_bpre[c].p[k], d);
          s_wpre[c].p[k] = fma(d, n2, s_wpre[c].p[k]);
          sa = add(sa, aw);
          san = fma(aw, n2, san);
          y[r][c].p[k] = n1;
          x[r][c].p[k] = n2;
          dh[r][c].p[k] = aw;
        }
      }
      v[2 * r] = sa.x + sa.y;
      v[2 * r + 1] = san.x + san.y;
    }
    sum(v);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float2 minus_a = pair(a.layer ? -v[2 * r] * inv_dim : 0.f), minus_an = pair(-v[2 * r + 1] * inv_dim);
      const int64_t row = row0 + r;
      float2 sc = pair(0.f), scn = pair(0.f);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        // Taken as late as this: its registers are needed until here.
        F8 dx = all8(0.f), out;
        if (live(r) && a.d_residual_out != nullptr) {
          if constexpr (RING)
            dx = staged8(in.d_x() + r * a.dim, col[c], a.dim);
          else
            dx = load8<TX, false>(static_cast<const TX*>(a.d_residual_out) + row * a.d_residual_out_stride, col[c], a.dim);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 n1 = y[r][c].p[k];
          const float2 t = fma(x[r][c].p[k], minus_an, add(dh[r][c].p[k], minus_a));
          const float2 grad = fma(pair(st[r].w), t, dx.p[k]);
          s_one[c].p[k] = add(s_one[c].p[k], grad);
          s_n1[c].p[k] = fma(grad, n1, s_n1[c].p[k]);
          const float2 cw = mul(grad, scale[c].p[k]);
          sc = add(sc, cw);  // used with a norm after the block only: its weight is zero outside the row
          scn = fma(cw, n1, scn);
          out.p[k] = mul(pair(a.alpha), grad);
          dh[r][c].p[k] = cw;
        }
        if (live(r)) store8<TX, RING>(static_cast<TX*>(a.d_residual) + row * a.dim, col[c], a.dim, out);
      }
      v[2 * r] = sc.x + sc.y;
      v[2 * r + 1] = scn.x + scn.y;
    }
    // Past this barrier every warp of the group has taken the stage's rows.
    if (post)
      sum(v);
    else if constexpr (RING && MULTI)
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(w * 32) : "memory");
    if constexpr (RING) {
      if (last) {
        if constexpr (!MULTI) __syncwarp();
        if (filler && s + ring < stages) fill(s + ring);
      }
    }
    if (post) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float2 minus_c = pair(a.layer ? -v[2 * r] * inv_dim : 0.f), minus_cn = pair(-v[2 * r + 1] * inv_dim);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            dh[r][c].p[k] = mul(pair(st[r].y), fma(y[r][c].p[k], minus_cn, add(dh[r][c].p[k], minus_c)));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (live(r)) store8<TY, RING>(static_cast<TY*>(a.d_y) + (row0 + r) * a.dim, col[c], a.dim, dh[r][c]);
  };

  for (int64_t s = 0; s < stages; ++s) {
    const int64_t row0 = run.begin + s * R;
    const int64_t stop = run.end < row0 + R ? run.end : row0 + R;
    if constexpr (RING) {
      // After a wait that ran out the rows are worked on as they are: the call
      // has failed, and leaving would strand the group's other warps.
      if (!ptx::mbar_wait(&full[group][s % ring], static_cast<uint32_t>(s / ring) & 1u, &dead, kWaitNs)) {
        dead = 1;
        report(a.status, MPM_ERR_DEVICE_TIMEOUT, 31);
      }
    }
    for (int64_t lo = row0; lo < stop;) {  // rows under one gate at a time
      if (lo >= image_end && image < a.batch - 1) {
        close_image();
        int b = image + 1;
        while (b < a.batch - 1 && lo >= __ldg(a.offsets + b + 1)) ++b;
        open_image(b);
      }
      const int64_t hi = image_end < stop && image < a.batch - 1 ? image_end : stop;
      if (hi - lo == R) work(std::true_type{}, s, lo, hi, true);
      else work(std::false_type{}, s, lo, hi, hi == stop);
      lo = hi;
    }
  }
  if (!per_image) close_gate(a.gate);
  else if (run.begin < run.end) close_image();

  // Column sums of the block's groups, joined in the groups' order.
  float* joined = reinterpret_cast<float*>(dynamic);
  auto leave = [&](F8(&sums)[C], int which) {
    float* out = parts.sums + (static_cast<int64_t>(which) * gridDim.x + blockIdx.x) * a.dim;
    for (int k = 0; k < groups; ++k) {
      if (groups > 1) __syncthreads();
      if (group != k) continue;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        // Each column belongs to the same lane and warp of every group.
        if (k > 0) {
          const F8 before = load8_shared<RING>(joined, col[c], a.dim);
#pragma unroll
          for (int i = 0; i < 4; ++i) sums[c].p[i] = add(sums[c].p[i], before.p[i]);
        }
        if (k == groups - 1) store8<float, RING>(out, col[c], a.dim, sums[c]);
        else store8_shared<RING>(joined, col[c], a.dim, sums[c]);
      }
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

int groups_of(int dim) { return block_warps(chunks_per_thread(dim)) / warps_per_row(dim); }

template <typename TY, typename TX, int C, bool RING, bool MULTI>
cudaError_t launch_instance(const NormBackward& a, int num_sms, cudaStream_t stream) {
  const auto kernel = block_norm_backward_kernel<TY, TX, C, RING, MULTI>;
  const int w = warps_per_row(a.dim), groups = groups_of(a.dim);
  const int stage = Stage<TY, TX, rows_at_once(C)>::bytes(a.dim);
  int ring = RING ? ring_bytes(C) / (groups * stage) : 0;
  if (ring > kMaxRing) ring = kMaxRing;
  const size_t rings = static_cast<size_t>(groups) * ring * stage, joined = groups > 1 ? sizeof(float) * a.dim : 0;
  static std::atomic<uint64_t> attr_done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(attr_done.load() & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(C));
    if (e != cudaSuccess) return e;
    attr_done.fetch_or(bit);
  }
  const int64_t want = a.rows > 0 ? (a.rows + groups - 1) / groups : 1;  // without rows the sums are still written
  const int most = num_sms < kMaxBlocks ? num_sms : kMaxBlocks;
  const int grid = static_cast<int>(want < most ? want : most);
  e = launch_dependent(kernel, dim3(grid), dim3(groups * w * 32), rings > joined ? rings : joined, stream, a, w, ring);
  if (e != cudaSuccess) return e;
  const bool per_image = a.gate != nullptr && a.gate_per_image && a.d_gate != nullptr;
  if (a.d_gate == nullptr && a.d_pre_weight == nullptr && a.d_pre_bias == nullptr && a.d_post_weight == nullptr &&
      a.d_post_bias == nullptr)
    return cudaSuccess;
  const int threads = kJoinCols * kJoinRows;
  const int64_t joins = static_cast<int64_t>(kSums) * ((a.dim + kJoinCols - 1) / kJoinCols) +
                        (per_image ? static_cast<int64_t>(a.batch) * ((a.dim + threads - 1) / threads) : 0);
  return launch_dependent(block_norm_join_kernel, dim3(static_cast<unsigned>(joins)), dim3(threads), 0, stream, a, grid,
                          groups);
}

template <typename TY, typename TX, bool RING>
cudaError_t launch_types(const NormBackward& a, int num_sms, cudaStream_t stream) {
  if (warps_per_row(a.dim) == 1) return launch_instance<TY, TX, 1, RING, false>(a, num_sms, stream);
  switch (chunks_per_thread(a.dim)) {
    case 1: return launch_instance<TY, TX, 1, RING, true>(a, num_sms, stream);
    case 2: return launch_instance<TY, TX, 2, RING, true>(a, num_sms, stream);
    default: return launch_instance<TY, TX, 4, RING, true>(a, num_sms, stream);
  }
}

template <typename TY, typename TX>
cudaError_t launch_vec(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  // Rows too long for a stage of the ring (fp32 from about 13,000 features) are loaded in place.
  const int rows = rows_at_once(chunks_per_thread(a.dim));
  const int stage = rows == 2 ? Stage<TY, TX, 2>::bytes(a.dim) : Stage<TY, TX, 1>::bytes(a.dim);
  const bool ring = vec && groups_of(a.dim) * stage <= ring_bytes(chunks_per_thread(a.dim));
  return ring ? launch_types<TY, TX, true>(a, num_sms, stream) : launch_types<TY, TX, false>(a, num_sms, stream);
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
