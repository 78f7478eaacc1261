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
// Bound: HBM (y, x, dx' and dh in, dy and dx out).  A group of warps, one where
// the row has up to 768 features, works on a run of neighbouring rows, with
// four column sums in registers; they leave them once, at the end of the run
// (or of an image, for its gate).  Column sums are joined in fixed order,
// first over the groups of a block in shared memory, then over blocks by a
// second kernel: no atomics, the same bits every time.
//
// The sums take most registers, so few warps are there to hide latencies.
// Rows that are 16-byte aligned therefore come through a ring in shared
// memory that bulk copies fill rows ahead; and a thread has 8 to 24 columns of
// a row (32 of one with more than 6144 features), whose chains overlap, without
// barriers in between.  54208 x 768 bf16, layer norm on both sides and a gate
// per image (500 MB): 192 us from loads in place, 164 with rows spread over
// three warps (two barriers a row), 107 with a warp a row, 8 of them the join.
// Opening and closing the images' gates is 9 of them: a gate per channel takes
// 98, none 97.  A copy of as many bytes takes 77, and with half of the reads
// from L2 (dx' and dh the tensors of x and y) it is 83: what is left is neither
// memory's alone nor the instructions', of which two warps a scheduler issue
// 0.35 a cycle.  With an fp32 stream, 1.5 times the bytes for the same work, the
// pass runs at 5.3 TB/s.
//
// Two files per pair of token types include this one, with and without a norm
// before the next block: the kernels of all take minutes to compile.
#pragma once

#include <atomic>

#include "block_launch.h"
#include "norm_rows.cuh"
#include "ptx.cuh"
#include "row_ring.cuh"

namespace mpm {
namespace {

using namespace norm;

constexpr int kMaxBlocks = 160;  // blocks of the row kernel: one per SM
constexpr int kSums = 5;         // column sums: w_pre, b_pre, w_post, b_post, gate per channel
constexpr int kMaxRing = 4;      // rows in a group's ring
constexpr uint64_t kWaitNs = 2000000000ull;

// Chunks of 256 columns that a warp holds (8 C columns a thread): a row's only
// one; three where they divide its chunks, or else two, the last warp of a row of
// an odd number half empty; four in rows of more than 24, which have to fit
// the block's warps.  Their sums and row take about 30 + 56 C registers, which
// sets the warps: 8 of 255 registers for three and four, 12 of 168, 16 of 128
// (rows of more than 8192 features need 16 for four chunks each, and spill).
__host__ __device__ constexpr int chunks_per_warp(int dim) {
  const int chunks = (dim + kNormWarpCols - 1) / kNormWarpCols;
  return chunks == 1 ? 1 : chunks > 24 ? 4 : chunks % 3 == 0 ? 3 : 2;
}
__host__ __device__ constexpr int block_warps(int dim) {
  const int c = chunks_per_warp(dim);
  return c == 3 ? 8 : c == 2 ? 12 : c == 1 || dim > 32 * kNormWarpCols ? 16 : 8;
}
__host__ __device__ constexpr int warps_per_row(int dim) {
  return (dim + kNormWarpCols * chunks_per_warp(dim) - 1) / (kNormWarpCols * chunks_per_warp(dim));
}
// Most groups of a block (a ring of long rows may leave room for fewer).
__host__ __device__ constexpr int max_groups(int dim) { return block_warps(dim) / warps_per_row(dim); }
// Shared memory of a block for the groups: 227 KB less 2 KB of barriers and sums.
constexpr int kSharedBytes = 225 * 1024;

// The run of rows of group g out of `all`, sizes one apart at most.
struct Run {
  int64_t begin, end;
};
// (32-bit quotients: rows are at most 2^31 - 1, and 64-bit ones are long subroutines.)
__device__ __forceinline__ Run run_of(int64_t g, int64_t all, int64_t total) {
  const uint32_t per = static_cast<uint32_t>(total) / static_cast<uint32_t>(all);
  const int64_t extra = total - static_cast<int64_t>(per) * all;
  const int64_t begin = g * per + (g < extra ? g : extra);
  return {begin, begin + per + (g < extra ? 1 : 0)};
}
__device__ __forceinline__ int64_t group_of(int64_t row, int64_t all, int64_t total) {
  const uint32_t per = static_cast<uint32_t>(total) / static_cast<uint32_t>(all);
  const int64_t extra = total - static_cast<int64_t>(per) * all, long_rows = extra * (per + 1);
  return row < long_rows ? static_cast<uint32_t>(row) / (per + 1)
                         : extra + static_cast<uint32_t>(row - long_rows) / per;
}

// Workspace: column sums [kSums][blocks][dim], then for each group the gate's
// parts of the images that its run shares with an earlier one (head) or a
// later one (tail), and the sums for w_post and b_post over the gates closed so far.
struct Parts {
  float* sums;
  float* head;
  float* tail;
  float* w_post;
  float* b_post;
};
__device__ __forceinline__ Parts parts_of(const NormBackward& a, int blocks, int64_t all) {
  float* sums = a.partial;
  float* head = sums + static_cast<int64_t>(kSums) * blocks * a.dim;
  return {sums, head, head + all * a.dim, head + 2 * all * a.dim, head + 3 * all * a.dim};
}

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   ptx::smem_addr(dst)),
               "l"(src), "r"(bytes), "r"(ptx::smem_addr(bar))
               : "memory");
}

// A row in a group's ring: y, dh, x and dx' one after another, each as wide as
// the warps' chunks, and the statistics.  What no copy fills (columns past the
// row, a gradient that is absent) is zero from the start, so that it can be
// read like the rest.
template <typename TY, typename TX>
struct Slot {
  static constexpr int kValueBytes = 2 * sizeof(TY) + 2 * sizeof(TX);
  __host__ __device__ static constexpr int bytes(int dim) { return width(dim) * kValueBytes + 16; }
  __host__ __device__ static constexpr int width(int dim) {
    return warps_per_row(dim) * chunks_per_warp(dim) * kNormWarpCols;
  }
  uint8_t* base;
  int wide;
  __device__ __forceinline__ TY* y() const { return reinterpret_cast<TY*>(base); }
  __device__ __forceinline__ TY* d_h() const { return y() + wide; }
  __device__ __forceinline__ TX* x() const { return reinterpret_cast<TX*>(d_h() + wide); }
  __device__ __forceinline__ TX* d_x() const { return x() + wide; }
  __device__ __forceinline__ float4* stats() const { return reinterpret_cast<float4*>(d_x() + wide); }
};

// Eight columns of a row in the ring.
template <typename T>
__device__ __forceinline__ F8 staged8(const T* row, int col) {
  if constexpr (sizeof(T) == 2) {
    return widen(*reinterpret_cast<const uint4*>(row + col));
  } else {
    const float4* p = reinterpret_cast<const float4*>(row + col);
    return join(p[0], p[1]);
  }
}

// Bytes of a SharedVector.
__host__ __device__ constexpr int vector_bytes(int dim) {
  return warps_per_row(dim) * chunks_per_warp(dim) * kNormWarpCols * static_cast<int>(sizeof(float));
}

// RING: 16-byte aligned rows through shared memory (vector accesses); otherwise loads of single elements.
// PRE: with a norm before the next block.  Without it G = dx': neither x nor x' has a
// part in the gradients, and where they are not finite the gradients are all the same.
template <typename TY, typename TX, bool PRE, int C, bool RING, bool MULTI, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 1)
    block_norm_backward_kernel(NormBackward a, int row_warps, int slots, int room) {
  using Row = Slot<TY, TX>;
  // w_pre; A and B of each group; the groups' rings.  Afterwards the groups' column sums.
  extern __shared__ __align__(16) uint8_t dynamic[];
  __shared__ float2 sh[2 * WARPS];
  __shared__ uint64_t full[WARPS][kMaxRing];
  __shared__ int dead;          // a wait ran out: no further one is taken
  __shared__ int asked[WARPS];  // rows that the group asked for
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
  const int w = MULTI ? row_warps : 1;
  const int groups = (blockDim.x >> 5) / w, group = warp / w, in_group = warp % w;
  if (threadIdx.x == 0) {
    dead = 0;
    if constexpr (RING) {
      for (int k = 0; k < groups; ++k) {
        asked[k] = 0;
        for (int s = 0; s < slots; ++s) ptx::mbar_init(&full[k][s], 1);
      }
      ptx::fence_barrier_init();
    }
  }
  __syncthreads();
  wait_for_previous_grid();
  allow_next_grid();
  check_offsets(a.offsets, a.batch, a.rows, a.status);
  PairSum<MULTI> sum{sh + group * 2 * w, w, in_group, group + 1, 0};
  const int64_t total = used_rows(a.offsets, a.batch, a.rows);
  const int64_t all = static_cast<int64_t>(gridDim.x) * groups, g = static_cast<int64_t>(blockIdx.x) * groups + group;
  const Run run = run_of(g, all, total);
  const Parts parts = parts_of(a, gridDim.x, all);
  const float inv_dim = 1.f / static_cast<float>(a.dim);
  const bool post = a.post_weight != nullptr, per_image = a.gate != nullptr && a.gate_per_image;
  const int vector = vector_bytes(a.dim);
  const auto shared_vector = [&](int k) {
    return SharedVector{reinterpret_cast<float4*>(dynamic + k * vector), w * 32, in_group * 32 + lane};
  };
  const SharedVector pre_weight = shared_vector(0), scale = shared_vector(1 + 2 * group), shift = shared_vector(2 + 2 * group);

  const int wide = w * C * kNormWarpCols, slot_bytes = wide * Row::kValueBytes + 16;
  uint8_t* const ring_base = dynamic + (1 + 2 * groups) * vector + group * slots * slot_bytes;
  if constexpr (RING) {
    if (wide != a.dim || (PRE && a.d_h == nullptr) || a.d_residual_out == nullptr) {
      uint4* const rings = reinterpret_cast<uint4*>(dynamic + (1 + 2 * groups) * vector);
      for (int i = threadIdx.x; i < groups * slots * slot_bytes / 16; i += blockDim.x) rings[i] = make_uint4(0, 0, 0, 0);
      // Before the copies into the same slots.
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncthreads();
    }
  }
  auto fill = [&](int64_t row, int k) {  // by an elected lane of the group's first warp
    const Row to{ring_base + k * slot_bytes, wide};
    uint64_t* bar = &full[group][k];
    const uint32_t bytes_y = a.dim * static_cast<uint32_t>(sizeof(TY)), bytes_x = a.dim * static_cast<uint32_t>(sizeof(TX));
    ptx::mbar_arrive_expect_tx(bar, bytes_y + (PRE ? bytes_x : 0) + (PRE && a.d_h != nullptr ? bytes_y : 0) +
                                        (a.d_residual_out != nullptr ? bytes_x : 0) + 16);
    bulk_load(to.y(), static_cast<const TY*>(a.y) + row * a.y_stride, bytes_y, bar);
    if constexpr (PRE) bulk_load(to.x(), static_cast<const TX*>(a.residual) + row * a.residual_stride, bytes_x, bar);
    if (PRE && a.d_h != nullptr) bulk_load(to.d_h(), static_cast<const TY*>(a.d_h) + row * a.d_h_stride, bytes_y, bar);
    if (a.d_residual_out != nullptr)
      bulk_load(to.d_x(), static_cast<const TX*>(a.d_residual_out) + row * a.d_residual_out_stride, bytes_x, bar);
    bulk_load(to.stats(), a.stats + row, 16, bar);
  };
  if constexpr (RING) {
    if (in_group == 0 && ptx::elect_one()) {
#pragma unroll 1
      for (int k = 0; k < slots && run.begin + k < run.end; ++k) ring::refill(&dead, &asked[group], [&] { fill(run.begin + k, k); });
    }
  }

  int col[C];
  F8 s_wpre[C], s_bpre[C], s_one[C], s_n1[C];  // sums of dh n2, dh, G and G n1
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = first_column<RING>(c * w + in_group, lane);
    if (PRE && group == 0) pre_weight.set(c, param8<RING>(a.pre_weight, col[c], a.dim, 0.f));
    s_wpre[c] = s_bpre[c] = s_one[c] = s_n1[c] = all8(0.f);
  }
  __syncthreads();

  // Rows under one gate: between opening and closing it.
  auto open_gate = [&](const float* gate) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const F8 g8 = param8<RING>(gate, col[c], a.dim, 1.f);
      F8 w8 = param8<RING>(a.post_weight, col[c], a.dim, 1.f), b8 = param8<RING>(a.post_bias, col[c], a.dim, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w8.p[k] = mul(g8.p[k], w8.p[k]);
        b8.p[k] = mul(g8.p[k], b8.p[k]);
      }
      scale.set(c, w8);  // each thread reads back its own columns only
      shift.set(c, b8);
    }
  };
  // What the sums under a gate give: the gradients of w_post and b_post (times gate), and of the gate.
  auto gated = [&](const F8& gate, const F8& s) {
    F8 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.p[k] = mul(gate.p[k], s.p[k]);
    return r;
  };
  auto gate_gradient = [&](int c) {
    const F8 w8 = param8<RING>(a.post_weight, col[c], a.dim, 1.f), b8 = param8<RING>(a.post_bias, col[c], a.dim, 0.f);
    F8 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.p[k] = fma(w8.p[k], s_n1[c].p[k], mul(b8.p[k], s_one[c].p[k]));
    return r;
  };
  int image = 0;
  int64_t image_begin = 0, image_end = INT64_MAX;
  bool closed = false;
  auto gate_of = [&](int b) { return a.gate + static_cast<int64_t>(b) * a.dim; };
  auto open_image = [&](int b) {
    image = b;
    image_begin = __ldg(a.offsets + b);
    image_end = __ldg(a.offsets + b + 1);
    open_gate(gate_of(b));
  };
  // The gate's gradient over this run's rows of the image: all of its rows, or
  // a part.  The sums of w_post and b_post wait in the workspace, out of
  // registers; the run's last image leaves them in s_n1 and s_one.
  auto close_image = [&](bool at_end) {
    float* to = image_begin < run.begin ? parts.head + g * a.dim
                : image_end <= run.end  ? (a.d_gate == nullptr ? nullptr : a.d_gate + static_cast<int64_t>(image) * a.dim)
                                        : parts.tail + g * a.dim;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (to != nullptr) store8<float, RING>(to, col[c], a.dim, gate_gradient(c));
      const F8 g8 = param8<RING>(gate_of(image), col[c], a.dim, 0.f);
      F8 w8 = gated(g8, s_n1[c]), b8 = gated(g8, s_one[c]);
      if (closed) {
        const F8 w0 = load8<float, RING>(parts.w_post + g * a.dim, col[c], a.dim);
        const F8 b0 = load8<float, RING>(parts.b_post + g * a.dim, col[c], a.dim);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w8.p[k] = add(w8.p[k], w0.p[k]);
          b8.p[k] = add(b8.p[k], b0.p[k]);
        }
      }
      if (at_end) {
        s_n1[c] = w8;
        s_one[c] = b8;
        continue;
      }
      store8<float, RING>(parts.w_post + g * a.dim, col[c], a.dim, w8);
      store8<float, RING>(parts.b_post + g * a.dim, col[c], a.dim, b8);
      s_n1[c] = s_one[c] = all8(0.f);
    }
    closed = true;
  };
  if (!per_image) open_gate(a.gate);
  else if (run.begin < run.end) open_image(find_image(a.offsets, a.batch, run.begin));

  int k_slot = 0;
  uint32_t phase = 0;
#pragma unroll 1
  for (int64_t row = run.begin; row < run.end; ++row) {
    if (row >= image_end && image < a.batch - 1) {
      close_image(false);
      int b = image + 1;
      while (b < a.batch - 1 && row >= __ldg(a.offsets + b + 1)) ++b;
      open_image(b);
    }
    const Row in{ring_base + k_slot * slot_bytes, wide};
    F8 y[C], x[C], dh[C];
    float4 st;
    if constexpr (RING) {
      // After a wait that ran out the rows are worked on as they are: the call
      // has failed, and leaving would strand the group's other warps.  No more
      // rows are asked for, and what is under way is waited for at the end.
      if (!ptx::mbar_wait(&full[group][k_slot], phase, &dead, kWaitNs)) {
        dead = 1;
        report(a.status, MPM_ERR_DEVICE_TIMEOUT, 31);
      }
      st = *in.stats();
    } else {
      st = __ldg(a.stats + row);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (RING) {
        y[c] = staged8(in.y(), col[c]);
        if constexpr (PRE) {
          x[c] = staged8(in.x(), col[c]);
          dh[c] = staged8(in.d_h(), col[c]);
        }
      } else {
        y[c] = load8<TY, false>(static_cast<const TY*>(a.y) + row * a.y_stride, col[c], a.dim);
        if constexpr (!PRE) continue;
        x[c] = load8<TX, false>(static_cast<const TX*>(a.residual) + row * a.residual_stride, col[c], a.dim);
        dh[c] = a.d_h != nullptr ? load8<TY, false>(static_cast<const TY*>(a.d_h) + row * a.d_h_stride, col[c], a.dim)
                                 : all8(0.f);
      }
    }
    float v[2];
    if constexpr (!PRE) {
      const float2 minus_m1 = pair(-st.x), r1 = pair(st.y);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) y[c].p[k] = mul(add(y[c].p[k], minus_m1), r1);
    } else {
      float2 sa = pair(0.f), san = pair(0.f);
      const float2 minus_m1 = pair(-st.x), r1 = pair(st.y), minus_m2 = pair(-st.z), r2 = pair(st.w), alpha = pair(a.alpha);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const F8 w_pre = pre_weight.get(c), A = scale.get(c), B = shift.get(c);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 n1 = mul(add(y[c].p[k], minus_m1), r1);
          const float2 xo = fma(n1, A.p[k], fma(alpha, x[c].p[k], B.p[k]));
          const float2 n2 = mul(add(xo, minus_m2), r2);
          const float2 d = dh[c].p[k], aw = mul(d, w_pre.p[k]);  // zero outside the row: dh is
          s_bpre[c].p[k] = add(s_bpre[c].p[k], d);
          s_wpre[c].p[k] = fma(d, n2, s_wpre[c].p[k]);
          sa = add(sa, aw);
          san = fma(aw, n2, san);
          y[c].p[k] = n1;
          x[c].p[k] = n2;
          dh[c].p[k] = aw;
        }
      }
      v[0] = sa.x + sa.y;
      v[1] = san.x + san.y;
      sum(v);
    }
    {
      const float2 minus_a = pair(PRE && a.layer ? -v[0] * inv_dim : 0.f), minus_an = pair(PRE ? -v[1] * inv_dim : 0.f);
      const float2 r2 = pair(st.w), alpha = pair(a.alpha);
      float2 sc = pair(0.f), scn = pair(0.f);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        // Taken as late as this: its registers are needed until here.
        F8 dx, out;
        if constexpr (RING)
          dx = staged8(in.d_x(), col[c]);
        else
          dx = a.d_residual_out == nullptr
                   ? all8(0.f)
                   : load8<TX, false>(static_cast<const TX*>(a.d_residual_out) + row * a.d_residual_out_stride, col[c], a.dim);
        const F8 A = scale.get(c);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 n1 = y[c].p[k];
          float2 grad = dx.p[k];
          if constexpr (PRE) grad = fma(r2, fma(x[c].p[k], minus_an, add(dh[c].p[k], minus_a)), grad);
          s_one[c].p[k] = add(s_one[c].p[k], grad);
          s_n1[c].p[k] = fma(grad, n1, s_n1[c].p[k]);
          const float2 cw = mul(grad, A.p[k]);
          sc = add(sc, cw);  // used with a norm after the block only: its weight is zero outside the row
          scn = fma(cw, n1, scn);
          out.p[k] = mul(alpha, grad);
          dh[c].p[k] = cw;
        }
        store8<TX, RING>(static_cast<TX*>(a.d_residual) + row * a.dim, col[c], a.dim, out);
      }
      v[0] = sc.x + sc.y;
      v[1] = scn.x + scn.y;
    }
    // Past this every warp of the group has taken the slot's row.
    if (post)
      sum(v);
    else if constexpr (RING && MULTI)
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(w * 32) : "memory");
    if constexpr (RING) {
      __syncwarp();
      if (in_group == 0 && row + slots < run.end && ptx::elect_one())
        ring::refill(&dead, &asked[group], [&] { fill(row + slots, k_slot); });
      __syncwarp();
      if (++k_slot == slots) {
        k_slot = 0;
        phase ^= 1u;
      }
    }
    if (post) {
      const float2 minus_c = pair(a.layer ? -v[0] * inv_dim : 0.f), minus_cn = pair(-v[1] * inv_dim), r1 = pair(st.y);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          dh[c].p[k] = mul(r1, fma(y[c].p[k], minus_cn, add(dh[c].p[k], minus_c)));
    }
#pragma unroll
    for (int c = 0; c < C; ++c) store8<TY, RING>(static_cast<TY*>(a.d_y) + row * a.dim, col[c], a.dim, dh[c]);
  }
  if (per_image && run.begin < run.end) close_image(true);

  // Column sums of the block's groups, side by side in shared memory (where A
  // and B and the rings were), as many at a time as have room there, then added
  // in the groups' order.
  const int quads = vector / 16;
  float4* const side = reinterpret_cast<float4*>(dynamic);
  int kept = 0;
  uint32_t which_kept = 0;  // four bits each
  auto join_kept = [&]() {
    __syncthreads();
    for (int i = threadIdx.x; i < kept * quads; i += blockDim.x) {
      const int n = i / quads, q = i - n * quads;
      const float4* from = side + n * groups * quads + q;
      float4 s = from[0];
      for (int k = 1; k < groups; ++k) {
        const float4 t = from[k * quads];
        s = make_float4(s.x + t.x, s.y + t.y, s.z + t.z, s.w + t.w);
      }
      float* out = parts.sums + (static_cast<int64_t>((which_kept >> (4 * n)) & 15u) * gridDim.x + blockIdx.x) * a.dim;
      const int at = q % (w * 32), c = q / (w * 32) / 2, half = q / (w * 32) % 2;
      const int first = first_column<RING>(c * w + at / 32, at % 32);
      const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (column<RING>(first, 4 * half + j) < a.dim) out[column<RING>(first, 4 * half + j)] = v[j];
    }
    __syncthreads();
    kept = 0;
    which_kept = 0;
  };
  auto leave = [&](int which, auto value) {
    const SharedVector mine{side + (kept * groups + group) * quads, w * 32, in_group * 32 + lane};
#pragma unroll
    for (int c = 0; c < C; ++c) mine.set(c, value(c));
    which_kept |= static_cast<uint32_t>(which) << (4 * kept);
    // One at a time for groups of several warps: with more, the compiler's code
    // for the rows is slower (30000 x 1024 bf16, dx' and dh the tensors of x and y:
    // 76 us, 95 with two or five; 81 with four tensors).
    if (++kept == (MULTI ? 1 : room)) join_kept();
  };
  // Over the gates of a run: what its last image left, or the one gate's sums.
  auto over_gates = [&](const F8(&s)[C], int c) {
    return per_image ? s[c] : gated(param8<RING>(a.gate, col[c], a.dim, 1.f), s[c]);
  };
  __syncthreads();
  if constexpr (RING) {
    if (dead != 0) {
      if (in_group == 0 && lane == 0) ring::drain(full[group], slots, asked[group], kWaitNs);
      __syncthreads();
    }
  }
  if (PRE && a.d_pre_weight != nullptr) leave(0, [&](int c) { return s_wpre[c]; });
  if (PRE && a.d_pre_bias != nullptr) leave(1, [&](int c) { return s_bpre[c]; });
  if (a.d_gate != nullptr && !per_image) leave(4, [&](int c) { return gate_gradient(c); });
  if (a.d_post_weight != nullptr) leave(2, [&](int c) { return over_gates(s_n1, c); });
  if (a.d_post_bias != nullptr) leave(3, [&](int c) { return over_gates(s_one, c); });
  if (kept > 0) join_kept();
}

// Blocks of the join: columns x parts that are added at once, 32 x 16 for the
// parameters (a part a block) and for gates whose images are shared by many
// runs, 128 x 4 where they are shared by few.
constexpr int kJoinThreads = 512;
constexpr int kJoinCols = 32, kGateCols = 128;
constexpr int kManyRuns = 32;

// Adds parts first, first + 1, .. last (their column's addresses by `at`) and
// writes the sum: rows of threads take every ROWS-th, and are added in order.
template <int COLS, typename At>
__device__ __forceinline__ void join_parts(float* part, int64_t first, int64_t last, bool in, float* out, At at) {
  constexpr int ROWS = kJoinThreads / COLS;
  const int x = threadIdx.x % COLS, r = threadIdx.x / COLS;
  float s = 0.f;
  if (in) {
#pragma unroll 4
    for (int64_t g = first + r; g <= last; g += ROWS) s += *at(g);
  }
  part[r * COLS + x] = s;
  __syncthreads();
  if (r == 0 && in) {
    for (int i = 1; i < ROWS; ++i) s += part[i * COLS + x];
    *out = s;
  }
}

// Column sums over blocks, and the gates of images that several runs share.
__global__ void __launch_bounds__(kJoinThreads) block_norm_join_kernel(NormBackward a, int blocks, int groups, int gate_cols) {
  wait_for_previous_grid();
  allow_next_grid();
  __shared__ float part[kJoinThreads];
  __shared__ int64_t ends[2];  // first and last group of the image's rows
  const int64_t all = static_cast<int64_t>(blocks) * groups;
  const Parts parts = parts_of(a, blocks, all);
  const bool per_image = a.gate != nullptr && a.gate_per_image;
  float* const outs[kSums] = {a.d_pre_weight, a.d_pre_bias, a.d_post_weight, a.d_post_bias,
                              per_image ? nullptr : a.d_gate};
  const int col_blocks = (a.dim + kJoinCols - 1) / kJoinCols;
  const int which = blockIdx.x / col_blocks;
  if (which < kSums) {
    if (outs[which] == nullptr) return;
    const int col = blockIdx.x % col_blocks * kJoinCols + threadIdx.x % kJoinCols;
    const float* in = parts.sums + static_cast<int64_t>(which) * blocks * a.dim + col;
    join_parts<kJoinCols>(part, 0, blocks - 1, col < a.dim, outs[which] + col,
                          [&](int64_t b) { return in + b * a.dim; });
    return;
  }
  const int gate_blocks = (a.dim + gate_cols - 1) / gate_cols, k = blockIdx.x - kSums * col_blocks;
  const int image = k / gate_blocks, col = k % gate_blocks * gate_cols + threadIdx.x % gate_cols;
  if (image >= a.batch || a.d_gate == nullptr) return;
  if (threadIdx.x == 0) {
    const int64_t total = used_rows(a.offsets, a.batch, a.rows);
    int64_t lo = __ldg(a.offsets + image), hi = __ldg(a.offsets + image + 1);
    lo = lo < 0 ? 0 : lo;
    hi = hi < total ? hi : total;
    ends[0] = hi > lo ? group_of(lo, all, total) : 0;
    ends[1] = hi > lo ? group_of(hi - 1, all, total) : -1;
  }
  __syncthreads();
  const int64_t first = ends[0], last = ends[1];
  if (last >= 0 && first == last) return;  // written by its run
  // Without rows (last < first) the sum is zero.
  float* out = a.d_gate + static_cast<int64_t>(image) * a.dim + col;
  auto at = [&](int64_t g) { return (g == first ? parts.tail : parts.head) + g * a.dim + col; };
  if (gate_cols == kGateCols) join_parts<kGateCols>(part, first, last, col < a.dim, out, at);
  else join_parts<kJoinCols>(part, first, last, col < a.dim, out, at);
}

// Groups of a block and rows of each one's ring: as many groups as warps allow
// two rows each, and up to kMaxRing rows.  No groups: the rows are too long for it.
struct RingPlan {
  int groups, rows;
};
RingPlan plan_ring(int dim, int row_bytes) {
  const int vector = vector_bytes(dim);
  for (int depth = 2; depth > 0; --depth) {
    int groups = (kSharedBytes - vector) / (depth * row_bytes + 2 * vector);
    if (groups > max_groups(dim)) groups = max_groups(dim);
    if (groups > 0) {
      const int rows = ((kSharedBytes - vector) / groups - 2 * vector) / row_bytes;
      return {groups, rows < kMaxRing ? rows : kMaxRing};
    }
  }
  return {0, 0};
}

template <typename TY, typename TX, bool PRE, int C, bool RING, bool MULTI, int WARPS>
cudaError_t launch_instance(const NormBackward& a, RingPlan ring, int num_sms, cudaStream_t stream) {
  const auto kernel = block_norm_backward_kernel<TY, TX, PRE, C, RING, MULTI, WARPS>;
  const int w = warps_per_row(a.dim), vector = vector_bytes(a.dim);
  int groups = ring.groups;
  if (!RING) {
    groups = (kSharedBytes - vector) / (2 * vector);
    if (groups > max_groups(a.dim)) groups = max_groups(a.dim);
  }
  const size_t smem = vector + groups * (2 * static_cast<size_t>(vector) + (RING ? ring.rows * Slot<TY, TX>::bytes(a.dim) : 0));
  static std::atomic<uint64_t> attr_done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(attr_done.load() & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
    if (e != cudaSuccess) return e;
    attr_done.fetch_or(bit);
  }
  const int64_t want = a.rows > 0 ? (a.rows + groups - 1) / groups : 1;  // without rows the sums are still written
  const int most = num_sms < kMaxBlocks ? num_sms : kMaxBlocks;
  const int grid = static_cast<int>(want < most ? want : most);
  const int room = static_cast<int>(smem / (static_cast<size_t>(groups) * vector));  // sums side by side at the end: two at least
  e = launch_dependent(kernel, dim3(grid), dim3(groups * w * 32), smem, stream, a, w, ring.rows,
                       room < kSums ? room : kSums);
  if (e != cudaSuccess) return e;
  const bool per_image = a.gate != nullptr && a.gate_per_image && a.d_gate != nullptr;
  if (a.d_gate == nullptr && a.d_pre_weight == nullptr && a.d_pre_bias == nullptr && a.d_post_weight == nullptr &&
      a.d_post_bias == nullptr)
    return cudaSuccess;
  const int gate_cols = static_cast<int64_t>(grid) * groups > static_cast<int64_t>(kManyRuns) * a.batch ? kJoinCols : kGateCols;
  const int64_t joins = static_cast<int64_t>(kSums) * ((a.dim + kJoinCols - 1) / kJoinCols) +
                        (per_image ? static_cast<int64_t>(a.batch) * ((a.dim + gate_cols - 1) / gate_cols) : 0);
  return launch_dependent(block_norm_join_kernel, dim3(static_cast<unsigned>(joins)), dim3(kJoinThreads), 0, stream, a, grid,
                          groups, gate_cols);
}

template <typename TY, typename TX, bool PRE, bool RING>
cudaError_t launch_types(const NormBackward& a, RingPlan ring, int num_sms, cudaStream_t stream) {
  const bool multi = warps_per_row(a.dim) > 1;
  switch (chunks_per_warp(a.dim)) {
    case 1: return launch_instance<TY, TX, PRE, 1, RING, false, 16>(a, ring, num_sms, stream);
    case 2: return multi ? launch_instance<TY, TX, PRE, 2, RING, true, 12>(a, ring, num_sms, stream)
                         : launch_instance<TY, TX, PRE, 2, RING, false, 12>(a, ring, num_sms, stream);
    case 3: return multi ? launch_instance<TY, TX, PRE, 3, RING, true, 8>(a, ring, num_sms, stream)
                         : launch_instance<TY, TX, PRE, 3, RING, false, 8>(a, ring, num_sms, stream);
    default: return block_warps(a.dim) == 8 ? launch_instance<TY, TX, PRE, 4, RING, true, 8>(a, ring, num_sms, stream)
                                            : launch_instance<TY, TX, PRE, 4, RING, true, 16>(a, ring, num_sms, stream);
  }
}

template <typename TY, typename TX, bool PRE>
cudaError_t launch_vec(const NormBackward& a, bool vec, int num_sms, cudaStream_t stream) {
  const RingPlan ring = vec ? plan_ring(a.dim, Slot<TY, TX>::bytes(a.dim)) : RingPlan{0, 0};
  return ring.groups > 0 ? launch_types<TY, TX, PRE, true>(a, ring, num_sms, stream)
                         : launch_types<TY, TX, PRE, false>(a, ring, num_sms, stream);
}

}  // namespace
}  // namespace mpm
