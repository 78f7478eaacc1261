// What the tensor-core attention kernels share: tiles of 128 rows by TMA, products
// whose left operand lies in tensor memory, and the tables and waits of their roles.
//
// A tile is 128 rows of one head: per 64 features a block of 128 x 128 bytes in
// the 128-byte swizzle.  The same bytes serve as an operand with the features
// along K (scores: rows x rows) and, with the rows along K, as the right operand
// of a product over rows (p v, ds k, ..): then the features are the contiguous
// dimension, in blocks of 64 that lie a block apart, and eight rows of 128 bytes
// are a group along K.  Features past the head's width read as zeros.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>

#include "attention_common.cuh"
#include "ptx.cuh"

namespace mpm {
namespace attn {

constexpr int kRows = 128;                  // rows of a tile
constexpr int kBlockBytes = kRows * 128;    // 64 features of a tile
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int64_t kMaxBlocks = INT32_MAX;

// Tokens as (feature, head, row); boxes of 64 features of one head of 128 rows.
inline PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return static_cast<PFN_cuTensorMapEncodeTiled_v12000>(nullptr);
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}
inline bool map_heads(CUtensorMap* map, const Heads& x, int64_t rows, int heads, int dim) {
  if (tensor_map_encoder() == nullptr) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
  // A stride that nothing goes by still has to be a multiple of 16 bytes.
  const int64_t head = heads > 1 ? x.head : (dim + 7) / 8 * 8, row = rows > 1 ? x.row : heads * head;
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(head) * 2, static_cast<cuuint64_t>(row) * 2};
  const cuuint32_t box[3] = {64, 1, kRows}, each[3] = {1, 1, 1};
  return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x.p), dims, strides, box, each,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

__device__ __forceinline__ void load_block(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int32_t x, int32_t head,
                                           int32_t row) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(ptx::smem_addr(bar)), "r"(x), "r"(head), "r"(row)
      : "memory");
}
// A tile of H blocks, counted on `bar`.
template <int H>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int32_t head, int32_t row) {
#pragma unroll
  for (int h = 0; h < H; ++h) load_block(dst + h * kBlockBytes, map, bar, 64 * h, head, row);
}

// Instruction descriptors of kind::f16: bf16 operands, fp32 sums, M = 128.
__host__ __device__ constexpr uint32_t by_features(uint32_t n) { return ptx::idesc_bf16_f32(kRows, n); }
__host__ __device__ constexpr uint32_t by_rows(uint32_t n) { return ptx::idesc_bf16_f32(kRows, n) | (1u << 16); }  // B is N-major

// Descriptor of a tile as the right operand with its rows along K: feature blocks
// kBlockBytes apart (leading offset), groups of eight rows 1024 bytes apart (stride
// offset), 128-byte swizzle.
__device__ __forceinline__ uint64_t desc_by_rows(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(kBlockBytes >> 4) << 16) |
         (static_cast<uint64_t>(1024u >> 4) << 32) | (static_cast<uint64_t>(1u) << 46) | (static_cast<uint64_t>(2u) << 61);
}

// D (+)= A B for one K = 16 slice with A in tensor memory.
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Products are issued four at a time: written one by one, what forms their operands
// took 50 cycles a product, and the issuing warp bounded the kernels (64 x 1024
// tokens, 12 heads of 64, forward: 233 us, 227 so).
// D [128, 128] (+)= four K = 16 slices of 64 features of both tiles.
__device__ __forceinline__ void mma_features4(uint32_t d, uint64_t a, uint64_t b, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, q;\n\t"
      "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, q;\n\t"
      "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, q;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(by_features(kRows)), "r"(accumulate), "r"(1u)
      : "memory");
}
// D [128, width] (+)= 64 columns of weights (bf16 pairs in 32 columns of tensor memory) times 64 rows of b.
__device__ __forceinline__ void mma_rows4(uint32_t d, uint32_t weights, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "add.u32 a, %1, 8;\n\tadd.s64 b, %2, 128;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, q;\n\t"
      "add.u32 a, %1, 16;\n\tadd.s64 b, %2, 256;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, q;\n\t"
      "add.u32 a, %1, 24;\n\tadd.s64 b, %2, 384;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, q;\n\t}" ::"r"(d),
      "r"(weights), "l"(b), "r"(idesc), "r"(accumulate), "r"(1u)
      : "memory");
}
// Scores of two tiles, [128 rows of a, 128 rows of b]: a sum over the features, `slices` times 16.
template <int H>
__device__ __forceinline__ void mma_scores(uint32_t d, uint32_t a, uint32_t b, int slices) {
  const uint64_t da = ptx::sdesc_k_sw128(a), db = ptx::sdesc_k_sw128(b);
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const uint64_t at = static_cast<uint64_t>(h * (kBlockBytes >> 4));
    if (slices >= 4 * h + 4) {
      mma_features4(d, da + at, db + at, h != 0 ? 1u : 0u);
    } else {
      for (int s = 4 * h; s < slices; ++s)
        ptx::mma_bf16(d, da + at + (s % 4) * 2, db + at + (s % 4) * 2, by_features(kRows), s != 0 ? 1u : 0u);
    }
  }
}
// d [128, width] (+)= weights [128, 128 rows of b] times b; `apart`: columns between the weights of rows 0 and 64.
__device__ __forceinline__ void mma_weighted(uint32_t d, uint32_t weights, uint32_t apart, uint32_t b, uint32_t idesc, bool accumulate) {
  const uint64_t db = desc_by_rows(b);
  mma_rows4(d, weights, db, idesc, accumulate ? 1u : 0u);
  mma_rows4(d, weights + apart, db + 512, idesc, 1u);
}

// 32 lanes x 32 consecutive columns: thread t writes lane t.
__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
      "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]),
      "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// How a block's roles give up.  A role may wait for as long as a work item takes,
// and that is as long as its sequence: 20 us are allowed for each of its tiles, ten
// times what they take.  So are places of sequences without rows, passed at some us each.
struct Bounds {
  volatile int failed;  // a wait ran out somewhere
  uint32_t limit_us;
  __device__ __forceinline__ void init(const AttentionArgs& a) {
    const uint64_t rows = static_cast<uint64_t>(a.q_rows) * (a.q_heads / a.kv_heads) + static_cast<uint64_t>(a.k_rows);
    const uint64_t empty = static_cast<uint64_t>(a.batch) * a.q_heads * (a.splits > a.key_splits ? a.splits : a.key_splits);
    const uint64_t us = kWaitNs / 1000 + rows / kRows * 20 + empty / 16;
    failed = 0;
    limit_us = us < 0xFFFFFFFFu ? static_cast<uint32_t>(us) : 0xFFFFFFFFu;
  }
};
// Bounded wait of a whole warp: one answer for all of its lanes.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, Bounds* bounds) {
  bool done = ptx::mbar_try_wait(bar, parity);
  if (!done) done = ptx::mbar_wait(bar, parity, &bounds->failed, static_cast<uint64_t>(bounds->limit_us) * 1000);
  return __all_sync(0xFFFFFFFFu, done);
}
// The wait for copies under way, at a block's end.
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity) { ptx::mbar_wait(bar, parity, nullptr, kWaitNs); }

// A value that all lanes hold, in a form that the compiler knows to be uniform: what
// the products' issuing warp computes with (see ptx::elect_one).
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }
// Arrives on the barrier at a shared address when all products issued so far have completed.
__device__ __forceinline__ void commit_at(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Work items are the grid's blocks: a block that runs takes the places of blocks that
// have not started yet, one after another, so that SMs whose items were short do more
// of them.  An item's result does not depend on who does it.
struct Claims {
  uint4 answer[2];
  uint64_t bar[2];
};
// By one warp, converged.
struct ClaimedItems {
  Claims* claims;
  int64_t item, items;
  uint32_t asked = 0, answered = 0;
  bool more;
  __device__ __forceinline__ ClaimedItems(Claims* c, int64_t n) : claims(c), item(blockIdx.x), items(n), more(item < n) {}
  // Asks for the block after this item's; the answer is read by next().
  __device__ __forceinline__ void ask() {
    if (asked != answered) return;
    const uint32_t i = asked++ & 1u;
    if ((threadIdx.x & 31) == 0) {
      // The answer's last value has been read.
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      ptx::mbar_arrive_expect_tx(&claims->bar[i], 16);
      asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                       ptx::smem_addr(&claims->answer[i])),
                   "r"(ptx::smem_addr(&claims->bar[i]))
                   : "memory");
    }
    __syncwarp();
  }
  // On to the next item, if there is one; false after a wait that ran out.
  __device__ __forceinline__ bool next(Bounds* bounds) {
    if (item + gridDim.x < items) {  // more items than a grid can have blocks
      item += gridDim.x;
      return true;
    }
    ask();
    if (!warp_wait(&claims->bar[answered & 1u], answered >> 1 & 1u, bounds)) return false;
    take();
    return true;
  }
  // Before the block leaves: an answer under way has come, and after a failure nobody starts on what is left.
  __device__ __forceinline__ void finish(Bounds* bounds) {
    while (asked != answered || (__any_sync(0xFFFFFFFFu, bounds->failed != 0) && more)) {
      ask();
      if (!__all_sync(0xFFFFFFFFu, ptx::mbar_wait(&claims->bar[answered & 1u], answered >> 1 & 1u, nullptr, kWaitNs))) return;
      take();
    }
  }

 private:
  __device__ __forceinline__ void take() {
    int32_t first;
    asm volatile(
        "{\n\t.reg .b128 a;\n\t.reg .pred p;\n\t.reg .b32 y, z, w;\n\t"
        "ld.shared.b128 a, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
        "mov.b32 %0, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, y, z, w}, a;\n\t}"
        : "=r"(first)
        : "r"(ptx::smem_addr(&claims->answer[answered & 1u]))
        : "memory");
    first = __shfl_sync(0xFFFFFFFFu, first, 0);
    ++answered;
    more = first >= 0;
    if (more) item = first;
  }
};

// Place in a ring of SLOTS.
template <int SLOTS>
struct RingPlace {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++slot == SLOTS) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// Which of the rows first .. first + 127 of a sequence are there: a bit each.
// By a whole converged warp; every lane gets all four words.
__device__ __forceinline__ uint4 rows_there(const Span& s, int first, const uint8_t* __restrict__ mask) {
  const int lane = threadIdx.x & 31;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = first + 32 * i + lane;
    w[i] = __ballot_sync(0xFFFFFFFFu, row < s.n && (mask == nullptr || __ldg(mask + s.lo + row) != 0));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Zeros the rows of a tile whose bit is not set, by a whole warp, for the tensor cores to read.
template <int H>
__device__ __forceinline__ void zero_rows(uint8_t* tile, const uint4& there) {
  const int lane = threadIdx.x & 31;
  const uint32_t w[4] = {there.x, there.y, there.z, there.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (w[i] == 0xFFFFFFFFu) continue;
    for (int r = lane / 8; r < 32; r += 4) {
      if (w[i] >> r & 1u) continue;
#pragma unroll
      for (int h = 0; h < H; ++h)
        *reinterpret_cast<uint4*>(tile + h * kBlockBytes + (32 * i + r) * 128 + lane % 8 * 16) = make_uint4(0, 0, 0, 0);
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}

// 32 features of a warp's 32 rows, a row a lane, times a factor a row, to global
// memory: as bf16, or what that rounding leaves (REST).  They change places in 2 KB
// of shared memory, so that a store's lanes write whole 64-byte runs of eight rows;
// lane by lane, 16 bytes of 32 rows at a time, the stores of 1024 rows of 80
// features took longer than all else.
constexpr int kStageBytes = 32 * 64;
template <bool REST>
__device__ __forceinline__ void store_rows32(__nv_bfloat16* first_row, int64_t pitch, int rows, int col, int dim, bool vec,
                                             uint8_t* stage, const uint32_t (&v)[32], float factor) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float x = __uint_as_float(v[8 * p + 2 * k]) * factor, y = __uint_as_float(v[8 * p + 2 * k + 1]) * factor;
      if constexpr (REST) {
        x = to_f32(rest_of<__nv_bfloat16>(x));
        y = to_f32(rest_of<__nv_bfloat16>(y));
      }
      u[k] = pack_bf16(x, y);
    }
    *reinterpret_cast<uint4*>(stage + lane * 64 + ((p ^ (lane >> 1 & 3)) * 16)) = make_uint4(u[0], u[1], u[2], u[3]);
  }
  __syncwarp();
  if (vec) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + lane / 4, p = lane & 3;
      if (row < rows && col + 8 * p < dim)
        *reinterpret_cast<uint4*>(first_row + row * pitch + col + 8 * p) =
            *reinterpret_cast<const uint4*>(stage + row * 64 + ((p ^ (row >> 1 & 3)) * 16));
    }
  } else {
    for (int row = 0; row < rows; ++row)
      if (col + lane < dim)
        first_row[row * pitch + col + lane] = *reinterpret_cast<const __nv_bfloat16*>(
            stage + row * 64 + (((lane / 8) ^ (row >> 1 & 3)) * 16) + lane % 8 * 2);
  }
  __syncwarp();
}
// 32 features of a warp's 32 rows to a part's fp32 rows, by the same way.
__device__ __forceinline__ void store_part32(float* first_row, int64_t pitch, int rows, int col, int dim, bool vec, uint8_t* stage,
                                             const uint32_t (&v)[32], float factor) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float4 u = make_float4(__uint_as_float(v[16 * h + 4 * p]) * factor, __uint_as_float(v[16 * h + 4 * p + 1]) * factor,
                                   __uint_as_float(v[16 * h + 4 * p + 2]) * factor, __uint_as_float(v[16 * h + 4 * p + 3]) * factor);
      *reinterpret_cast<float4*>(stage + lane * 64 + ((p ^ (lane >> 1 & 3)) * 16)) = u;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + lane / 4, p = lane & 3, c = col + 16 * h + 4 * p;
      if (row < rows && c < dim) {
        const float4 u = *reinterpret_cast<const float4*>(stage + row * 64 + ((p ^ (row >> 1 & 3)) * 16));
        float* to = first_row + row * pitch + c;
        if (vec) {
          *reinterpret_cast<float4*>(to) = u;
        } else {
          to[0] = u.x;
          if (c + 1 < dim) to[1] = u.y;
          if (c + 2 < dim) to[2] = u.z;
          if (c + 3 < dim) to[3] = u.w;
        }
      }
    }
    __syncwarp();
  }
}

}  // namespace attn
}  // namespace mpm
