// out[m, n] = sum_k A[m, k] B[n, k] + bias[n] for MXFP4 operands (mxfp4.cuh),
// accumulated in fp32 on the tensor cores: tcgen05.mma kind::mxf4 with a
// power-of-two scale per 32 elements.
//
// A cluster of two CTAs (an SM pair) computes 256 x 192 tiles with
// cta_group::2: each CTA stages its 128 rows of A, half of the tile's rows of
// B, the scales of its A rows and those of all of the tile's B rows.  A stage
// holds 256 elements of every row, one 128-byte swizzle row of packed codes,
// and takes four K = 64 products.  Scales go from shared memory to tensor
// memory by tcgen05.cp, into columns that belong to the stage: the products
// that read them have completed before the stage is filled again.
//
// Bound: with few features the output's bytes (2 M N of them against
// (M + N) K / 2: 256 x 192 tiles of K = 768 take the tensor cores a quarter of
// the time that their output takes HBM), with many the tensor cores.  Hence
// two accumulators (2 x 192 of the 512 tensor-memory columns, which leaves
// 128 for the scales of five stages): a tile's output is written while the
// next tile is computed.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>

#include "common.cuh"
#include "mxfp4.cuh"
#include "ptx.cuh"

namespace mpm {
namespace {

constexpr int kHalf = 128;             // rows of A per CTA
constexpr int kTileM = 2 * kHalf;
constexpr int kTileN = 192;
constexpr int kStageK = 256;           // elements of a row per stage: 128 bytes
constexpr int kBytesA = kHalf * 128;
constexpr int kBytesB = kTileN / 2 * 128;
constexpr int kScaleTiles = kStageK / (mx::kBlock * mx::kTileBlocks);      // scale tiles along K per stage
constexpr int kBytesSA = kScaleTiles * mx::kTileBytes;
constexpr int kBytesSB = 2 * kBytesSA;  // a tile's 192 rows of B lie in at most two row tiles
constexpr int kStageBytes = kBytesA + kBytesB + kBytesSA + kBytesSB;
constexpr int kStages = 5;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kScaleCols = 2 * kTileN;                 // first column of the scales
constexpr uint32_t kColsSA = 4, kColsSB = 8;                // columns of one scale tile of A, of two of B
constexpr uint32_t kStageCols = kScaleTiles * (kColsSA + kColsSB);
constexpr int kWarpCols = 64;                               // columns of the tile that an epilogue warp writes
constexpr int kEpilogueWarps = 4 * (kTileN / kWarpCols);
constexpr int kThreads = (2 + kEpilogueWarps) * 32;
constexpr int kBoxBytes = 32 * 128;                         // staged output: 32 rows of 128 bytes, swizzled
constexpr uint64_t kWaitNs = 2000000000ull;
static_assert(kScaleCols + kStages * kStageCols <= kTmemCols, "accumulators and scales share tensor memory");
static_assert(kStageBytes % 1024 == 0 && kBytesA % 1024 == 0 && kBytesB % 1024 == 0, "swizzled tiles on 1024 bytes");

// Instruction descriptor of kind::mxf4: E2M1 operands (1) in K-major order,
// scales of type UE8M0 (bit 23), N / 8 and M / 16 in their fields.
constexpr uint32_t kIdesc = (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kTileN >> 3) << 17) | (1u << 23) |
                            (static_cast<uint32_t>(kTileM >> 4) << 24);
// Which half of a 32-bit column's four scales a K = 64 product takes: fields of B and of A.
__device__ __forceinline__ constexpr uint32_t scale_half(uint32_t which) { return (which << 4) | (which << 29); }

struct Control {
  uint64_t full[kStages];   // leader: both CTAs' operands of the stage landed
  uint64_t empty[kStages];  // both: products reading the stage completed
  uint64_t acc_full[2];     // both: accumulator complete
  uint64_t acc_empty[2];    // leader: both CTAs read the accumulator
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
};

constexpr size_t kSmemBytes = 1024 + static_cast<size_t>(kStages) * kStageBytes + kEpilogueWarps * kBoxBytes + sizeof(Control);

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t saddr, uint32_t rank) {
  uint32_t out;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(saddr), "r"(rank));
  return out;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void remote_arrive(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Load into this CTA, counted on a barrier of either CTA of the pair.
__device__ __forceinline__ void load_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
      "[%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
// Scales are stored as 8-row x 16-byte matrices 128 bytes apart, unswizzled.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128u >> 4) << 32) |
         (static_cast<uint64_t>(1u) << 46);
}
// 512 bytes of scales of each CTA into 32 lanes x 4 columns of its tensor memory, repeated for every warp's lanes.
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void commit_both(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          ptx::smem_addr(bar)),
      "h"(static_cast<uint16_t>(3))
      : "memory");
}
__device__ __forceinline__ void commit_local(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(ptx::smem_addr(bar))
               : "memory");
}
// Staged output box to global memory; what lies past the matrix is cut off.
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t src, int32_t x, int32_t y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(src), "r"(x), "r"(y)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void wait_box_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void wait_box_written() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Bounded wait of a whole warp: one answer for all of its lanes, which go on converged.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar, parity, abort_flag, kWaitNs));
}
__device__ __forceinline__ void fail(Control* ctl, int32_t* status, int32_t role) {
  ctl->abort_flag = 1;
  report(status, MPM_ERR_DEVICE_TIMEOUT, role);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1)
    mxfp4_matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                        const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                        const __grid_constant__ CUtensorMap map_out, MxMatmulArgs a, bool tma_out, bool bias_vec) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_addr(smem_raw) & 1023u)) & 1023u);
  Control* ctl = reinterpret_cast<Control*>(smem + kStages * kStageBytes + kEpilogueWarps * kBoxBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(&ctl->full[s], 1);
      ptx::mbar_init(&ctl->empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&ctl->acc_full[i], 1);
      ptx::mbar_init(&ctl->acc_empty[i], 2 * kEpilogueWarps);
    }
    ptx::mbar_init(&ctl->drain, 1);
    ctl->abort_flag = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tensor_map(&map_a);
    ptx::prefetch_tensor_map(&map_b);
    ptx::prefetch_tensor_map(&map_sa);
    ptx::prefetch_tensor_map(&map_sb);
    if (tma_out) ptx::prefetch_tensor_map(&map_out);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     ptx::smem_addr(&ctl->tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  cluster_sync();  // barriers of both CTAs exist before any remote signal
  ptx::tc_fence_after_sync();
  const uint32_t tmem = ctl->tmem_base;
  wait_for_previous_grid();
  allow_next_grid();

  const int tiles_n = (a.n + kTileN - 1) / kTileN;
  const int64_t tiles = (a.m + kTileM - 1) / kTileM * tiles_n;
  const int64_t clusters = gridDim.x / 2, cluster = blockIdx.x / 2;
  const int stages_k = (a.k + kStageK - 1) / kStageK;
  const int tiles_k = mx::scale_tiles(a.k);
  volatile int* abort_flag = &ctl->abort_flag;

  if (warp == 0) {
    // ---------------- TMA producer (both CTAs) ----------------
    // The whole warp runs this loop and the next one; an elected lane issues.
    // In a branch of one lane every operand of a copy or product first moves to
    // a uniform register, about 70 cycles an instruction, which bound the
    // kernel: 8192 x 8192 x 8192 took 316 us instead of 176.
    {
      int stage = 0, issued = 0;
      uint32_t phase = 0, issued_phase = 0;
      bool ok = true;
      const uint32_t smem0 = __shfl_sync(0xFFFFFFFFu, ptx::smem_addr(smem), 0);
      const uint32_t full0 = __shfl_sync(0xFFFFFFFFu, map_to_rank(ptx::smem_addr(&ctl->full[0]), 0), 0);
      for (int64_t t = cluster; ok && t < tiles; t += clusters) {
        const int32_t m0 = static_cast<int32_t>(t / tiles_n) * kTileM + kHalf * static_cast<int32_t>(rank);
        const int32_t n0 = static_cast<int32_t>(t % tiles_n) * kTileN;
        for (int kb = 0; kb < stages_k; ++kb) {
          if (!warp_wait(&ctl->empty[stage], phase ^ 1u, abort_flag)) {
            fail(ctl, a.status, 21);
            ok = false;
            break;
          }
          const uint32_t at = smem0 + stage * kStageBytes, full = full0 + stage * 8;
          // A scale tile past the last one along K belongs to other rows, or reads as zeros: no product uses it.
          const int32_t kt = kb * kScaleTiles, nt = n0 / mx::kTileRows;
          if (ptx::elect_one()) {
            if (leader) ptx::mbar_arrive_expect_tx(&ctl->full[stage], 2 * kStageBytes);
            load_pair(at, &map_a, full, kb * 128, m0);
            load_pair(at + kBytesA, &map_b, full, kb * 128, n0 + kTileN / 2 * static_cast<int32_t>(rank));
            load_pair(at + kBytesA + kBytesB, &map_sa, full, 0, m0 / mx::kTileRows * tiles_k + kt);
            load_pair(at + kBytesA + kBytesB + kBytesSA, &map_sb, full, 0, nt * tiles_k + kt);
            load_pair(at + kBytesA + kBytesB + 2 * kBytesSA, &map_sb, full, 0, (nt + 1) * tiles_k + kt);
          }
          __syncwarp();
          issued |= 1 << stage;
          issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (!ok && leader) {
        for (int s = 0; s < kStages; ++s)
          if (issued & (1 << s)) ptx::mbar_wait(&ctl->full[s], (issued_phase >> s) & 1u, nullptr, kWaitNs);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA issuer (leader) ----------------
    if (leader) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      const uint32_t smem0 = __shfl_sync(0xFFFFFFFFu, ptx::smem_addr(smem), 0);
      const uint32_t tmem0 = __shfl_sync(0xFFFFFFFFu, tmem, 0);
      const uint64_t desc0 = ptx::sdesc_k_sw128(smem0);
      for (int64_t t = cluster; ok && t < tiles; t += clusters) {
        if (!warp_wait(&ctl->acc_empty[acc], acc_phase ^ 1u, abort_flag)) {
          fail(ctl, a.status, 22);
          break;
        }
        ptx::tc_fence_after_sync();
        const uint32_t d = tmem0 + static_cast<uint32_t>(acc * kTileN);
        // The tile's first row of B within its scale tile: a column of scales holds 32 rows.
        const uint32_t sb_shift = static_cast<uint32_t>(t % tiles_n) * kTileN % mx::kTileRows / 32;
        for (int kb = 0; kb < stages_k; ++kb) {
          if (!warp_wait(&ctl->full[stage], phase, abort_flag)) {
            fail(ctl, a.status, 23);
            ok = false;
            break;
          }
          ptx::tc_fence_after_sync();
          const uint64_t da = desc0 + static_cast<uint64_t>((stage * kStageBytes) >> 4), db = da + (kBytesA >> 4);
          const uint32_t scales = smem0 + stage * kStageBytes + kBytesA + kBytesB;
          const uint32_t sa = tmem0 + kScaleCols + stage * kStageCols, sb = sa + kScaleTiles * kColsSA;
          const int products = min(kStageK / 64, (a.k - kb * kStageK + 63) / 64);
          if (ptx::elect_one()) {
#pragma unroll
            for (int j = 0; j < kScaleTiles; ++j) {
              if (2 * j < products) {
                copy_scales(sa + j * kColsSA, scale_desc(scales + j * mx::kTileBytes));
                copy_scales(sb + j * kColsSB, scale_desc(scales + kBytesSA + j * mx::kTileBytes));
                copy_scales(sb + j * kColsSB + 4, scale_desc(scales + 2 * kBytesSA + j * mx::kTileBytes));
              }
            }
#pragma unroll
            for (int p = 0; p < kStageK / 64; ++p) {
              if (p < products)
                mma_mx(d, da + 2 * p, db + 2 * p, kIdesc | scale_half((p & 1) * 2), sa + (p / 2) * kColsSA,
                       sb + (p / 2) * kColsSB + sb_shift, (kb | p) != 0 ? 1u : 0u);
            }
            commit_both(&ctl->empty[stage]);
          }
          __syncwarp();
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!ok) break;
        if (ptx::elect_one()) commit_both(&ctl->acc_full[acc]);
        __syncwarp();
        if (++acc == 2) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
      if (ptx::elect_one()) commit_local(&ctl->drain);
      __syncwarp();
      ptx::mbar_wait(&ctl->drain, 0, nullptr, kWaitNs);
    }
    __syncwarp();
  } else {
    // ---------------- epilogue (both CTAs) ----------------
    // Warp (q, part): rows 32 q .. + 31 of this CTA, columns 64 part .. + 63 of
    // the tile, through a staged box of 32 rows x 128 bytes (64 bf16 or 32
    // fp32): a lane writes its own row, 16-byte piece p at p ^ (row & 7), which
    // is the 128-byte swizzle and free of bank conflicts; a TMA store takes the
    // box to global memory in whole 128-byte runs.  Stores from registers,
    // 16 bytes a row and instruction, took 144 us instead of the 75 that this
    // takes for 54208 x 768 x 2304 to bf16.
    const int q = warp & 3, part = (warp - 2) >> 2;
    const uint32_t empty0 = map_to_rank(ptx::smem_addr(&ctl->acc_empty[0]), 0);
    const uint32_t empty1 = map_to_rank(ptx::smem_addr(&ctl->acc_empty[1]), 0);
    uint8_t* box = smem + kStages * kStageBytes + (warp - 2) * kBoxBytes;
    constexpr int kBoxCols = 128 / static_cast<int>(sizeof(T));
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int64_t t = cluster; t < tiles; t += clusters) {
      const int64_t row0 = t / tiles_n * kTileM + kHalf * rank + q * 32;
      const int n0 = static_cast<int>(t % tiles_n) * kTileN + part * kWarpCols;
      const bool live = row0 < a.m && n0 < a.n;
      if (!warp_wait(&ctl->acc_full[acc], acc_phase, abort_flag)) {
        fail(ctl, a.status, 24);
        break;
      }
      ptx::tc_fence_after_sync();
      const uint32_t from = tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(acc * kTileN + part * kWarpCols);
#pragma unroll
      for (int c = 0; c < kWarpCols; c += 32) {
        uint32_t r[32];
        ptx::tmem_ld_32x32b_x32(from + c, r);
        ptx::tmem_wait_ld(r);
        if (c + 32 == kWarpCols) {
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) remote_arrive(acc == 0 ? empty0 : empty1);
        }
        if (!live) continue;
        const int n = n0 + c;
        if (a.bias != nullptr) {
          if (n + 32 <= a.n && bias_vec) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const float4 b = __ldg(reinterpret_cast<const float4*>(a.bias + n + i));
              r[i] = __float_as_uint(__uint_as_float(r[i]) + b.x);
              r[i + 1] = __float_as_uint(__uint_as_float(r[i + 1]) + b.y);
              r[i + 2] = __float_as_uint(__uint_as_float(r[i + 2]) + b.z);
              r[i + 3] = __float_as_uint(__uint_as_float(r[i + 3]) + b.w);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (n + i < a.n) r[i] = __float_as_uint(__uint_as_float(r[i]) + __ldg(a.bias + n + i));
          }
        }
        // The box that left from here last has been read.
        if ((sizeof(T) == 4 || c == 0) && lane == 0) wait_box_read();
        __syncwarp();
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            __nv_bfloat162 h[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
              h[j] = __floats2bfloat162_rn(__uint_as_float(r[8 * p + 2 * j]), __uint_as_float(r[8 * p + 2 * j + 1]));
            *reinterpret_cast<uint4*>(box + lane * 128 + (((c / 8 + p) ^ (lane & 7)) * 16)) = *reinterpret_cast<const uint4*>(h);
          }
        } else {
#pragma unroll
          for (int p = 0; p < 8; ++p)
            *reinterpret_cast<uint4*>(box + lane * 128 + ((p ^ (lane & 7)) * 16)) =
                make_uint4(r[4 * p], r[4 * p + 1], r[4 * p + 2], r[4 * p + 3]);
        }
        if (sizeof(T) == 2 && c + 32 < kWarpCols) continue;
        const int first = sizeof(T) == 2 ? n0 : n;
        if (tma_out) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0 && first < a.n) store_box(&map_out, ptx::smem_addr(box), first, static_cast<int32_t>(row0));
        } else {
          // Rows that are not 16-byte aligned: element by element, a warp along each row.
          __syncwarp();
          T* out = static_cast<T*>(a.out) + row0 * a.stride + first;
          const int rows = a.m - row0 < 32 ? static_cast<int>(a.m - row0) : 32;
          for (int i = 0; i < rows; ++i)
#pragma unroll
            for (int j = lane; j < kBoxCols; j += 32)
              if (first + j < a.n)
                out[i * a.stride + j] =
                    *reinterpret_cast<const T*>(box + i * 128 + (((j * static_cast<int>(sizeof(T)) / 16) ^ (i & 7)) * 16) +
                                                j * sizeof(T) % 16);
          __syncwarp();
        }
      }
      if (++acc == 2) {
        acc = 0;
        acc_phase ^= 1u;
      }
    }
    if (lane == 0) wait_box_written();  // shared memory outlives the stores that read it
    __syncwarp();
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  cluster_sync();  // no CTA leaves while its peer may still signal it
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
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

// Codes: boxes of 128 bytes x `box_rows` rows, swizzled.
bool map_codes(CUtensorMap* map, const uint8_t* codes, int64_t rows, int k, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(mx::code_pitch(k)), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {dims[0]};
  const cuuint32_t box[2] = {128, static_cast<cuuint32_t>(box_rows)}, each[2] = {1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(codes), dims, strides, box, each,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Scales: a row per 512-byte tile, boxes of one stage's tiles.
bool map_scales(CUtensorMap* map, const uint8_t* scales, int64_t rows, int k) {
  const cuuint64_t dims[2] = {mx::kTileBytes / 4, static_cast<cuuint64_t>(mx::row_tiles(rows) * mx::scale_tiles(k))};
  const cuuint64_t strides[1] = {mx::kTileBytes};
  const cuuint32_t box[2] = {mx::kTileBytes / 4, kScaleTiles}, each[2] = {1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t*>(scales), dims, strides, box, each,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Output: boxes of 32 rows x 128 bytes, swizzled.
template <typename T>
bool map_output(CUtensorMap* map, const MxMatmulArgs& a) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.n), static_cast<cuuint64_t>(a.m)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.m > 1 ? a.stride : (a.n + 15) / 16 * 16) * sizeof(T)};
  const cuuint32_t box[2] = {128 / sizeof(T), 32}, each[2] = {1, 1};
  return encoder()(map, sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, a.out,
                   dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T>
cudaError_t launch_instance(const MxMatmulArgs& a, int num_sms, cudaStream_t stream) {
  if (encoder() == nullptr) return cudaErrorNotSupported;
  CUtensorMap map_a, map_b, map_sa, map_sb;
  if (!map_codes(&map_a, a.a_codes, a.m, a.k, kHalf) || !map_codes(&map_b, a.b_codes, a.n, a.k, kTileN / 2) ||
      !map_scales(&map_sa, a.a_scales, a.m, a.k) || !map_scales(&map_sb, a.b_scales, a.n, a.k))
    return cudaErrorInvalidValue;
  static std::atomic<uint64_t> attr_done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(attr_done.load() & bit)) {
    e = cudaFuncSetAttribute(mxfp4_matmul_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(kSmemBytes));
    if (e != cudaSuccess) return e;
    attr_done.fetch_or(bit);
  }
  const int64_t tiles = (a.m + kTileM - 1) / kTileM * ((a.n + kTileN - 1) / kTileN);
  const int64_t pairs = num_sms > 1 ? num_sms / 2 : 1;
  CUtensorMap map_out = map_a;
  const bool tma_out = (a.m == 1 || a.stride * static_cast<int64_t>(sizeof(T)) % 16 == 0) &&
                       reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  if (tma_out && !map_output<T>(&map_out, a)) return cudaErrorInvalidValue;
  const bool bias_vec = reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * (tiles < pairs ? tiles : pairs)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, mxfp4_matmul_kernel<T>, map_a, map_b, map_sa, map_sb, map_out, a, tma_out,
                            bias_vec);
}

}  // namespace

cudaError_t launch_mxfp4_matmul(const MxMatmulArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  return bf16 ? launch_instance<__nv_bfloat16>(a, num_sms, stream) : launch_instance<float>(a, num_sms, stream);
}

}  // namespace mpm
