// out[m, n] = sum_k A[m, k] B[n, k] + bias[n] for MXFP4 operands (mxfp4.cuh),
// accumulated in fp32 on the tensor cores: tcgen05.mma kind::mxf4 with a
// power-of-two scale per 32 elements.
//
// A cluster of two CTAs (an SM pair) computes 256 x N tiles (N = 192, or 64, 128
// or 256) with cta_group::2: each CTA stages its 128 rows of A, half of the tile's rows
// of B, the scales of its A rows and those of all of the tile's B rows.  A step
// takes 256 elements of every row, one 128-byte swizzle row of packed codes,
// and four K = 64 products.  Scales go from shared memory to tensor memory by
// tcgen05.cp, into columns that belong to the slot they came in: the products
// that read them have completed before the slot is filled again.
//
// Bound: with few features the output's bytes (2 M N of them against
// (M + N) K / 2: 256 x 192 tiles of K = 768 take the tensor cores a third of
// the time that their output takes HBM), with many shared memory.  Hence
//  - tiles of 192 columns with two accumulators: a tile's output is written
//    while the next one is computed;
//  - A and B in rings of their own: where a row of A fits (K <= 1280; 1024 with
//    tiles of 256 columns), the A panel of a run of tiles stays in shared memory,
//    and with it its scales in tensor memory.  Loading it again for every tile
//    took as long as half of the output's writes (54208 x 768 x 2304 to bf16: 61
//    us, resident 57, which is 4.4 TB/s of writes; filling as much memory with
//    zeros reaches 3.9);
//  - tiles of 256 columns for many features.  A step's operands are written to
//    shared memory once and read once: 60 KB a CTA for 192 columns, 467 cycles
//    at 128 bytes a cycle against 384 of the products; 68 KB and 530 cycles
//    against 512 for 256 columns.  Tensor memory has room for one accumulator
//    then, and a tile waits until the last one's has been read: 16384 x 4096 x
//    1024 takes 34 us with 192 columns and 30 with 256, where that traffic and
//    the rounds of tiles alone would allow 22; 8192 x 8192 x 8192 180 and 172.
//    Tiles of 128 took as long as 192 for two thirds of the work.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>

#include "common.cuh"
#include "mxfp4.cuh"
#include "pair_ring.cuh"
#include "ptx.cuh"

namespace mpm {
namespace {

using pair::cluster_sync;
using pair::load_pair;
using pair::map_to_rank;

constexpr int kHalf = 128;             // rows of A per CTA
constexpr int kTileM = 2 * kHalf;
constexpr int kStepK = 256;            // elements of a row per step: 128 bytes
constexpr int kScaleTiles = kStepK / (mx::kBlock * mx::kTileBlocks);  // scale tiles along K per step
constexpr int kBytesA = kHalf * 128, kBytesSA = kScaleTiles * mx::kTileBytes, kSlotA = kBytesA + kBytesSA;
constexpr int kWarpCols = 64;              // columns of the tile that an epilogue warp writes
constexpr int kBoxBytes = 32 * 128;        // staged output: 32 rows of 128 bytes, swizzled
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColsSA = 4;            // tensor-memory columns of a scale tile
constexpr uint64_t kWaitNs = 2000000000ull;

// What depends on a tile's columns.
template <int N>
struct Tile {
  static constexpr int kAccumulators = N == 256 ? 1 : 2;
  static constexpr int kSlotsA = N == 256 ? 5 : 6, kSlotsB = N == 256 ? 4 : N == 192 ? 5 : 6;
  static constexpr int kRowTiles = N > mx::kTileRows ? 2 : 1;  // scale tiles along N that a tile's rows of B lie in
  static constexpr uint32_t kColsSB = kRowTiles * kColsSA;
  static constexpr int kMaxResident = kSlotsA - 1;  // steps of a panel that stays: one slot is left to begin the next one
  static constexpr int kBytesB = N / 2 * 128, kBytesSB = kRowTiles * kBytesSA, kSlotB = kBytesB + kBytesSB;
  // Tensor memory: the accumulators, the scales of A's slots, those of B's.
  static constexpr uint32_t kScalesA = kAccumulators * N, kScalesB = kScalesA + kSlotsA * kScaleTiles * kColsSA;
  static constexpr int kEpilogueWarps = 4 * (N / kWarpCols);
  static constexpr int kThreads = (2 + kEpilogueWarps) * 32;
  static constexpr int kRings = kSlotsA * kSlotA + kSlotsB * kSlotB;
  static_assert(kScalesB + kSlotsB * kScaleTiles * kColsSB <= kTmemCols, "accumulators and scales share tensor memory");
  static_assert(kSlotA % 1024 == 0 && kSlotB % 1024 == 0 && kBytesB % 1024 == 0, "swizzled tiles on 1024 bytes");
};
constexpr int kWideK = 2048;  // features from which tiles take 256 columns, if there is a round of them

// Instruction descriptor of kind::mxf4: E2M1 operands (1) in K-major order,
// scales of type UE8M0 (bit 23), N / 8 and M / 16 in their fields.
__host__ __device__ constexpr uint32_t instruction(int n) {
  return (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) |
         (static_cast<uint32_t>(kTileM >> 4) << 24);
}
// Which half of a 32-bit column's four scales a K = 64 product takes: fields of B and of A.
__device__ __forceinline__ constexpr uint32_t scale_half(uint32_t which) { return (which << 4) | (which << 29); }

constexpr int kMaxSlots = 6;
struct Control {
  uint64_t full_a[kMaxSlots], full_b[kMaxSlots];    // leader: both CTAs' operands of the slot landed
  uint64_t empty_a[kMaxSlots], empty_b[kMaxSlots];  // both: products reading the slot completed
  uint64_t acc_full[2];                           // both: accumulator complete
  uint64_t acc_empty[2];                          // leader: both CTAs read the accumulator
  uint64_t drain;
  uint32_t tmem_base;
  pair::State pair;  // its rings: A, B
};

template <int N>
constexpr size_t smem_bytes() {
  return 1024 + static_cast<size_t>(Tile<N>::kRings) + Tile<N>::kEpilogueWarps * kBoxBytes + sizeof(Control);
}
static_assert(smem_bytes<64>() <= 227 * 1024 && smem_bytes<128>() <= 227 * 1024 && smem_bytes<192>() <= 227 * 1024 &&
                  smem_bytes<256>() <= 227 * 1024,
              "a block's shared memory");

// Place in a ring.
template <int SLOTS>
struct Ring {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++slot == SLOTS) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// A cluster's run of tiles, numbered with n fastest.
struct Tiles {
  int64_t begin, end;
  int n;  // tiles along n
  __device__ __forceinline__ int64_t m_of(int64_t t) const { return t / n; }
};
__device__ __forceinline__ Tiles tiles_of(const MxMatmulArgs& a, int tile_n) {
  const int n = (a.n + tile_n - 1) / tile_n;
  const int64_t all = (a.m + kTileM - 1) / kTileM * n, clusters = gridDim.x / 2, c = blockIdx.x / 2;
  const int64_t per = all / clusters, extra = all % clusters, begin = c * per + (c < extra ? c : extra);
  return {begin, begin + per + (c < extra ? 1 : 0), n};
}

__device__ __forceinline__ void remote_arrive(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
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
  pair::give_up(&ctl->pair);
  report(status, MPM_ERR_DEVICE_TIMEOUT, role);
}

template <typename T, int N>
__global__ void __launch_bounds__(Tile<N>::kThreads, 1)
    mxfp4_matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                        const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                        const __grid_constant__ CUtensorMap map_out, MxMatmulArgs a, bool tma_out, bool bias_vec) {
  using W = Tile<N>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_addr(smem_raw) & 1023u)) & 1023u);
  Control* ctl = reinterpret_cast<Control*>(smem + W::kRings + W::kEpilogueWarps * kBoxBytes);
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = pair::cluster_rank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < W::kSlotsA; ++s) {
      ptx::mbar_init(&ctl->full_a[s], 1);
      ptx::mbar_init(&ctl->empty_a[s], 1);
    }
    for (int s = 0; s < W::kSlotsB; ++s) {
      ptx::mbar_init(&ctl->full_b[s], 1);
      ptx::mbar_init(&ctl->empty_b[s], 1);
    }
    for (int i = 0; i < W::kAccumulators; ++i) {
      ptx::mbar_init(&ctl->acc_full[i], 1);
      ptx::mbar_init(&ctl->acc_empty[i], 2 * W::kEpilogueWarps);
    }
    ptx::mbar_init(&ctl->drain, 1);
    ctl->pair.failed = ctl->pair.peer_failed = 0;
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

  const Tiles run = tiles_of(a, N);
  const int steps = (a.k + kStepK - 1) / kStepK;
  const int tiles_k = mx::scale_tiles(a.k);
  // A panel (the 256 rows of A of a tile) stays for the run's next tiles of the same rows.
  const bool resident = steps <= W::kMaxResident;
  auto panel_begins = [&](int64_t t) { return !resident || t == run.begin || run.m_of(t) != run.m_of(t - 1); };
  auto panel_ends = [&](int64_t t) { return !resident || t + 1 == run.end || run.m_of(t + 1) != run.m_of(t); };
  volatile int* abort_flag = &ctl->pair.failed;

  if (warp == 0) {
    // ---------------- TMA producer (both CTAs) ----------------
    // The whole warp runs this loop and the next one; an elected lane issues.
    // In a branch of one lane every operand of a copy or product first moves to
    // a uniform register, about 70 cycles an instruction, which bound the
    // kernel: 8192 x 8192 x 8192 took 316 us instead of 176 (192
    // columns; 172 with 256).
    Ring<W::kSlotsA> ra;
    Ring<W::kSlotsB> rb;
    int loads_a = 0, loads_b = 0;
    bool ok = true;
    const uint32_t smem0 = __shfl_sync(0xFFFFFFFFu, ptx::smem_addr(smem), 0);
    const uint32_t full_a0 = __shfl_sync(0xFFFFFFFFu, map_to_rank(ptx::smem_addr(&ctl->full_a[0]), 0), 0);
    const uint32_t full_b0 = __shfl_sync(0xFFFFFFFFu, map_to_rank(ptx::smem_addr(&ctl->full_b[0]), 0), 0);
    for (int64_t t = run.begin; ok && t < run.end; ++t) {
      const int32_t m0 = static_cast<int32_t>(run.m_of(t)) * kTileM + kHalf * static_cast<int32_t>(rank);
      const int32_t n0 = static_cast<int32_t>(t - run.m_of(t) * run.n) * N, nt = n0 / mx::kTileRows;
      const bool begins = panel_begins(t);
      for (int kb = 0; kb < steps; ++kb) {
        // A scale tile past the last one along K belongs to other rows, or reads as zeros: no product uses it.
        const int32_t kt = kb * kScaleTiles;
        if (begins) {
          if (!warp_wait(&ctl->empty_a[ra.slot], ra.phase ^ 1u, abort_flag)) {
            fail(ctl, a.status, 21);
            ok = false;
            break;
          }
          const uint32_t at = smem0 + ra.slot * kSlotA, full = full_a0 + ra.slot * 8;
          if (ptx::elect_one()) {
            if (leader) ptx::mbar_arrive_expect_tx(&ctl->full_a[ra.slot], 2 * kSlotA);
            load_pair(at, &map_a, full, kb * 128, m0);
            load_pair(at + kBytesA, &map_sa, full, 0, m0 / mx::kTileRows * tiles_k + kt);
          }
          __syncwarp();
          ++loads_a;
          ra.next();
        }
        if (!warp_wait(&ctl->empty_b[rb.slot], rb.phase ^ 1u, abort_flag)) {
          fail(ctl, a.status, 22);
          ok = false;
          break;
        }
        const uint32_t at = smem0 + W::kSlotsA * kSlotA + rb.slot * W::kSlotB, full = full_b0 + rb.slot * 8;
        if (ptx::elect_one()) {
          if (leader) ptx::mbar_arrive_expect_tx(&ctl->full_b[rb.slot], 2 * W::kSlotB);
          load_pair(at, &map_b, full, kb * 128, n0 + N / 2 * static_cast<int32_t>(rank));
#pragma unroll
          for (int j = 0; j < W::kRowTiles; ++j)
            load_pair(at + W::kBytesB + j * kBytesSA, &map_sb, full, 0, (nt + j) * tiles_k + kt);
        }
        __syncwarp();
        ++loads_b;
        rb.next();
      }
    }
    if (lane == 0) {
      ctl->pair.loads[0] = loads_a;
      ctl->pair.loads[1] = loads_b;
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA issuer (leader) ----------------
    if (leader) {
      Ring<W::kSlotsA> ra;
      Ring<W::kSlotsB> rb;
      int acc = 0;
      uint32_t acc_phase = 0;
      bool ok = true;
      const uint32_t smem0 = __shfl_sync(0xFFFFFFFFu, ptx::smem_addr(smem), 0);
      const uint32_t tmem0 = __shfl_sync(0xFFFFFFFFu, tmem, 0);
      const uint64_t desc0 = ptx::sdesc_k_sw128(smem0);
      for (int64_t t = run.begin; ok && t < run.end; ++t) {
        if (!warp_wait(&ctl->acc_empty[acc], acc_phase ^ 1u, abort_flag)) {
          fail(ctl, a.status, 23);
          break;
        }
        ptx::tc_fence_after_sync();
        const uint32_t d = tmem0 + static_cast<uint32_t>(acc * N);
        // The tile's first row of B within its scale tile: a column of scales holds 32 rows.
        const uint32_t sb_shift = static_cast<uint32_t>(t - run.m_of(t) * run.n) * N % mx::kTileRows / 32;
        const bool begins = panel_begins(t), ends = panel_ends(t);
        Ring<W::kSlotsA> at = ra;  // the panel's slots
        for (int kb = 0; kb < steps; ++kb) {
          if ((begins && !warp_wait(&ctl->full_a[at.slot], at.phase, abort_flag)) ||
              !warp_wait(&ctl->full_b[rb.slot], rb.phase, abort_flag)) {
            fail(ctl, a.status, 24);
            ok = false;
            break;
          }
          ptx::tc_fence_after_sync();
          const uint32_t slot_a = at.slot * kSlotA, slot_b = W::kSlotsA * kSlotA + rb.slot * W::kSlotB;
          const uint64_t da = desc0 + static_cast<uint64_t>(slot_a >> 4), db = desc0 + static_cast<uint64_t>(slot_b >> 4);
          const uint32_t sa = tmem0 + W::kScalesA + at.slot * (kScaleTiles * kColsSA);
          const uint32_t sb = tmem0 + W::kScalesB + rb.slot * (kScaleTiles * W::kColsSB);
          const int products = min(kStepK / 64, (a.k - kb * kStepK + 63) / 64);
          if (ptx::elect_one()) {
#pragma unroll
            for (int j = 0; j < kScaleTiles; ++j) {
              if (2 * j < products) {
                if (begins) copy_scales(sa + j * kColsSA, scale_desc(smem0 + slot_a + kBytesA + j * mx::kTileBytes));
#pragma unroll
                for (int i = 0; i < W::kRowTiles; ++i)
                  copy_scales(sb + j * W::kColsSB + 4 * i,
                              scale_desc(smem0 + slot_b + W::kBytesB + i * kBytesSA + j * mx::kTileBytes));
              }
            }
#pragma unroll
            for (int p = 0; p < kStepK / 64; ++p) {
              if (p < products)
                mma_mx(d, da + 2 * p, db + 2 * p, instruction(N) | scale_half((p & 1) * 2), sa + (p / 2) * kColsSA,
                       sb + (p / 2) * W::kColsSB + sb_shift, (kb | p) != 0 ? 1u : 0u);
            }
            commit_both(&ctl->empty_b[rb.slot]);
            if (ends) commit_both(&ctl->empty_a[at.slot]);
          }
          __syncwarp();
          at.next();
          rb.next();
        }
        if (!ok) break;
        if (ends) ra = at;
        if (ptx::elect_one()) commit_both(&ctl->acc_full[acc]);
        __syncwarp();
        if (++acc == W::kAccumulators) {
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
    // 16 bytes a row and instruction, took 144 us instead of 75 for 54208 x
    // 768 x 2304 to bf16, before the A panel stayed (54 to 57 now).
    const int q = warp & 3, part = (warp - 2) >> 2;
    const uint32_t empty0 = map_to_rank(ptx::smem_addr(&ctl->acc_empty[0]), 0);
    const uint32_t empty1 = map_to_rank(ptx::smem_addr(&ctl->acc_empty[1]), 0);
    uint8_t* box = smem + W::kRings + (warp - 2) * kBoxBytes;
    constexpr int kBoxCols = 128 / static_cast<int>(sizeof(T));
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int64_t t = run.begin; t < run.end; ++t) {
      const int64_t row0 = run.m_of(t) * kTileM + kHalf * rank + q * 32;
      const int n0 = static_cast<int>(t - run.m_of(t) * run.n) * N + part * kWarpCols;
      const bool live = row0 < a.m && n0 < a.n;
      if (!warp_wait(&ctl->acc_full[acc], acc_phase, abort_flag)) {
        fail(ctl, a.status, 25);
        break;
      }
      ptx::tc_fence_after_sync();
      const uint32_t from = tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(acc * N + part * kWarpCols);
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
      if (++acc == W::kAccumulators) {
        acc = 0;
        acc_phase ^= 1u;
      }
    }
    if (lane == 0) wait_box_written();  // shared memory outlives the stores that read it
    __syncwarp();
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  // No CTA leaves while its peer may still signal it, or a copy of a pair that gave up may still land.
  pair::leave(&ctl->pair, [&] {
    pair::drain(ctl->full_a, W::kSlotsA, kSlotA, ctl->pair.loads[0], ctl->pair.peer_loads[0], kWaitNs);
    pair::drain(ctl->full_b, W::kSlotsB, W::kSlotB, ctl->pair.loads[1], ctl->pair.peer_loads[1], kWaitNs);
  });
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

template <typename T, int N>
cudaError_t launch_instance(const MxMatmulArgs& a, int num_sms, cudaStream_t stream) {
  if (encoder() == nullptr) return cudaErrorNotSupported;
  const auto kernel = mxfp4_matmul_kernel<T, N>;
  CUtensorMap map_a, map_b, map_sa, map_sb;
  if (!map_codes(&map_a, a.a_codes, a.m, a.k, kHalf) || !map_codes(&map_b, a.b_codes, a.n, a.k, N / 2) ||
      !map_scales(&map_sa, a.a_scales, a.m, a.k) || !map_scales(&map_sb, a.b_scales, a.n, a.k))
    return cudaErrorInvalidValue;
  static std::atomic<uint64_t> attr_done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(attr_done.load() & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<N>()));
    if (e != cudaSuccess) return e;
    attr_done.fetch_or(bit);
  }
  const int64_t tiles = (a.m + kTileM - 1) / kTileM * ((a.n + N - 1) / N);
  const int64_t pairs = num_sms > 1 ? num_sms / 2 : 1;
  CUtensorMap map_out = map_a;
  const bool tma_out = (a.m == 1 || a.stride * static_cast<int64_t>(sizeof(T)) % 16 == 0) &&
                       reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  if (tma_out && !map_output<T>(&map_out, a)) return cudaErrorInvalidValue;
  const bool bias_vec = reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * (tiles < pairs ? tiles : pairs)));
  cfg.blockDim = dim3(Tile<N>::kThreads);
  cfg.dynamicSmemBytes = smem_bytes<N>();
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
  return cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, map_sa, map_sb, map_out, a, tma_out, bias_vec);
}

// The width of the tiles.  Where they are fewer than the SM pairs, narrow ones:
// more pairs share the work (graph of launches, N = 64 / 128 / 192: 128 x 768 x
// 768 3.5 / 4.0 / 4.5 us, 1000 x 1024 x 1024 4.3 / 4.3 / 4.7, 1 x 1024 x 4096 4.6
// / 3.9 / 4.0: 64 columns for at most two thirds of the pairs).  256 columns
// where those make one round and 192 would make two (1 x 4096 x 16384: 15.3 us
// with 192, 13.7), and for many features and at least a round of them
// (20000 x 2048 x 2048: 40 us with 192, 39; at 16384 x 1280 x 4096 39 and 42).
template <typename T>
cudaError_t launch_widths(const MxMatmulArgs& a, int num_sms, cudaStream_t stream) {
  const int64_t pairs = num_sms > 1 ? num_sms / 2 : 1;
  auto tiles = [&](int width) { return (a.m + kTileM - 1) / kTileM * ((static_cast<int64_t>(a.n) + width - 1) / width); };
  if (3 * tiles(64) <= 2 * pairs) return launch_instance<T, 64>(a, num_sms, stream);
  if (tiles(128) <= pairs) return launch_instance<T, 128>(a, num_sms, stream);
  const bool one_round = a.m <= kTileM && tiles(256) <= pairs && tiles(192) > pairs;
  if (one_round || (a.k >= kWideK && tiles(256) >= pairs)) return launch_instance<T, 256>(a, num_sms, stream);
  return launch_instance<T, 192>(a, num_sms, stream);
}

}  // namespace

cudaError_t launch_mxfp4_matmul(const MxMatmulArgs& a, bool bf16, int num_sms, cudaStream_t stream) {
  return bf16 ? launch_widths<__nv_bfloat16>(a, num_sms, stream) : launch_widths<float>(a, num_sms, stream);
}

}  // namespace mpm
