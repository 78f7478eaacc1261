// Two CTAs whose copies are counted on the first one's barriers, as in the 4-bit
// product (csrc/pair_ring.cuh): compiled and launched by test_gpu_row_ring.py.
// Both take `common` loads in step; then one issues up to load `mine`, the other
// up to `theirs`, and the pair gives up.  All copies lie inside the buffers and
// every wait ends by its limit.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>
#include <stdint.h>

#include "pair_ring.cuh"
#include "ptx.cuh"

namespace {

constexpr int kSlots = 3, kRows = 8, kCols = 32, kThreads = 64;
constexpr uint32_t kBytes = kRows * kCols * 4;

struct Result {
  int drained;              // what drain() said; -1: not called
  int in_step;              // waits of the loads in step that ended well
  int landed[2][kSlots];    // the load that each CTA's slots hold whole (-1: none)
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads)
    run_pair(const __grid_constant__ CUtensorMap map, int common, int mine, int theirs, int failed_rank, uint64_t limit_ns, Result* result) {
  __shared__ __align__(128) int slot[kSlots][kRows * kCols];
  __shared__ uint64_t full[kSlots];
  __shared__ mpm::pair::State state;
  const uint32_t rank = mpm::pair::cluster_rank();
  for (int i = threadIdx.x; i < kSlots * kRows * kCols; i += kThreads) slot[i / (kRows * kCols)][i % (kRows * kCols)] = -1;
  if (threadIdx.x == 0) {
    state.failed = state.peer_failed = 0;
    for (int k = 0; k < kSlots; ++k) mpm::ptx::mbar_init(&full[k], 1);
    mpm::ptx::fence_barrier_init();
    if (rank == 0) result->drained = -1, result->in_step = 0;
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncthreads();
  mpm::pair::cluster_sync();
  auto load = [&](int n) {
    if (rank == 0) mpm::ptx::mbar_arrive_expect_tx(&full[n % kSlots], 2 * kBytes);
    mpm::pair::load_pair(mpm::ptx::smem_addr(slot[n % kSlots]), &map,
                         mpm::pair::map_to_rank(mpm::ptx::smem_addr(&full[n % kSlots]), 0), 0, (2 * n + static_cast<int>(rank)) * kRows);
  };
  for (int n = 0; n < common; ++n) {
    if (threadIdx.x == 0) {
      load(n);
      if (rank == 0 && mpm::ptx::mbar_wait(&full[n % kSlots], static_cast<uint32_t>(n / kSlots) & 1u, nullptr, limit_ns))
        ++result->in_step;
    }
    __syncwarp();
    mpm::pair::cluster_sync();
  }
  const int count = rank == 0 ? mine : theirs;
  if (threadIdx.x == 0) {
    for (int n = common; n < count; ++n) load(n);
    state.loads[0] = count;
    state.loads[1] = 0;
    if (static_cast<int>(rank) == failed_rank) mpm::pair::give_up(&state);
  }
  __syncthreads();
  mpm::pair::leave(&state, [&] {
    result->drained = mpm::pair::drain(full, kSlots, kBytes, state.loads[0], state.peer_loads[0], limit_ns) ? 1 : 0;
  });
  if (failed_rank >= 0 && threadIdx.x < kSlots) {
    const int* s = slot[threadIdx.x];
    const int n = s[0] / 10000;
    bool whole = s[0] >= 0;
    for (int i = 0; i < kRows * kCols; ++i) whole = whole && s[i] == 10000 * n + 1000 * static_cast<int>(rank) + i;
    result->landed[rank][threadIdx.x] = whole ? n : -1;
  }
}

}  // namespace

// values: int32 [2 loads x 8 rows, 32]
extern "C" __attribute__((visibility("default"))) int run_pair_ring(const void* values, int loads, int common, int mine, int theirs,
                                                                     int failed_rank, unsigned limit_us, void* result, void* stream) {
  if (common < 0 || mine < common || theirs < common || mine > common + kSlots || theirs > common + kSlots || mine > loads ||
      theirs > loads || limit_us < 1 || limit_us > 1000000u)
    return 1;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
      q != cudaDriverEntryPointSuccess)
    return 2;
  CUtensorMap map;
  const cuuint64_t dims[2] = {kCols, static_cast<cuuint64_t>(2 * loads * kRows)}, strides[1] = {kCols * 4};
  const cuuint32_t box[2] = {kCols, kRows}, each[2] = {1, 1};
  if (reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p)(
          &map, CU_TENSOR_MAP_DATA_TYPE_INT32, 2, const_cast<void*>(values), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return 3;
  run_pair<<<2, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(map, common, mine, theirs, failed_rank, 1000ull * limit_us,
                                                                  static_cast<Result*>(result));
  return cudaGetLastError() == cudaSuccess ? 0 : 4;
}
