// A run of rows through one ring, with csrc/row_ring.cuh as the backward pass of
// block_norm uses it: compiled and launched by test_gpu_row_ring.py.  The
// barrier of row `stuck` expects 16 bytes that no copy brings, so that the wait
// for it runs out; every wait ends by its limit and every copy that is asked
// for is inside the buffers.
#include <cuda_runtime.h>
#include <stdint.h>

#include "ptx.cuh"
#include "row_ring.cuh"

namespace {

constexpr int kSlots = 3, kWords = 64, kThreads = 64;

struct Result {
  int asked;       // rows that were asked for
  int ran_out;     // waits that gave up, of the first warp
  int drained;     // what drain() said: 1 landed, 0 one did not, -1 not called
  int landed[kSlots];  // after it: the row that each slot holds whole (-1: none)
};

__global__ void __launch_bounds__(kThreads) run_rows(const int* rows, int n, int stuck, uint64_t limit_ns, int* sums, Result* result) {
  __shared__ __align__(16) int slot[kSlots][kWords];
  __shared__ uint64_t full[kSlots];
  __shared__ int dead, asked;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kSlots * kWords; i += kThreads) slot[i / kWords][i % kWords] = -1;
  if (threadIdx.x == 0) {
    dead = asked = 0;
    for (int k = 0; k < kSlots; ++k) mpm::ptx::mbar_init(&full[k], 1);
    mpm::ptx::fence_barrier_init();
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncthreads();
  auto fill = [&](int row) {
    uint64_t* bar = &full[row % kSlots];
    mpm::ptx::mbar_arrive_expect_tx(bar, 4 * kWords + (row == stuck ? 16 : 0));
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     mpm::ptx::smem_addr(slot[row % kSlots])),
                 "l"(rows + row * kWords), "r"(4 * kWords), "r"(mpm::ptx::smem_addr(bar))
                 : "memory");
  };
  if (warp == 0 && mpm::ptx::elect_one())
    for (int r = 0; r < kSlots && r < n; ++r) mpm::ring::refill(&dead, &asked, [&] { fill(r); });
  __syncwarp();
  int ran_out = 0;
  for (int r = 0; r < n; ++r) {
    const bool ok = mpm::ptx::mbar_wait(&full[r % kSlots], static_cast<uint32_t>(r / kSlots) & 1u, &dead, limit_ns);
    if (!ok) {
      dead = 1;
      ++ran_out;
    }
    int v = slot[r % kSlots][threadIdx.x];
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if (lane == 0) sums[2 * r + warp] = v;
    __syncthreads();  // both warps have taken the row
    if (warp == 0 && r + kSlots < n && mpm::ptx::elect_one())
      mpm::ring::refill(&dead, &asked, [&] { fill(r + kSlots); });
    __syncwarp();
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    result->ran_out = ran_out;
    result->drained = -1;
    if (dead != 0) result->drained = mpm::ring::drain(full, kSlots, asked, limit_ns) ? 1 : 0;
    result->asked = asked;
    for (int k = 0; k < kSlots; ++k) {
      const int row = slot[k][0] / 1000;
      bool whole = slot[k][0] >= 0;
      for (int i = 0; i < kWords; ++i) whole = whole && slot[k][i] == 1000 * row + i;
      result->landed[k] = whole ? row : -1;
    }
  }
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int run_row_ring(const void* rows, int n, int stuck, unsigned limit_us, void* sums, void* result, void* stream) {
  if (n < 1 || limit_us < 1 || limit_us > 1000000u) return 1;
  run_rows<<<1, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const int*>(rows), n, stuck, 1000ull * limit_us, static_cast<int*>(sums), static_cast<Result*>(result));
  return cudaGetLastError() == cudaSuccess ? 0 : 2;
}
