// A pair of CTAs (a cluster of two) whose copies are counted on the barriers of
// the first, the leader: how a pair that gives up waits for copies under way.
//
// Both CTAs load the same sequence into their slots: load n goes to slot n % slots,
// and completes phase n / slots of the slot's barrier in the leader, which arms it
// with both CTAs' bytes when it issues its own half.  When a wait has run out
// somewhere, one may have issued loads that the other has not.
#pragma once

#include <stdint.h>

#include "ptx.cuh"

namespace mpm {
namespace pair {

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
// A word of the other CTA's shared memory, at the place of this one's.
__device__ __forceinline__ void store_to(const void* local, uint32_t rank, int value) {
  asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(map_to_rank(ptx::smem_addr(local), rank)), "r"(value) : "memory");
}
// Load into this CTA, counted on a barrier of either CTA of the pair.
__device__ __forceinline__ void load_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
      "[%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
      : "memory");
}

// By one thread of the leader, once neither CTA issues any more: waits, each
// time up to limit_ns, for the last loads of a ring, of which the leader issued
// `mine` and its peer `theirs`; `bytes` is one CTA's half.  False if one did not land.
static __device__ __noinline__ bool drain(uint64_t* full, int slots, uint32_t bytes, int mine, int theirs, uint64_t limit_ns) {
  const int last = mine > theirs ? mine : theirs;
  bool landed = true;
  for (int n = last > slots ? last - slots : 0; n < last; ++n) {
    uint64_t* bar = &full[n % slots];
    if (n >= mine)  // the peer's half alone, and nothing that it could complete
      ptx::mbar_arrive_expect_tx(bar, bytes);
    else if (n >= theirs)  // the peer's half will not come
      asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(ptx::smem_addr(bar)), "r"(bytes) : "memory");
    landed = ptx::mbar_wait(bar, static_cast<uint32_t>(n / slots) & 1u, nullptr, limit_ns) && landed;
  }
  return landed;
}

// What a CTA keeps in shared memory for this.
struct __align__(8) State {
  volatile int failed;                // a wait ran out in this CTA: zero at first, and so is
  volatile int peer_failed;           // the same of its peer
  int loads[2];                       // loads that it issued to each of its rings,
  int peer_loads[2];                  // and its peer did (leader)
};

// A wait ran out.
__device__ __forceinline__ void give_up(State* s) {
  s->failed = 1;
  store_to(const_cast<int*>(&s->peer_failed), cluster_rank() ^ 1u, 1);
}

// The end of a pair, by all threads of both CTAs, after all roles are done and
// a __syncthreads: no CTA leaves while its peer may still signal it or, where a
// wait ran out in either, while copies of either are under way.
// drain_rings() is called by one thread of the leader.
template <typename Drain>
__device__ __forceinline__ void leave(State* s, Drain drain_rings) {
  cluster_sync();
  if (*reinterpret_cast<volatile unsigned long long*>(s) == 0) return;  // neither failed
  const uint32_t rank = cluster_rank();
  if (rank != 0 && threadIdx.x == 0) {
    store_to(&s->peer_loads[0], 0, s->loads[0]);
    store_to(&s->peer_loads[1], 0, s->loads[1]);
  }
  cluster_sync();
  if (rank == 0 && threadIdx.x == 0) drain_rings();
  cluster_sync();
}

}  // namespace pair
}  // namespace mpm
