// What a ring of rows in shared memory does when a wait for a row ran out.
//
// One lane of a group issues the copies into the group's slots: row n of the
// group's run goes to slot n % slots, and its barrier's phase n / slots.  A wait
// that runs out sets `dead` for the block.  From then on no row is asked for;
// and before shared memory is put to another use, or the block leaves it to
// the next one, the copies that are still under way are waited for.
#pragma once

#include <stdint.h>

#include "ptx.cuh"

namespace mpm {
namespace ring {

// Asks for the run's next row by fill(), and counts it in `asked`; not once a
// wait has run out.  By the group's issuing lane only, row after row.
template <typename Fill>
__device__ __forceinline__ void refill(const volatile int* dead, int* asked, Fill fill) {
  if (*dead != 0) return;
  fill();
  ++*asked;
}

// Waits, each time up to limit_ns, for the copies of the last of the `asked`
// rows; false if one did not land.
static __device__ __noinline__ bool drain(uint64_t* full, int slots, int asked, uint64_t limit_ns) {
  bool landed = true;
  for (int n = asked > slots ? asked - slots : 0; n < asked; ++n)
    landed = ptx::mbar_wait(&full[n % slots], static_cast<uint32_t>(n / slots) & 1u, nullptr, limit_ns) && landed;
  return landed;
}

}  // namespace ring
}  // namespace mpm
