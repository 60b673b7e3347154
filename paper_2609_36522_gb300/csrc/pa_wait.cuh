// A bounded wait on an mbarrier for the layer kernels.
#pragma once

#include "pa_bulk.cuh"
#include "pa_internal.h"

namespace pa {

// Bounded wait (about a second); after a failure a thread no longer waits, runs
// on with accesses in bounds, and the call's results are not valid.
__device__ __forceinline__ void wait_or_bad(uint64_t* bar, uint32_t parity, bool& bad, int32_t* status) {
  if (bad || mbar_test(bar, parity)) return;
  const long long t0 = clock64();
  while (!mbar_try(bar, parity)) {
    if (clock64() - t0 > 2000000000ll) {
      bad = true;
      atomicCAS(status, 0, kDevTimeout);
      return;
    }
  }
}

}  // namespace pa
