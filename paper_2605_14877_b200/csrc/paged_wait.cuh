// Waits of the paged-cache kernels: bounded by the clock, so that a hand-over that never comes ends a call within seconds.
#pragma once
#include "paged.h"
#include "tc_common.cuh"

namespace heatkv {

constexpr long long PAGED_WAIT_CYCLES = 4000000000ll;   // about two seconds: far above any launch's longest legitimate wait for one tile

// Returns false when the CTA is leaving (this wait or another one ran out); the first to run out leaves its `code` in the status word.
__device__ __forceinline__ bool timed_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status, uint32_t code,
                                           long long limit = PAGED_WAIT_CYCLES) {
  uint32_t tries = 0;
  long long begun = 0;
#pragma unroll 1
  while (!tc::mbar_try(bar, parity)) {
    if (*abort_flag) return false;
    if ((++tries & 63u) == 0) {                        // (the clock is looked at seldom: a wait's end sits on the chain of every tile)
      const long long now = clock64();
      if (begun == 0) {
        begun = now;
      } else if (now - begun > limit) {
        *abort_flag = 1;
        atomicCAS(status, 0u, code);
        return false;
      }
    }
  }
  return true;
}
// ... by a whole warp, with one answer
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status, uint32_t code,
                                         long long limit = PAGED_WAIT_CYCLES) {
  return __all_sync(0xffffffffu, timed_wait(bar, parity, abort_flag, status, code, limit));
}
// Before leaving early: a copy under way lands (or a second passes).
__device__ __forceinline__ void settle(uint32_t bar, uint32_t parity, long long limit = PAGED_WAIT_CYCLES / 2) {
  const long long begun = clock64();
#pragma unroll 1
  while (!tc::mbar_try(bar, parity) && clock64() - begun < limit) {}
}

}  // namespace heatkv
