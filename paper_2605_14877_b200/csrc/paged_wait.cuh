// Waits of the paged-cache kernels: bounded by the clock, so that a hand-over that never comes ends a call within seconds.
#pragma once
#include "paged.h"
#include "tc_common.cuh"

namespace heatkv {

constexpr uint64_t PAGED_WAIT_NS = 2000000000ull;      // far above any launch's longest legitimate wait for one tile

__device__ __forceinline__ uint64_t global_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// Returns false when the CTA is leaving (this wait or another one ran out); the first to run out leaves its `code` in the status word.
__device__ __forceinline__ bool timed_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status, uint32_t code) {
  if (tc::mbar_try(bar, parity)) return true;
  const uint64_t begun = global_ns();
#pragma unroll 1
  while (!tc::mbar_try(bar, parity)) {
    if (*abort_flag) return false;
    if (global_ns() - begun > PAGED_WAIT_NS) {
      *abort_flag = 1;
      atomicCAS(status, 0u, code);
      return false;
    }
  }
  return true;
}
// ... by a whole warp, with one answer
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status, uint32_t code) {
  return __all_sync(0xffffffffu, timed_wait(bar, parity, abort_flag, status, code));
}
// Before leaving early: a copy under way lands (or a second passes).
__device__ __forceinline__ void settle(uint32_t bar, uint32_t parity) {
  const uint64_t begun = global_ns();
#pragma unroll 1
  while (!tc::mbar_try(bar, parity) && global_ns() - begun < PAGED_WAIT_NS / 2) {}
}

}  // namespace heatkv
