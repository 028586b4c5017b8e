// Waits of the roles of a CTA on its mbarriers.
#pragma once

#include "common.cuh"
#include "warp_wait.cuh"

namespace lsp {

// Bounded wait that also gives up when another role has; for whole warps, the same answer in every lane.
struct BarrierWait {
  uint32_t bar, parity;
  volatile int* abort;
  unsigned* err;
  __device__ __forceinline__ bool ready() const { return mbar_try_wait(bar, parity); }
  __device__ __forceinline__ bool all(bool x) const { return __all_sync(0xffffffffu, x); }
  __device__ __forceinline__ bool any(bool x) const { return __any_sync(0xffffffffu, x); }
  __device__ __forceinline__ bool gone() const { return *abort != 0; }
  __device__ __forceinline__ uint64_t now() const { return global_ns(); }
  __device__ __forceinline__ void give_up(bool late) const {
    if (late) set_err(err, LSP_DEV_TIMEOUT);
    *abort = 1;
  }
};
__device__ __forceinline__ bool tc_wait(uint32_t bar, uint32_t parity, volatile int* abort, unsigned* err) {
  return warp_wait(BarrierWait{bar, parity, abort, err}, kWaitLimitNs);
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Arrival of a warp at the barrier behind which a copy may write over what it has read
// in shared memory.  An arrival does not wait for loads that are on their way, and the
// copy does not queue behind them: so it is made to need them.  read: bits of every
// load's result; zero: a 0 that the compiler does not know of.
__device__ __forceinline__ void arrive_after_reads(uint32_t bar, uint32_t read, uint32_t zero) {
  const uint32_t none = __ballot_sync(0xffffffffu, (read & zero) != 0);          // (0, once every lane has its values)
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar + none);
}

struct Place {                                   // of the ring: a stage, and the parity of its use
  uint32_t stage, phase;
  __device__ __forceinline__ void next(uint32_t count) {
    if (++stage == count) stage = 0, phase ^= 1;
  }
};

}  // namespace lsp
