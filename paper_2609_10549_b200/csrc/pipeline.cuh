// Bounded waits of the 8-bit products and the weight gradients: what their kernels' roles share.
#pragma once

#include "internal.h"
#include "ptx_sm100.cuh"

namespace compass {

enum PipelineSite : int { SITE_EMPTY = 1, SITE_FULL = 2, SITE_ACC_EMPTY = 3, SITE_ACC_FULL = 4, SITE_DRAIN = 5, SITE_SCALES_FULL = 8, SITE_SCALES_EMPTY = 9 };

struct WaitContext {
  StatusBlock* status;
  int* abort;              // of this CTA, in shared memory
  uint32_t limit_us;
};

// Waits for an mbarrier's phase; gives up after the limit, or when another role of this CTA has.  kCluster: for one by which another
// CTA hands over what it wrote.
template <bool kCluster = false>
__device__ __forceinline__ bool wait_phase(uint64_t* bar, uint32_t parity, const WaitContext& w, int site, int tile) {
  auto there = [&] { return kCluster ? ptx::mbar_try_wait_cluster(bar, parity) : ptx::mbar_try_wait(bar, parity); };
  if (there()) return true;
  const uint64_t t0 = ptx::globaltimer_ns();
  const uint64_t limit = uint64_t(w.limit_us) * 1000ull;
  for (uint32_t spins = 1; spins < (1u << 30); ++spins) {
    if (there()) return true;
    if ((spins & 0xFF) == 0) {
      if (*reinterpret_cast<volatile int*>(w.abort)) return false;
      if (ptx::globaltimer_ns() - t0 > limit) break;
    }
  }
  *reinterpret_cast<volatile int*>(w.abort) = 1;
  if (atomicCAS(&w.status->code, 0, int(COMPASS_ERR_TIMEOUT)) == 0) {
    w.status->detail = site;
    w.status->block_idx = int(blockIdx.x);
    w.status->tile = tile;
  }
  return false;
}

// The same for a whole warp, which goes on or gives up as one.
template <bool kCluster = false>
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, const WaitContext& w, int site, int tile) {
  return __all_sync(0xffffffffu, wait_phase<kCluster>(bar, parity, w, site, tile));
}

// After giving up: copies or products in flight, whatever the others do, before this CTA's memory may go (100 ms at most).
__device__ __forceinline__ void wait_settled(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = ptx::globaltimer_ns();
  for (uint32_t spins = 1; spins < (1u << 30) && !ptx::mbar_try_wait(bar, parity); ++spins)
    if ((spins & 0xFF) == 0 && ptx::globaltimer_ns() - t0 > 100000000ull) break;
}

}  // namespace compass
