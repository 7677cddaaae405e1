// Bounded waits and shared-memory addresses of the asynchronous kernels.
#pragma once
#include "hg_mma.cuh"

namespace hg {

constexpr uint32_t kWaitTimeoutBit = 1;    // status word: a wait ran out
constexpr uint32_t kAsyncRounds = 1 << 18;  // rounds of 3.8 us each as measured, whatever longer time is asked for: a second
constexpr uint32_t kAsyncSleepNs = 50000;

// Wait for a phase of `bar`.  One that runs out flags the workspace's status word and *abort, by which every other
// wait of the CTA ends too, and returns false.  This one is suspended from the start: for a warp that is ahead of the
// others, whose questions would only be in their way (prompt attention's loads, 1,541 -> 1,562 TFLOP/s).
__device__ __forceinline__ bool wait_asleep(uint32_t bar, uint32_t parity, volatile int* abort, uint32_t* status) {
  for (uint32_t i = 0; i < kAsyncRounds; ++i) {
    if (mbar_try_wait_sleep(bar, parity, kAsyncSleepNs)) return true;
    if (*abort) return false;
  }
  *abort = 1;
  atomicOr(status, kWaitTimeoutBit);
  return false;
}

// The same for those that others wait for: two plain questions, which the hardware holds back for a while, then
// suspensions.  (Long prompts: 64 questions before the first suspension 5% slower, none 12%.)
__device__ __forceinline__ bool wait_phase_briefly(uint32_t bar, uint32_t parity) {
  return mbar_try_wait(bar, parity) || mbar_try_wait(bar, parity);
}
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, volatile int* abort, uint32_t* status) {
  return wait_phase_briefly(bar, parity) || wait_asleep(bar, parity, abort, status);
}

// The wait of a whole warp, which stays together: all of its threads go on, or none.
template <bool ASLEEP = false>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort, uint32_t* status) {
  return __all_sync(0xffffffffu, ASLEEP ? wait_asleep(bar, parity, abort, status) : wait_phase(bar, parity, abort, status));
}

// The wait of a warp that fills the place it waited for.  A warp that gave up on a copy may have handed the place on all
// the same, and one more arrival on a barrier whose bytes are still expected is an error: nothing is filled once *abort
// is set (which it was before the place was handed on).
template <bool ASLEEP = false>
__device__ __forceinline__ bool wait_to_fill(uint32_t bar, uint32_t parity, volatile int* abort, uint32_t* status) {
  const bool there = ASLEEP ? wait_asleep(bar, parity, abort, status) : wait_phase(bar, parity, abort, status);
  return __all_sync(0xffffffffu, there && !*abort);
}

// The wait of a whole warp that may have nothing to do for as long as others have: it runs out once *progress, which they
// move, has stood still for as long as a wait lasts.
__device__ __forceinline__ bool wait_for_others(uint32_t bar, uint32_t parity, volatile int* progress, volatile int* abort,
                                                uint32_t* status) {
  bool there = wait_phase_briefly(bar, parity);
  for (uint32_t i = 0, last = *progress; !there; ++i) {
    there = mbar_try_wait_sleep(bar, parity, kAsyncSleepNs);
    const uint32_t now = *progress;
    if (now != last) i = 0;
    last = now;
    if (there || *abort) break;
    if (i >= kAsyncRounds) {
      *abort = 1;
      atomicOr(status, kWaitTimeoutBit);
      break;
    }
  }
  return __all_sync(0xffffffffu, there);
}

// The same as wait_warp where a vote would lengthen a chain of products and softmax (by 1.5%): the warp goes on in any
// case, over whatever is there, and finds *abort at its next wait_warp.  For data that no address is made from.
__device__ __forceinline__ void wait_data(uint32_t bar, uint32_t parity, volatile int* abort, uint32_t* status) {
  wait_phase(bar, parity, abort, status);
  __syncwarp();
}

// For a CTA that gave up: until the copies that complete this phase have landed, or a second has passed.
__device__ __forceinline__ void drain_phase(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kAsyncRounds && !mbar_try_wait_sleep(bar, parity, kAsyncSleepNs); ++i) {
  }
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory");
}

template <int THREADS>
__device__ __forceinline__ void named_barrier(int id) {
  asm volatile("bar.sync %0, %1;\n" ::"r"(id), "n"(THREADS) : "memory");
}

// Byte offset of 16-byte chunk `chunk` of row r in rows of 128 bytes under the 128-byte swizzle (base 1024-aligned).
__device__ __forceinline__ uint32_t swizzled(int r, int chunk) { return (uint32_t)(r * 128 + ((chunk ^ (r & 7)) << 4)); }

__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace hg
