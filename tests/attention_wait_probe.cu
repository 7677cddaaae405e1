// The bounded waits of the 16-bit kernels, run out on purpose: on barriers that nobody completes, with no copy in flight.
#include "hg_wait.cuh"

using namespace hg;

namespace {

// Warp 1 fills a place whose copy never comes (the bytes are expected, no copy is issued) and waits to fill it again;
// warp 0 waits for the copy, gives up, and hands the place on all the same, as the decode's consumers do.  Warps 2 and 3
// wait for something else that does not come either.  result: what each warp's wait said, then the abort flag.
__global__ void ring_kernel(uint32_t* status, int* result) {
  __shared__ __align__(8) uint64_t bars[4];
  __shared__ volatile int abort;
  const uint32_t full = smem_u32(bars), empty = full + 8, never = full + 16;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 3; ++i) mbar_init(full + 8 * i, 1);
    mbar_init_fence();
    abort = 0;
  }
  __syncthreads();
  bool there;
  if (warp == 0) {
    there = wait_warp(full, 0, &abort, status);
    if (lane == 0) mbar_arrive(empty);
  } else if (warp == 1) {
    if (lane == 0) mbar_arrive_expect_tx(full, 128);
    __syncwarp();
    there = wait_to_fill(empty, 0, &abort, status);
  } else if (warp == 2) {
    there = wait_warp<true>(never, 0, &abort, status);
  } else {
    wait_data(never, 0, &abort, status);  // goes on in any case
    there = mbar_try_wait(never, 0);
  }
  if (lane == 0) result[warp] = there;
  __syncthreads();
  drain_phase(full, 0);  // the copy never lands: it has to end all the same
  if (threadIdx.x == 0) result[4] = abort;
}

// Warp 0 waits for warp 1, which takes `ns` and moves what they share all the while, or not.
__global__ void slow_kernel(uint32_t* status, int* result, uint64_t ns, bool moves) {
  __shared__ __align__(8) uint64_t bar;
  __shared__ volatile int abort, progress;
  const uint32_t done = smem_u32(&bar);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    mbar_init(done, 1);
    mbar_init_fence();
    abort = progress = 0;
  }
  __syncthreads();
  if (warp == 0) {
    const bool there = wait_for_others(done, 0, &progress, &abort, status);
    if (lane == 0) result[0] = there;
  } else if (lane == 0) {
    uint64_t begin, now;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(begin));
    for (int i = 0; i < 100000; ++i) {
      __nanosleep(100000);
      if (moves) progress = i + 1;
      asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
      if (now - begin > ns) break;
    }
    mbar_arrive(done);
  }
  __syncthreads();
  if (threadIdx.x == 0) result[1] = abort;
}

}  // namespace

extern "C" int run_slow(uint32_t* status, int* result, uint64_t ns, int moves) {
  slow_kernel<<<1, 64>>>(status, result, ns, moves != 0);
  return (int)cudaGetLastError();
}
extern "C" int run_ring(uint32_t* status, int* result) {
  ring_kernel<<<1, 128>>>(status, result);
  return (int)cudaGetLastError();
}
