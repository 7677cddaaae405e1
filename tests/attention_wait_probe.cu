// The bounded waits of the 16-bit kernels, run out on purpose: on barriers that nobody completes, with no copy in flight.
#include "hg_tcgen05.cuh"

using namespace hg;

namespace {

// Warp 1 fills a place whose copy never comes (the bytes are expected, no copy is issued) and waits to fill it again;
// warp 0 waits for the copy, gives up, and hands the place on all the same, as a warp does that goes on.  Warps 2 and 3
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

// A wait that runs out; products issued all the same (128 x 128 x 16 `steps` times over operands of ones, one after the
// other); the drain, and then tensor memory is read and freed.  result: whether the wait was met, whether the products had ended when
// the drain returned, and how many of the 128 x 128 sums are right.
constexpr int kOperandBytes = 128 * 128;
__global__ void products_kernel(uint32_t* status, int* result, int steps) {
  extern __shared__ char raw[];
  __shared__ __align__(8) uint64_t bars[2];
  __shared__ volatile int abort;
  __shared__ int address;
  const uint32_t base = (smem_u32(raw) + 1023) & ~1023u, never = smem_u32(bars), ended = never + 8;
  const int warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    mbar_init(never, 1);
    mbar_init(ended, 1);
    mbar_init_fence();
    abort = 0;
  }
  for (int i = threadIdx.x; i < 2 * kOperandBytes / 16; i += blockDim.x)
    st_shared16(base + 16 * i, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));  // BF16 ones
  fence_proxy_async_shared();
  if (warp == 0) tmem_alloc(smem_u32(&address), 128);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)address;
  if (warp == 0) {
    const bool there = wait_warp(never, 0, &abort, status);
    if (elect_one()) {
      const uint32_t a = smem_operand(base, 16), b = smem_operand(base + kOperandBytes, 16), shape = mma_shape(false, 128, false);
      for (int i = 0; i < steps; ++i) tc_mma_ss(tmem, a, b, shape, i > 0);
    }
    __syncwarp();
    if (elect_one()) tc_commit(ended);
    __syncwarp();
    drain_phase(ended, 0);
    if (threadIdx.x == 0) {
      result[0] = there;
      result[1] = mbar_try_wait(ended, 0);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  int right = 0;
  for (int i = 0; i < 4; ++i) {
    uint32_t d[32];
    tmem_load32(d, tmem + ((uint32_t)(warp * 32) << 16) + 32 * i);
    tmem_wait_loads();
    for (int k = 0; k < 32; ++k) right += __uint_as_float(d[k]) == 16.f * steps;
  }
  atomicAdd(result + 2, right);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_free(tmem, 128);
  }
}

}  // namespace

extern "C" int run_products(uint32_t* status, int* result, int steps) {
  constexpr int bytes = 2 * kOperandBytes + 1024;
  products_kernel<<<1, 128, bytes>>>(status, result, steps);
  return (int)cudaGetLastError();
}
extern "C" int run_slow(uint32_t* status, int* result, uint64_t ns, int moves) {
  slow_kernel<<<1, 64>>>(status, result, ns, moves != 0);
  return (int)cudaGetLastError();
}
extern "C" int run_ring(uint32_t* status, int* result) {
  ring_kernel<<<1, 128>>>(status, result);
  return (int)cudaGetLastError();
}
