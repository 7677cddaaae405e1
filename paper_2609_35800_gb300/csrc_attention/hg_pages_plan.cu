// Page tables, slots and positions of a batch's new tokens from the requests' lengths.
//
// Request r has ceil(cached / P) pages and needs ceil((cached + new) / P); the difference is taken from the end of the
// free list behind which the pages of requests that end are put first.  Three running sums over the requests (new tokens,
// pages taken, pages given back) give every token's row, every new page's place in the list and every page's place behind
// it; each token, page and place is then found by a search in its sum, one after the other by any thread.  A few bytes a
// request and eight a token: nothing but latency, so one CTA does it all in one launch, the sums in shared memory.
#include "hg_attention.h"
#include "hg_mma.cuh"

namespace hg {
namespace {

constexpr int kThreads = 1024;
constexpr unsigned kAll = 0xffffffffu;

struct Sums {
  int64_t tokens, taken, freed;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return {a.tokens + b.tokens, a.taken + b.taken, a.freed + b.freed};
}

// What request r wants of the call.
struct Wish {
  int cached, tokens, have, taken, freed;
  bool outgrows;
};
__device__ __forceinline__ Wish wish_of(const PagesPlanParams& p, int r) {
  const int mask = (1 << p.page_shift) - 1, given = p.new_tokens[r];
  Wish w;
  w.cached = max(p.cached[r], 0);
  const int64_t after = (int64_t)w.cached + max(given, 0), want = (after + mask) >> p.page_shift;
  w.have = (int)(((int64_t)w.cached + mask) >> p.page_shift);
  w.tokens = max(given, 0);
  w.freed = w.taken = 0;
  w.outgrows = given >= 0 && (want > p.table_stride || after > INT32_MAX);
  if (given < 0) w.freed = min(w.have, p.table_stride);
  else w.taken = (int)(want - w.have);
  return w;
}

// The last r with sums[r] <= x, sums not decreasing from 0.
__device__ __forceinline__ int find(const int* sums, int n, int x) {
  int r = 0;
  while (n > 1) {
    const int half = n / 2;
    if (sums[r + half] <= x) {
      r += half;
      n -= half;
    } else {
      n = half;
    }
  }
  return r;
}

__global__ void __launch_bounds__(kThreads) pages_plan_kernel(const __grid_constant__ PagesPlanParams p) {
  extern __shared__ int sums[];
  __shared__ Sums warp_sums[kThreads / 32];
  __shared__ int flags[2];  // some request outgrows its row; the longest length
  grid_launch_dependents();
  grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  int *tokens_to = sums, *taken_to = sums + p.batch + 1, *freed_to = taken_to + p.batch + 1;
  if (tid < 2) flags[tid] = 0;
  const int per = (p.batch + kThreads - 1) / kThreads, r0 = min(tid * per, p.batch), r1 = min(r0 + per, p.batch);
  Sums mine = {0, 0, 0};
  bool outgrows = false;
  int longest = 0, held = 0;  // after the call; before it
  for (int r = r0; r < r1; ++r) {
    const Wish w = wish_of(p, r);
    mine = mine + Sums{w.tokens, w.taken, w.freed};
    outgrows |= w.outgrows;
    held = max(held, w.cached);
    if (p.new_tokens[r] >= 0) longest = max(longest, w.cached + (w.outgrows ? 0 : w.tokens));
  }
  Sums before = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums x = {__shfl_up_sync(kAll, before.tokens, o), __shfl_up_sync(kAll, before.taken, o),
                    __shfl_up_sync(kAll, before.freed, o)};
    if (lane >= o) before = before + x;
  }
  if (lane == 31) warp_sums[warp] = before;
  before = {before.tokens - mine.tokens, before.taken - mine.taken, before.freed - mine.freed};
  __syncthreads();
  Sums all = {0, 0, 0};
  for (int i = 0; i < kThreads / 32; ++i) {
    if (i == warp) before = before + all;
    all = all + warp_sums[i];
  }
  // a refused call's sums are not used: they may pass 32 bits
  for (int r = r0; r < r1; ++r) {
    const Wish w = wish_of(p, r);
    tokens_to[r] = (int)before.tokens;
    taken_to[r] = (int)before.taken;
    freed_to[r] = (int)before.freed;
    before = before + Sums{w.tokens, w.taken, w.freed};
  }
  if (outgrows) atomicOr(&flags[0], 1);
  const int count = min(max(*p.free_count, 0), p.free_capacity);
  const int64_t left = count + all.freed - all.taken;
  __syncthreads();
  const int refused = flags[0] ? -1 : all.tokens > p.tokens ? -2 : left < 0 ? (int)min(-left, (int64_t)INT32_MAX)
                                                                : left > p.free_capacity ? -3 : 0;
  atomicMax(&flags[1], refused ? held : longest);
  const int tokens = refused ? 0 : (int)all.tokens, taken = refused ? 0 : (int)all.taken, freed = (int)all.freed;
  // a page of the list's end, of those given back by their number
  const auto given_back = [&](int j) {
    const int r = find(freed_to, p.batch, j);
    return p.table[(int64_t)r * p.table_stride + j - freed_to[r]];
  };
  const auto page_taken = [&](int k) { return k < freed ? given_back(freed - 1 - k) : p.free_pages[count - 1 - (k - freed)]; };

  for (int k = tid; k < taken; k += kThreads) {
    const int r = find(taken_to, p.batch, k);
    p.table[(int64_t)r * p.table_stride + wish_of(p, r).have + k - taken_to[r]] = page_taken(k);
  }
  for (int i = tid; i < p.tokens; i += kThreads) {
    int slot = -1, position = 0;
    if (i < tokens) {
      const int r = find(tokens_to, p.batch, i);
      const Wish w = wish_of(p, r);
      position = w.cached + i - tokens_to[r];
      const int at = position >> p.page_shift;
      const int page = at < w.have ? p.table[(int64_t)r * p.table_stride + at] : page_taken(taken_to[r] + at - w.have);
      slot = (int)((uint32_t)page << p.page_shift) + (position & ((1 << p.page_shift) - 1));
    }
    p.slots[i] = slot;
    if (p.positions) p.positions[i] = position;
  }
  if (!refused)
    for (int j = tid; j < (int)left - count; j += kThreads) p.free_pages[count + j] = given_back(j);
  for (int r = r0; r < r1; ++r) p.begin[r] = refused ? 0 : tokens_to[r];
  __syncthreads();  // cached and free_count may be lengths and counts
  for (int r = r0; r < r1; ++r) {
    const Wish w = wish_of(p, r);
    p.lengths[r] = refused ? p.cached[r] : p.new_tokens[r] < 0 ? 0 : w.cached + w.tokens;
  }
  if (tid == 0) {
    p.begin[p.batch] = tokens;
    p.counts[HG_PLAN_FREE] = refused ? count : (int)left;
    p.counts[HG_PLAN_REFUSED] = refused;
    p.counts[HG_PLAN_TOKENS] = tokens;
    p.counts[HG_PLAN_LONGEST] = flags[1];
  }
}

}  // namespace

cudaError_t launch_pages_plan(const PagesPlanParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};  // devices whose shared-memory limit is raised
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(pages_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * (kPlanMaxBatch + 1) * 4);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_overlapped(pages_plan_kernel, dim3(1), kThreads, 3 * (p.batch + 1) * 4, s, p);
}

}  // namespace hg
