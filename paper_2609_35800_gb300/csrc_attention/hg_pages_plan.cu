// Page tables, slots and positions of a batch's new tokens from the requests' lengths.
//
// Request r has ceil(cached / P) pages and needs ceil((cached + new) / P); the difference is taken from the end of the
// free list behind which the pages of requests that end are put first.  Three running sums over the requests (new tokens,
// pages taken, pages given back) give every token's row, every new page's place in the list and every page's place behind
// it; each token, page and place is then found by a search in its sum.  A few bytes a request and eight a token: nothing
// but latency.  Every CTA works out the sums for itself, in shared memory, and takes some of the tokens and pages: what it
// reads for them no other one writes, but for lengths and counts where they are the inputs' own: then a call of up to
// kAlone tokens is one CTA, which writes those last, and a larger one has a second launch that does it.  Measured
// (device): 64 requests of one token, seven that end 4.2 us (7.1 with tokens, new pages and the list's places one after the
// other); 1,000 requests, 484,000 tokens 8.2 us (one CTA 411; 64 tokens a warp 7.6 and 4.8, 128 10.5 and 5.4), most of it
// for the sums and the searches.
#include "hg_attention.h"
#include "hg_mma.cuh"

namespace hg {
namespace {

constexpr int kThreads = 1024;
constexpr int kAlone = 4096;  // tokens that one CTA places where a second launch is the alternative
constexpr unsigned kAll = 0xffffffffu;

// More tokens than a call may have room for, as a sum that stays there; pages stay in 32 bits, as the table's entries do.
constexpr uint32_t kTooMany = 0x7fffffff;
struct Sums {
  uint32_t tokens;
  int taken, freed;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return {min(a.tokens + b.tokens, kTooMany), a.taken + b.taken, a.freed + b.freed};
}
__device__ __forceinline__ Sums from_lane(const Sums& x, int lane) {
  return {__shfl_sync(kAll, x.tokens, lane), __shfl_sync(kAll, x.taken, lane), __shfl_sync(kAll, x.freed, lane)};
}
// The sum of the lanes up to this one.
__device__ __forceinline__ Sums up_to(Sums x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums below = from_lane(x, max(lane - o, 0));
    if (lane >= o) x = x + below;
  }
  return x;
}

// What request r wants of the call.
struct Wish {
  int cached, tokens, have, taken, freed;
  bool outgrows;
};
__device__ __forceinline__ Wish wish_of(const PagesPlanParams& p, int r) {
  const uint32_t mask = (1u << p.page_shift) - 1;
  const int given = p.new_tokens[r];
  Wish w;
  w.cached = max(p.cached[r], 0);
  w.tokens = max(given, 0);
  const uint32_t after = (uint32_t)w.cached + (uint32_t)w.tokens;
  const int want = (int)(after >> p.page_shift) + ((after & mask) != 0 ? 1 : 0);
  w.have = (w.cached >> p.page_shift) + ((w.cached & mask) != 0 ? 1 : 0);
  w.outgrows = given >= 0 && (want > p.table_stride || after > INT32_MAX);
  w.freed = given < 0 ? min(w.have, p.table_stride) : 0;
  w.taken = given >= 0 && !w.outgrows ? want - w.have : 0;
  return w;
}

// The last r of [r, r + n) with sums[r] <= x, sums not decreasing and the first not above x.
__device__ __forceinline__ int find(const int* sums, int r, int n, int x) {
  while (n > 1) {
    const int half = n / 2;
    const bool right = sums[r + half] <= x;
    r += right ? half : 0;
    n = right ? n - half : half;
  }
  return r;
}

__global__ void __launch_bounds__(kThreads) pages_plan_kernel(const __grid_constant__ PagesPlanParams p) {
  extern __shared__ int sums[];
  __shared__ Sums warp_sums[kThreads / 32];
  __shared__ int top;  // the longest length
  grid_launch_dependents();
  grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  int *tokens_to = sums, *taken_to = sums + p.batch + 1, *freed_to = taken_to + p.batch + 1;
  if (tid == 0) top = 0;
  const int count = min(max(*p.free_count, 0), p.free_capacity);
  const int per = (p.batch + kThreads - 1) / kThreads, r0 = min(tid * per, p.batch), r1 = min(r0 + per, p.batch);
  Sums mine = {0, 0, 0};
  bool outgrows = false;
  int longest = 0, held = 0;  // after the call; before it
  for (int r = r0; r < r1; ++r) {
    const Wish w = wish_of(p, r);
    mine = mine + Sums{(uint32_t)w.tokens, w.taken, w.freed};
    outgrows |= w.outgrows;
    held = max(held, w.cached);
    if (p.new_tokens[r] >= 0) longest = max(longest, w.cached + (w.outgrows ? 0 : w.tokens));
  }
  const Sums upto = up_to(mine, lane);
  if (lane == 31) warp_sums[warp] = upto;
  const bool outgrown = __syncthreads_or(outgrows) != 0;
  if (warp == 0) {  // a lane a warp
    const Sums x = up_to(lane < kThreads / 32 ? warp_sums[lane] : Sums{0, 0, 0}, lane);
    if (lane < kThreads / 32) warp_sums[lane] = x;
  }
  Sums before = from_lane(upto, max(lane - 1, 0));
  if (lane == 0) before = {0, 0, 0};
  __syncthreads();
  const Sums all = warp_sums[kThreads / 32 - 1];
  if (warp > 0) before = before + warp_sums[warp - 1];
  for (int r = r0; r < r1; ++r) {
    const Wish w = wish_of(p, r);
    tokens_to[r] = (int)before.tokens;
    taken_to[r] = before.taken;
    freed_to[r] = before.freed;
    before = before + Sums{(uint32_t)w.tokens, w.taken, w.freed};
  }
  const int64_t left = (int64_t)count + all.freed - all.taken;
  const int refused = outgrown ? -1 : all.tokens > (uint32_t)p.tokens ? -2 : left < 0 ? (int)-left
                                                                              : left > p.free_capacity ? -3 : 0;
  __syncthreads();
  if (blockIdx.x == 0) {
    longest = __reduce_max_sync(kAll, refused ? held : longest);
    if (lane == 0) atomicMax(&top, longest);
  }
  const int tokens = refused ? 0 : (int)all.tokens, taken = refused ? 0 : all.taken, freed = all.freed;
  // a page of the list's end, of those given back by their number
  const auto given_back = [&](int j) {
    const int r = find(freed_to, 0, p.batch, j);
    return p.table[(int64_t)r * p.table_stride + j - freed_to[r]];
  };
  const auto page_taken = [&](int k) { return k < freed ? given_back(freed - 1 - k) : p.free_pages[count - 1 - (k - freed)]; };

  if (p.part != kPlanEnd) {
    // a warp takes 32 tokens, pages taken or places of the list at a time, one kind beside the other
    const int back = refused ? 0 : max((int)left - count, 0);
    const int token_units = (p.tokens + 31) / 32, page_units = (taken + 31) / 32;
    const int units = token_units + page_units + (back + 31) / 32, step = gridDim.x * (kThreads / 32);
    for (int u = blockIdx.x * (kThreads / 32) + warp; u < units; u += step) {
      if (u >= token_units + page_units) {
        const int j = (u - token_units - page_units) * 32 + lane;
        if (j < back) p.free_pages[count + j] = given_back(j);
        continue;
      }
      if (u >= token_units) {
        const int k = (u - token_units) * 32 + lane;
        if (k >= taken) continue;
        const int r = find(taken_to, 0, p.batch, k);
        p.table[(int64_t)r * p.table_stride + wish_of(p, r).have + k - taken_to[r]] = page_taken(k);
        continue;
      }
      const int i = u * 32 + lane;
      int slot = -1, position = 0;
      if (i < tokens) {
        // the warp's first token's request, and how far it is to the last one's
        const int least = find(tokens_to, 0, p.batch, u * 32), last = min(u * 32 + 31, tokens - 1);
        int requests = 1;
        while (least + requests < p.batch && tokens_to[least + requests] <= last) requests *= 2;
        const int r = find(tokens_to, least, min(requests, p.batch - least), i);
        const int cached = max(p.cached[r], 0), mask = (1 << p.page_shift) - 1;
        position = cached + i - tokens_to[r];
        const int at = position >> p.page_shift, have = (cached >> p.page_shift) + ((cached & mask) != 0 ? 1 : 0);
        const int page = at < have ? p.table[(int64_t)r * p.table_stride + at] : page_taken(taken_to[r] + at - have);
        slot = (int)((uint32_t)page << p.page_shift) + (position & mask);
      }
      if (i < p.tokens) {
        p.slots[i] = slot;
        if (p.positions) p.positions[i] = position;
      }
    }
    if (blockIdx.x == 0) {
      for (int r = r0; r < r1; ++r) p.begin[r] = refused ? 0 : tokens_to[r];
      if (tid == 0) p.begin[p.batch] = tokens;
    }
  }
  if (p.part == kPlanFill || blockIdx.x > 0) return;
  __syncthreads();  // cached and free_count may be lengths and counts
  for (int r = r0; r < r1; ++r) {
    const Wish w = wish_of(p, r);
    p.lengths[r] = refused ? p.cached[r] : p.new_tokens[r] < 0 ? 0 : w.cached + w.tokens;
  }
  if (tid == 0) {
    p.counts[HG_PLAN_FREE] = refused ? count : (int)left;
    p.counts[HG_PLAN_REFUSED] = refused;
    p.counts[HG_PLAN_TOKENS] = tokens;
    p.counts[HG_PLAN_LONGEST] = top;
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
  const int smem = 3 * (p.batch + 1) * 4;
  const int ctas = p.in_place && p.tokens <= kAlone ? 1 : std::min((p.tokens + kThreads - 1) / kThreads, device_sms());
  PagesPlanParams a = p;
  a.part = ctas > 1 && p.in_place ? kPlanFill : kPlanAll;
  e = launch_overlapped(pages_plan_kernel, dim3((unsigned)std::max(ctas, 1)), kThreads, smem, s, a);
  if (e != cudaSuccess || a.part == kPlanAll) return e;
  a.part = kPlanEnd;
  return launch_overlapped(pages_plan_kernel, dim3(1), kThreads, smem, s, a);
}

}  // namespace hg
