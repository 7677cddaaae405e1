// The paged decodes' division of work (division.inc: the header's own text) on the CPU: a CTA's threads are fibers that run
// from one barrier to the next in an order of the caller's.
#include <ucontext.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <memory>
#include <vector>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;

namespace {

struct Index {
  int x;
};
Index threadIdx, blockIdx, gridDim;

enum Wait { kRuns, kAtWarp, kAtBlock, kDone };
struct Fiber {
  ucontext_t context;
  std::vector<char> stack;
  Wait wait;
};
std::vector<std::unique_ptr<Fiber>> fibers;
ucontext_t scheduler;
int slots[1024];  // what the threads show to their warps or to all

void pause(Wait w) {
  const int me = threadIdx.x;
  fibers[me]->wait = w;
  swapcontext(&fibers[me]->context, &scheduler);
}
void __syncthreads() { pause(kAtBlock); }
int shown(int from, int value) {
  slots[threadIdx.x] = value;
  pause(kAtWarp);
  const int x = slots[from];
  pause(kAtWarp);
  return x;
}
int __shfl_up_sync(unsigned, int value, int by) {
  const int lane = threadIdx.x % 32;
  return shown(lane >= by ? threadIdx.x - by : threadIdx.x, value);
}
template <class F>
int over_warp(int value, F f) {
  slots[threadIdx.x] = value;
  pause(kAtWarp);
  int x = value;
  for (int i = threadIdx.x / 32 * 32, n = i + 32; i < n; ++i) x = f(x, slots[i]);
  pause(kAtWarp);
  return x;
}
int __reduce_max_sync(unsigned, int value) {
  return over_warp(value, [](int a, int b) { return max(a, b); });
}
int __reduce_min_sync(unsigned, int value) {
  return over_warp(value, [](int a, int b) { return min(a, b); });
}
void atomicMax(int* at, int value) { *at = max(*at, value); }
constexpr int kDecodeJoinCtas = 16, kDecodeJoinCounters = 128, kHeadDim = 128;

#include "division.inc"

struct Kind {
  static constexpr int kTile = TILE, kConsumers = CONSUMERS, kItemCost = ITEM_COST, kJoinCost = JOIN_COST;
  static int least_share(int group) { return group > 8 ? LEAST_MANY : LEAST_FEW; }
  static constexpr bool kWeighsWhole = WEIGHS_WHOLE;
};
struct Pool {
  int page_shift, heads;
};
struct Params {
  int batch, group, table_stride;
  const int* lengths;
  Pool pool;
};

// A CTA's shared memory: what find_work is given, of the words that the kernels have.
int scan[24], kept[kKeptLengths], room[64 * 16 + kThreads<Kind> + 2];

Params params;
int32_t* result;

void thread_main() {
  const int me = threadIdx.x;
  Work w = {};
  Cursor c = {};
  const int tiles = find_work<Kind>(params, scan, kept, room, w, c);
  // then consumers stage their queries where the room was
  if (me / 32 < Kind::kConsumers)
    for (int i = me; i < (int)(sizeof room / sizeof *room); i += Kind::kConsumers * 32) room[i] = 0;
  const int32_t mine[] = {tiles, c.b, c.h, c.t, w.u0, w.first_unit, w.share, w.ctas};
  std::memcpy(result + 8 * me, mine, sizeof mine);
  threadIdx.x = me;
  pause(kDone);
}

}  // namespace

// Every thread's {tiles, request, head, tile, first unit, its unit of the item, share, CTAs} of CTA `cta` of `ctas`.
// Threads of warp `late` run only when no other can (-1: none).  1: a barrier that not every thread came to.
extern "C" int divide(int batch, int heads, int group, int page_shift, int table_stride, const int32_t* lengths, int ctas,
                      int cta, int late, int32_t* out) {
  params = {batch, group, table_stride, lengths, {page_shift, heads}};
  result = out;
  blockIdx.x = cta;
  gridDim.x = ctas;
  std::fill(scan, scan + 24, 12345);
  std::fill(kept, kept + kKeptLengths, 12345);
  std::fill(std::begin(room), std::end(room), 12345);
  const int n = kThreads<Kind>;
  fibers.clear();
  std::vector<int> order;
  for (int i = 0; i < n; ++i) {
    fibers.push_back(std::make_unique<Fiber>());
    Fiber& f = *fibers.back();
    f.stack.resize(1 << 16);
    f.wait = kRuns;
    getcontext(&f.context);
    f.context.uc_stack.ss_sp = f.stack.data();
    f.context.uc_stack.ss_size = f.stack.size();
    f.context.uc_link = &scheduler;
    makecontext(&f.context, thread_main, 0);
    if (i / 32 != late) order.push_back(i);
  }
  for (int i = 0; i < n; ++i)
    if (i / 32 == late) order.push_back(i);
  const auto release = [&](Wait w, int first, int last) {  // where every thread still there has come to the barrier
    int there = 0;
    for (int i = first; i < last; ++i) {
      if (fibers[i]->wait == kDone) continue;
      if (fibers[i]->wait != w) return false;
      ++there;
    }
    for (int i = first; i < last; ++i)
      if (fibers[i]->wait == w) fibers[i]->wait = kRuns;
    return there > 0;
  };
  for (;;) {
    bool moved = false;
    for (int i : order) {
      if (fibers[i]->wait != kRuns) continue;
      threadIdx.x = i;
      swapcontext(&scheduler, &fibers[i]->context);
      moved = true;
      break;
    }
    for (int w = 0; w < n / 32; ++w) moved |= release(kAtWarp, 32 * w, 32 * w + 32);
    moved |= release(kAtBlock, 0, n);
    if (!moved) break;
  }
  for (const auto& f : fibers)
    if (f->wait != kDone) return 1;
  return 0;
}
