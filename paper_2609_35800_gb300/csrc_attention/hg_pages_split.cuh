// The paged decode kernels' division of work and what becomes of its parts: an even share of a launch's tiles for every
// CTA whatever the requests' lengths, parts of an item joined by the last CTA to arrive, results written.  What a tile
// holds, and how it is computed, is the kernels' own.  P: their launch parameters.  K:
//   kTile         tokens of a tile
//   kItemCost     an item's fixed costs, in tiles
//   kJoinCost     a ticket and a join, in tiles
//   least_share   units that a CTA gets where there are fewer than that for each
//   kTwoLevels    parts for each of the groups of threads that share a query's, from which on they are joined 16 CTAs at a
//                 time first
//   kWeighsWhole  whether the fullest CTA counts, not the longest item alone
//   kConsumers    warps, ahead of the producer's
//   kF16          the rows' type
//   kUnlift       1 / the factor that probabilities are lifted by
//   kUnits        whether a query's sums are in a unit of their own, a power of two
//   result        what an output entry becomes before it is rounded
//   place         a fragment's two channels into a row of sums
#pragma once
#include "hg_rows.cuh"
#include "hg_wait.cuh"

namespace hg {
namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kKeptLengths = 72;
constexpr int kJoinCtas = kDecodeJoinCtas, kJoinCounters = kDecodeJoinCounters;
constexpr int kSumFloats = kHeadDim + 4;  // a query's sums in shared memory: 128 channels, m, l, unit; rows 4 banks apart

template <class K>
constexpr int kThreads = (K::kConsumers + 1) * 32;
template <class K>
constexpr int kGroups = K::kConsumers * 4;  // of eight threads

// Where a run of tiles stands.
struct Cursor {
  int b, h, t;     // request, KV head, tile of its item
  int len, tiles;  // of request b
};

template <class P>
__device__ __forceinline__ int request_length(const P& p, int b) {
  return min(max(p.lengths[b], 0), p.table_stride << p.pool.page_shift);
}
// A request without a token counts as a tile too: its zeros have to be written.
template <class K>
__device__ __forceinline__ int tiles_of(int len) {
  return max(1, (len + K::kTile - 1) / K::kTile);
}

template <class K, class P>
__device__ __forceinline__ void next_item(const P& p, const int* kept, Cursor& c) {
  c.t = 0;
  if (++c.h < p.pool.heads) return;
  c.h = 0;
  if (++c.b >= p.batch) return;
  c.len = c.b < kKeptLengths ? kept[c.b] : request_length(p, c.b);
  c.tiles = tiles_of<K>(c.len);
}

// The launch's units, cut into `ctas` runs of `share` units, the first `more` of them one longer; those of this CTA are
// [u0, u1).
struct Work {
  int u0, u1, total, ctas, share, more;
  int first_unit;  // of its item, that u0 is
  __device__ __forceinline__ int start_of(int cta) const { return cta * share + min(cta, more); }
  __device__ __forceinline__ int cta_of(int u) const {
    const int longer = more * (share + 1);
    return u < longer ? u / (share + 1) : more + (u - longer) / share;
  }
};

// Units of the CTA that would get the most if each took the whole items that begin in its run.  Every thread looks for the
// first item at or behind some of the runs' starts, in the requests of the thread whose units hold it.  `room`: words of
// shared memory, kThreads + the CTAs + 2.
template <class K, class P>
__device__ int fullest_of_whole(const P& p, const int* kept, int* room, const Work& w, int units_before) {
  const int tid = threadIdx.x, heads = p.pool.heads, per = (p.batch + kThreads<K> - 1) / kThreads<K>;
  int *ahead = room, *firsts = room + kThreads<K>, *most = firsts + w.ctas + 1;
  ahead[tid] = units_before;
  if (tid == 0) *most = 0;
  __syncthreads();
  for (int j = tid; j <= w.ctas; j += kThreads<K>) {
    const int u = w.start_of(j);
    int at = u;
    if (u < w.total) {
      int t = 0;  // the last thread with requests whose units begin at u or before
      for (int n = min(kThreads<K>, (p.batch + per - 1) / per); n > 1;) {
        const int half = n / 2;
        const bool right = ahead[t + half] <= u;
        t += right ? half : 0;
        n = right ? n - half : half;
      }
      int left = u - ahead[t];
      for (int b = t * per; b < p.batch; ++b) {
        const int units = tiles_of<K>(b < kKeptLengths ? kept[b] : request_length(p, b)) + K::kItemCost;
        if (left < units * heads) {
          const int in_item = left % units;
          at = u + (in_item > 0 ? units - in_item : 0);
          break;
        }
        left -= units * heads;
      }
    }
    firsts[j] = at;
  }
  __syncthreads();
  int mine = 0;
  for (int j = tid; j < w.ctas; j += kThreads<K>) mine = max(mine, firsts[j + 1] - firsts[j]);
  mine = __reduce_max_sync(kAll, mine);
  if (tid % 32 == 0) atomicMax(most, mine);
  __syncthreads();
  const int units = *most;
  __syncthreads();  // every thread has read it: the room is the kernel's again
  return units;
}

// The CTA's work, the first tile of it and how many there are; 0: none.  Every thread adds up the units of its share of
// the requests; the one whose share holds u0 looks for it there.
template <class K, class P>
__device__ int find_work(const P& p, int* scan, int* kept, int* room, Work& w, Cursor& c) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, heads = p.pool.heads;
  const int per = (p.batch + kThreads<K> - 1) / kThreads<K>;
  const int b0 = min(tid * per, p.batch), b1 = min(b0 + per, p.batch);
  int mine = 0, longest = 0, shortest = 0x7fffffff;
  for (int b = b0; b < b1; ++b) {
    const int len = request_length(p, b), units = tiles_of<K>(len) + K::kItemCost;
    if (b < kKeptLengths) kept[b] = len;
    mine += units;
    longest = max(longest, units);
    shortest = min(shortest, units);
  }
  longest = __reduce_max_sync(kAll, longest);
  if (K::kWeighsWhole) shortest = __reduce_min_sync(kAll, shortest);
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kAll, sum, o);
    if (lane >= o) sum += x;
  }
  if (lane == 31) {
    scan[warp] = sum;
    scan[12 + warp] = longest;
    if (K::kWeighsWhole) scan[16 + warp] = shortest;
  }
  __syncthreads();
  int before = sum - mine, all = 0;
#pragma unroll
  for (int i = 0; i < K::kConsumers + 1; ++i) {
    if (i < warp) before += scan[i];
    all += scan[i];
    longest = max(longest, scan[12 + i]);
    if (K::kWeighsWhole) shortest = min(shortest, scan[16 + i]);
  }
  w.total = all * heads;
  const int least = K::least_share(p.group);
  w.ctas = min((int)gridDim.x, (w.total + least - 1) / least);
  if ((int)blockIdx.x >= w.ctas) return 0;
  w.share = w.total / w.ctas;
  w.more = w.total - w.share * w.ctas;
  w.u0 = w.start_of(blockIdx.x);
  w.u1 = w.start_of(blockIdx.x + 1);
  int left = w.u0 - before * heads;
  if (left >= 0 && left < mine * heads) {
    int b = b0, len = 0, units = 0;
    for (;; ++b) {
      len = b < kKeptLengths ? kept[b] : request_length(p, b);
      units = tiles_of<K>(len) + K::kItemCost;
      if (left < units * heads) break;
      left -= units * heads;
    }
    scan[8] = b;
    scan[9] = left / units;
    scan[10] = left - scan[9] * units;
    scan[11] = len;
  }
  __syncthreads();
  w.first_unit = scan[10];
  c = {scan[8], scan[9], max(0, w.first_unit - K::kItemCost), scan[11], tiles_of<K>(scan[11])};
  int tiles = 0;
  bool whole = longest <= w.share + K::kJoinCost;
  // (8-bit pages.)  With no more items than CTAs, a CTA that has more to read than the others is faster while they share the
  // memory with it, up to twice: whole where the fullest CTA gets up to 1.5 shares (4 requests of 2,000 tokens, 32 heads, 2.4
  // shares: 27.6 us whole, 19.4 cut; 32 of 8,577, 8 heads, 1.2 shares: 86 whole, 91 cut).  That is the longest item where no
  // item is shorter than a run, so that none begins in another's; and the fullest CTA gets less than a share and the longest
  // item in any case.  Otherwise, and with more items than CTAs, where some begin a second item when the others end, the
  // fullest one is looked for (16 of 4,000 and 16 of 8,577 in turn, 8 heads: 102 us whole, 71 cut; 40 of 8,577, 8 heads: 156
  // whole, 112 cut), which takes 2 us, more than short items can lose (64 of 500 tokens, 8 heads: 17.3 us whole, 19.3 so).
  if (K::kWeighsWhole) {
    const auto fullest = [&] { return fullest_of_whole<K>(p, kept, room, w, before * heads); };
    if ((int64_t)p.batch * heads <= w.ctas) {
      const int64_t most = 3 * (int64_t)w.share + 2 * K::kJoinCost;
      whole = 2 * (int64_t)longest <= most;
      if (whole && shortest < w.share + (w.more > 0) && 2 * ((int64_t)longest + w.share) > most)
        whole = 2 * (int64_t)fullest() <= most;
    } else if (longest > 2 * K::kJoinCost) {
      whole = whole && fullest() <= w.share + K::kJoinCost;
    } else {
      whole = true;
    }
  }
  if (whole) {
    // from the first item that begins at u0 or later to the last that begins before u1
    int at = w.u0;
    if (w.first_unit > 0) {
      at += c.tiles + K::kItemCost - w.first_unit;
      w.first_unit = 0;
      if (at < w.u1) next_item<K>(p, kept, c);
    }
    w.u0 = at;
    for (Cursor x = c; at < w.u1;) {
      tiles += x.tiles;
      at += x.tiles + K::kItemCost;
      if (at < w.u1) next_item<K>(p, kept, x);
    }
    return tiles;
  }
  // the run's units less those that stand for fixed costs
  int rest = w.u1 - w.u0, skip = max(0, K::kItemCost - w.first_unit);
  for (Cursor x = c; rest > skip; skip = K::kItemCost) {
    rest -= skip;
    const int n = min(rest, x.tiles - x.t);
    tiles += n;
    rest -= n;
    if (rest > 0) next_item<K>(p, kept, x);
  }
  return tiles;
}

// Lets the launch's page ids, queries and rotations into L2 before the caches' reads fill the memory's queues: a request
// by each CTA in turn.
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];\n" ::"l"(p)); }
template <class K, class P>
__device__ void prefetch_queries(const P& p) {
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    const int heads = p.group * p.pool.heads;
    for (int i = 32 * threadIdx.x; i < p.table_stride; i += 32 * kThreads<K>)
      prefetch_l2(p.table + (int64_t)b * p.table_stride + i);
    for (int i = threadIdx.x; i < 2 * heads; i += kThreads<K>)
      prefetch_l2(p.q.data + b * p.q.token_stride + (i / 2) * p.q.head_stride + (i % 2) * 64);
    if (p.rot.table == nullptr) continue;
    for (int i = threadIdx.x; i < 3 * 4; i += kThreads<K>) {
      if (i >= 4 && p.rot.position_stride == 0) break;
      const int pos = min(max(p.rot.positions[(int64_t)(i / 4) * p.rot.position_stride + b], 0), p.rot.table_len - 1);
      if (i % 4 * 32 < 2 * p.rot.half) prefetch_l2(p.rot.table + (int64_t)pos * (2 * p.rot.half) + i % 4 * 32);
    }
  }
}

// An item's query rows on their way: 8 lanes a row, four rows at a time.
template <int NT>
struct Queries {
  uint4 lo[NT][2], hi[NT][2];
  LaneAngles angles;
};

template <int NT, class P>
__device__ __forceinline__ void fetch_queries(const P& p, int b, int h, Queries<NT>& x) {
  const int lane = threadIdx.x % 32, c = lane % 8;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr);
  const uint16_t* row = p.q.data + b * p.q.token_stride + (int64_t)h * p.group * p.q.head_stride;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = nt * 8 + lane / 8 + 4 * i;
      x.lo[nt][i] = x.hi[nt][i] = make_uint4(0u, 0u, 0u, 0u);
      if (q < p.group) {
        x.lo[nt][i] = ldg16(row + q * p.q.head_stride + at.lo);
        x.hi[nt][i] = ldg16(row + q * p.q.head_stride + at.hi);
      }
    }
  if (at.turns) x.angles = lane_angles(p.rot, c, b);
}

// What a consumer warp keeps of its item: queries 8 nt + 2 (lane % 4) and the next one (rows of S^T, columns of O^T).
template <int NT>
struct State {
  float m[NT][2], l[NT][2];  // l: this lane's own tokens
  float o[NT][8][4];         // [query tile][16 channels][fragment]
};

// A CTA's part of the item that begins in its run (`begins`), or of the one that began before it.
template <class P>
__device__ __forceinline__ float* partial_of(const P& p, int cta, bool begins) {
  return p.partials + ((int64_t)cta * 2 + (begins ? 1 : 0)) * p.group * kPartialFloats;
}

// A query's sums, 16 channels of them, in units of u (0: there are none).  The unit is applied once the sums are divided by l:
// times the largest values of a cache they would pass binary32's end, where their average does not.
struct Part {
  float m = -INFINITY, l = 0.f, u = 0.f, o[16] = {};
};
// A row's maximum, sum and unit, as they lie in a part or behind a row of sums in shared memory.
template <class K>
__device__ __forceinline__ float3 load_mlu(const float* at) {
  if (K::kUnits) {
    const float4 x = *reinterpret_cast<const float4*>(at);
    return make_float3(x.x, x.y, x.z);
  }
  const float2 x = *reinterpret_cast<const float2*>(at);
  return make_float3(x.x, x.y, 0.f);
}
template <class K>
__device__ __forceinline__ float3 load_mlu_l2(const float* at) {
  if (K::kUnits) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(at));
    return make_float3(x.x, x.y, x.z);
  }
  const float2 x = __ldcg(reinterpret_cast<const float2*>(at));
  return make_float3(x.x, x.y, 0.f);
}
template <class K>
__device__ __forceinline__ void store_mlu(float* at, float m, float l, float u) {
  if (K::kUnits) *reinterpret_cast<float4*>(at) = make_float4(m, l, u, 0.f);
  else *reinterpret_cast<float2*>(at) = make_float2(m, l);
}
// What sums in units of u are multiplied by to be in units of `to`, not below it; powers of two, or 0.
__device__ __forceinline__ float units_in(float u, float to) {
  return u * __uint_as_float((uint32_t)(254 - (int)(__float_as_uint(to) >> 23)) << 23);
}
// Adds up N rows of sums in shared memory, `apart` floats from one to the next: one maximum, then independent terms.
template <class K, int N>
__device__ __forceinline__ Part add_rows(const float* row, int apart, int count, int channel, float cs) {
  Part a;
  float3 mlu[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    mlu[i] = i < count ? load_mlu<K>(row + i * apart + kHeadDim) : make_float3(-INFINITY, 0.f, 0.f);
    a.m = fmaxf(a.m, mlu[i].x);
    a.u = fmaxf(a.u, mlu[i].z);
  }
  const float base = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i >= count) break;
    float e = exp2_approx((mlu[i].x - base) * cs);
    a.l += mlu[i].y * e;
    if (K::kUnits) e *= units_in(mlu[i].z, a.u);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(row + i * apart + channel + 4 * k);
      a.o[4 * k] += x.x * e;
      a.o[4 * k + 1] += x.y * e;
      a.o[4 * k + 2] += x.z * e;
      a.o[4 * k + 3] += x.w * e;
    }
  }
  return a;
}
template <class K>
__device__ __forceinline__ void store_part(const Part& a, float* channels, float* ml, int channel) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4*>(channels + channel + 4 * i) =
        make_float4(a.o[4 * i], a.o[4 * i + 1], a.o[4 * i + 2], a.o[4 * i + 3]);
  if (channel == 0) store_mlu<K>(ml, a.m, a.l, a.u);
}

// out = o / l in the cache's type, and the query's log-sum-exp (o and l are lifted alike).
template <class K, class P>
__device__ __forceinline__ void write_query(const P& p, int b, int h, int len, int q, int channel,
                                            const Part& a) {
  const float r = len > 0 ? 1.0f / a.l : 0.f, u = K::kUnits ? a.u : 1.f;
  const int head = h * p.group + q;
  uint16_t* out = p.out.data + b * p.out.token_stride + head * p.out.head_stride + channel;
  uint32_t x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = pack2<K::kF16>(K::result(a.o[2 * i] * r * u), K::result(a.o[2 * i + 1] * r * u));
  *reinterpret_cast<uint4*>(out) = make_uint4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<uint4*>(out + 8) = make_uint4(x[4], x[5], x[6], x[7]);
  if (p.lse && channel == 0)
    p.lse[(int64_t)b * p.pool.heads * p.group + head] = a.l == 0.f ? -INFINITY : a.m * p.scale + logf(a.l * K::kUnlift);
}

// Takes a number; what the CTA's threads wrote before their last barrier is visible to whoever takes a later one.
__device__ __forceinline__ uint32_t take_ticket(uint32_t* counter) {
  uint32_t n;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;\n" : "=r"(n) : "l"(counter) : "memory");
  return n;
}

// The CTA's part of an item over the CTAs [cta0, cta1] is written: whoever comes last joins them.  (Inlined: called, it
// cost launches of 10 to 30 us up to 5%.)
template <class K, class P>
__device__ __forceinline__ void join_item(const P& p, int b, int h, int len, int cta0, int cta1, float* scratch,
                                       volatile int* misc, float cs) {
  const int lane = threadIdx.x % 32, mine = threadIdx.x / 8, channel = 16 * (threadIdx.x % 8);
  // up to six queries: several groups of threads share a query's parts, each takes every `subs`-th
  const int subs = max(1, kGroups<K> / p.group);
  const bool two_levels = cta1 - cta0 >= (subs > 1 ? K::kTwoLevels : 24) * subs;
  for (int level = two_levels ? 0 : 1; level < 2; ++level) {
    // the parts of this level: CTA `first` (level 1 of two: then the first CTA of each further 16), `stride` apart
    const int round = blockIdx.x & ~(kJoinCtas - 1);
    const int first = level == 0 ? max(cta0, round) : cta0, stride = two_levels && level == 1 ? kJoinCtas : 1;
    const int count = level == 0 ? min(cta1, round + kJoinCtas - 1) - first + 1
                                 : two_levels ? cta1 / kJoinCtas - cta0 / kJoinCtas + 1 : cta1 - cta0 + 1;
    const auto part = [&](int k) {
      const int cta = k == 0 ? first : stride == 1 ? first + k : (first & ~(kJoinCtas - 1)) + k * stride;
      return partial_of(p, cta, cta == cta0);
    };
    if (count > 1) {
      if (threadIdx.x == 0) {
        uint32_t* counter = level == 0 ? p.counters + blockIdx.x / kJoinCtas * 2 + (cta0 >= round)
                                       : p.counters + kJoinCounters + (int64_t)b * p.pool.heads + h;
        const bool last = take_ticket(counter) == (uint32_t)(count - 1);
        if (last) *counter = 0u;
        misc[1] = last;
      }
      named_barrier<K::kConsumers * 32>(1);
      if (!misc[1]) return;
    }
    const int sub = mine / p.group, lane8 = lane % 8;
    const unsigned group_mask = 0xffu << (lane & 24);
    for (int q = subs > 1 ? mine % p.group : mine; q < p.group && (subs == 1 || sub < subs); q += kGroups<K>) {
      Part a;
#pragma unroll 1
      for (int k0 = subs > 1 ? sub : 0; k0 < count; k0 += 8 * subs) {
        // eight parts at a time: a lane has one's m and l, all lanes 16 channels of each, of four at once
        const int k = k0 + lane8 * subs;
        float3 mlu = make_float3(-INFINITY, 0.f, 0.f);
        if (k < count) mlu = load_mlu_l2<K>(part(k) + q * kPartialFloats);
        float e = 0.f;
#pragma unroll
        for (int j0 = 0; j0 < 8; j0 += 4) {
          float4 o[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int kj = k0 + (j0 + j) * subs;
            const float* row = part(kj) + q * kPartialFloats + 4 + channel;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              o[j][i] = kj < count ? __ldcg(reinterpret_cast<const float4*>(row + 4 * i)) : make_float4(0.f, 0.f, 0.f, 0.f);
          }
          if (j0 == 0) {
            float top = fmaxf(a.m, mlu.x);
#pragma unroll
            for (int i = 1; i < 8; i <<= 1) top = fmaxf(top, __shfl_xor_sync(group_mask, top, i));
            const float base = top == -INFINITY ? 0.f : top;
            float keep = exp2_approx((a.m - base) * cs);
            e = exp2_approx((mlu.x - base) * cs);
            float l = mlu.y * e;
#pragma unroll
            for (int i = 1; i < 8; i <<= 1) l += __shfl_xor_sync(group_mask, l, i);
            a.m = top;
            a.l = a.l * keep + l;
            if (K::kUnits) {
              float to = fmaxf(a.u, mlu.z);
#pragma unroll
              for (int i = 1; i < 8; i <<= 1) to = fmaxf(to, __shfl_xor_sync(group_mask, to, i));
              keep *= units_in(a.u, to);
              e *= units_in(mlu.z, to);
              a.u = to;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) a.o[i] *= keep;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float ej = __shfl_sync(group_mask, e, (lane & 24) + j0 + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              a.o[4 * i] += o[j][i].x * ej;
              a.o[4 * i + 1] += o[j][i].y * ej;
              a.o[4 * i + 2] += o[j][i].z * ej;
              a.o[4 * i + 3] += o[j][i].w * ej;
            }
          }
          if (k0 + 4 * subs >= count) break;
        }
      }
      if (subs > 1) {  // then this is the only round
        float* row = scratch + (sub * p.group + q) * kSumFloats;
        store_part<K>(a, row, row + kHeadDim, channel);
      } else if (level == 1) {
        write_query<K>(p, b, h, len, q, channel, a);
      } else {
        float* row = part(0) + q * kPartialFloats;
        store_part<K>(a, row + 4, row, channel);
      }
    }
    if (subs > 1) {
      named_barrier<K::kConsumers * 32>(1);
      if (mine < p.group) {
        const Part a = add_rows<K, kGroups<K>>(scratch + mine * kSumFloats, p.group * kSumFloats, subs, channel, cs);
        if (level == 1) {
          write_query<K>(p, b, h, len, mine, channel, a);
        } else {
          float* row = part(0) + mine * kPartialFloats;
          store_part<K>(a, row + 4, row, channel);
        }
      }
    }
    named_barrier<K::kConsumers * 32>(1);  // the scratch is free again; the joined part is written
  }
}

// The end of the CTA's part of an item: the warps' sums are added up, 8 queries at a time, 8 threads to a query; a whole
// item is written, a part goes to the workspace, and the last part's CTA joins them all.  unit: of the warp's sums.
template <class K, int NT, class P>
__device__ void finish_item(const P& p, State<NT>& st, const Cursor& c, bool whole, bool begins, int tile_u0,
                            const Work& w, float* scratch, volatile int* misc, float cs, float unit) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, tq = lane % 4;
  const int mine = threadIdx.x / 8, channel = 16 * (threadIdx.x % 8);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 4; i < 32; i <<= 1) st.l[nt][j] += __shfl_xor_sync(kAll, st.l[nt][j], i);
    if (nt > 0) named_barrier<K::kConsumers * 32>(1);  // the first queries' sums are read
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float* row = scratch + (warp * 8 + 2 * tq + j) * kSumFloats;
#pragma unroll
      for (int d = 0; d < 8; ++d) K::place(row + 16 * d, g, st.o[nt][d][j], st.o[nt][d][2 + j]);
      if (g == 0) {  // (as one store of four words it spills: 16 bytes with 16 queries)
        *reinterpret_cast<float2*>(row + kHeadDim) = make_float2(st.m[nt][j], st.l[nt][j]);
        if (K::kUnits) row[kHeadDim + 2] = unit;
      }
    }
    named_barrier<K::kConsumers * 32>(1);
    const int q = 8 * nt + mine;
    if (mine < 8 && q < p.group) {
      const Part a = add_rows<K, K::kConsumers>(scratch + mine * kSumFloats, 8 * kSumFloats, K::kConsumers, channel, cs);
      if (whole) {
        write_query<K>(p, c.b, c.h, c.len, q, channel, a);
      } else {
        float* row = partial_of(p, blockIdx.x, begins) + q * kPartialFloats;
        store_part<K>(a, row + 4, row, channel);
      }
    }
  }
  named_barrier<K::kConsumers * 32>(1);  // the scratch is free again; the part is written
  if (whole) return;
  join_item<K>(p, c.b, c.h, c.len, w.cta_of(tile_u0), w.cta_of(tile_u0 + c.tiles - 1), scratch, misc, cs);
}

}  // namespace
}  // namespace hg
