// Attention of one new token per request over a paged cache, split over the cache's length and joined.
//
// For a request, KV head and its G queries: s_t = scale q.k_t, m = max s_t, out = sum e^(s_t - m) v_t / sum e^(s_t - m).
// Every key and value is used by G <= 16 queries only, G flop per byte, so the kernel is bound by the reads of the cache;
// it has to keep enough of them in flight and to spread them evenly.  Measured: 32 requests x 8,577 tokens x 8 KV heads
// 171 us, 6.60 TB/s, 0.97 of a copy's rate; one request of 131,073 tokens 88 us (0.90); 37 of 1 to 9,001 tokens and 12
// queries a KV head 29 us (0.53; start and tail); 321 tokens 7.5 us.
//
// The work is cut into tiles of 32 tokens of one (request, KV head), numbered request by request, head by head; each
// such item counts as kItemCost tiles more, ahead of its first, for its queries, sums and result (19 shapes, geometric
// mean: 15.2 us at 4 tiles, 15.0 at 8, 14.9 at 12 and 16).  A CTA takes an even share of the units, whatever the
// requests' lengths, which the kernel reads on the device.  Its run cuts at most two items, the first and the last; it
// leaves their (m, l, o) in the workspace, and the last CTA to arrive at an item (a ticket, no waiting) joins its parts
// in a fixed order, so the result does not depend on who comes last.  The parts of an item over many CTAs are joined 16
// CTAs at a time first (one KV head, 131,072 tokens: 79 -> 23 us).  Where no item is more than kJoinCost units longer
// than the share, a CTA takes the whole items that begin in its units, as a join costs more than a few units (321 tokens:
// 8.9 us cut, 7.5 whole).  That bounds the longest item, not what a CTA gets, up to a share and an item: 40 requests of
// 8,577 tokens and 8 KV heads, 320 items on 304 CTAs, take 278 us, where 32 of them, cut, take 172 and 64 take 328.
//
// A producer warp copies tiles into a ring of six 16 KB stages with TMA, a box per page (swizzled rows; a page id
// outside the pool reads as zeros).  Three consumer warps take the tiles in turn, each with its own running maximum and
// sums, so that three tiles' chains of load, product, maximum, exponential and product run side by side, about 950
// cycles each (four warps on 16 tokens each of one 64-token tile took 1,200 cycles a tile).  Two of the stages belong to
// each warp: it waits for every phase of their barriers, in order, as a wait by parity needs.  They compute with mma.sync
// m16n8k16 (a tcgen05 product would have M = 128 tokens by N = 8 queries and its probabilities would pass through tensor
// memory; the tensor pipe is 7% busy):
//   S^T[token][query] = K . q        A = keys (ldmatrix), B = the queries, padded to 8 or 16
//   O^T[channel][query] += V^T . P^T A = values (ldmatrix.trans), B = P^T (movmatrix of the scores' fragment)
// Scores, maxima, sums and outputs are held in 32 bits; probabilities are rounded to the cache's type for the second
// product only, lifted in FP16 (kLift).  The running maximum moves when a score passes it by more than 2^8.
#include "hg_rows.cuh"
#include "hg_wait.cuh"

namespace hg {
namespace {

constexpr int kTile = kDecodeTile, kTileShift = 5;
static_assert(kTile == 1 << kTileShift, "tile");
constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kTile * kHeadDim * 2;  // keys, then values
constexpr int kConsumers = 3;
constexpr int kThreads = (kConsumers + 1) * 32;
static_assert(kStages % kConsumers == 0, "a stage belongs to one warp");
constexpr int kQRowBytes = 272;  // a staged query row: 256 bytes, 16 more so that ldmatrix meets every bank once
constexpr int kGroups = kConsumers * 4;  // of eight threads
constexpr unsigned kAll = 0xffffffffu;

constexpr int kItemCost = kDecodeItemCost;
constexpr int kJoinCost = 24;  // a ticket and a join, in tiles
constexpr int kKeptLengths = 72;
constexpr int kJoinCtas = kDecodeJoinCtas, kJoinCounters = kDecodeJoinCounters;
constexpr int kSumFloats = kHeadDim + 4;  // a query's sums in shared memory: 128 channels, m, l; rows 4 banks apart

// Shared memory, two CTAs an SM.  The staged queries (8 rows a warp) and the warps' parts that are added up at an item's
// end (8 queries at a time) take turns in one region.
struct Smem {
  static constexpr int scratch = kStages * kStageBytes;
  static constexpr int scratch_bytes = kConsumers * 8 * kSumFloats * 4;
  static constexpr int bars = scratch + scratch_bytes;
  static constexpr int misc = bars + 2 * kStages * 8;  // abort flag, last part, start of the CTA's work, scan
  static constexpr int lengths = misc + 128;           // the first requests' lengths
  static constexpr int bytes = lengths + 4 * kKeptLengths;
};
static_assert(Smem::scratch_bytes >= kConsumers * 8 * kQRowBytes, "queries are staged there too");
static_assert((8 + 12 + kConsumers + 1) * 4 <= Smem::lengths - Smem::misc, "the scan's words");
static_assert(2 * (Smem::bytes + 1024) <= 228 * 1024, "two CTAs an SM");

// Where a run of tiles stands.
struct Cursor {
  int b, h, t;     // request, KV head, tile of its item
  int len, tiles;  // of request b
};

__device__ __forceinline__ int request_length(const PagesDecodeParams& p, int b) {
  return min(max(p.lengths[b], 0), p.table_stride << p.pool.page_shift);
}
// A request without a token counts as a tile too: its zeros have to be written.
__device__ __forceinline__ int tiles_of(int len) { return max(1, (len + kTile - 1) / kTile); }

__device__ __forceinline__ void next_item(const PagesDecodeParams& p, const int* kept, Cursor& c) {
  c.t = 0;
  if (++c.h < p.pool.heads) return;
  c.h = 0;
  if (++c.b >= p.batch) return;
  c.len = c.b < kKeptLengths ? kept[c.b] : request_length(p, c.b);
  c.tiles = tiles_of(c.len);
}

__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, int row, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], "
      "[%6];\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(head), "r"(page), "r"(bar)
      : "memory");
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

// The CTA's work, the first tile of it and how many there are; 0: none.  Every thread adds up the units of its share of
// the requests; the one whose share holds u0 looks for it there.
__device__ int find_work(const PagesDecodeParams& p, int* scan, int* kept, Work& w, Cursor& c) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, heads = p.pool.heads;
  const int per = (p.batch + kThreads - 1) / kThreads;
  const int b0 = min(tid * per, p.batch), b1 = min(b0 + per, p.batch);
  int mine = 0, longest = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = request_length(p, b), units = tiles_of(len) + kItemCost;
    if (b < kKeptLengths) kept[b] = len;
    mine += units;
    longest = max(longest, units);
  }
  longest = __reduce_max_sync(kAll, longest);
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kAll, sum, o);
    if (lane >= o) sum += x;
  }
  if (lane == 31) {
    scan[warp] = sum;
    scan[12 + warp] = longest;
  }
  __syncthreads();
  int before = sum - mine, all = 0;
#pragma unroll
  for (int i = 0; i < kConsumers + 1; ++i) {
    if (i < warp) before += scan[i];
    all += scan[i];
    longest = max(longest, scan[12 + i]);
  }
  w.total = all * heads;
  w.ctas = min((int)gridDim.x, w.total);
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
      units = tiles_of(len) + kItemCost;
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
  c = {scan[8], scan[9], max(0, w.first_unit - kItemCost), scan[11], tiles_of(scan[11])};
  int tiles = 0;
  if (longest <= w.share + kJoinCost) {
    // from the first item that begins at u0 or later to the last that begins before u1
    int at = w.u0;
    if (w.first_unit > 0) {
      at += c.tiles + kItemCost - w.first_unit;
      w.first_unit = 0;
      if (at < w.u1) next_item(p, kept, c);
    }
    w.u0 = at;
    for (Cursor x = c; at < w.u1;) {
      tiles += x.tiles;
      at += x.tiles + kItemCost;
      if (at < w.u1) next_item(p, kept, x);
    }
    return tiles;
  }
  // the run's units less those that stand for fixed costs
  int rest = w.u1 - w.u0, skip = max(0, kItemCost - w.first_unit);
  for (Cursor x = c; rest > skip; skip = kItemCost) {
    rest -= skip;
    const int n = min(rest, x.tiles - x.t);
    tiles += n;
    rest -= n;
    if (rest > 0) next_item(p, kept, x);
  }
  return tiles;
}

// Lets the launch's page ids, queries and rotations into L2 before the caches' reads fill the memory's queues: a request
// by each CTA in turn.
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];\n" ::"l"(p)); }
__device__ void prefetch_queries(const PagesDecodeParams& p) {
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    const int heads = p.group * p.pool.heads;
    for (int i = 32 * threadIdx.x; i < p.table_stride; i += 32 * kThreads)
      prefetch_l2(p.table + (int64_t)b * p.table_stride + i);
    for (int i = threadIdx.x; i < 2 * heads; i += kThreads)
      prefetch_l2(p.q.data + b * p.q.token_stride + (i / 2) * p.q.head_stride + (i % 2) * 64);
    if (p.rot.table == nullptr) continue;
    for (int i = threadIdx.x; i < 3 * 4; i += kThreads) {
      if (i >= 4 && p.rot.position_stride == 0) break;
      const int pos = min(max(p.rot.positions[(int64_t)(i / 4) * p.rot.position_stride + b], 0), p.rot.table_len - 1);
      if (i % 4 * 32 < 2 * p.rot.half) prefetch_l2(p.rot.table + (int64_t)pos * (2 * p.rot.half) + i % 4 * 32);
    }
  }
}

// Copies the CTA's tiles into the ring, in order; returns how many it asked for.
__device__ uint32_t produce(const PagesDecodeParams& p, Cursor c, int tiles, const int* kept, uint32_t stages, uint32_t full,
                            uint32_t empty, volatile int* abort) {
  const int lane = threadIdx.x % 32;
  const int shift = min(p.pool.page_shift, kTileShift), rows = 1 << shift;  // tokens of a box
  const int boxes = kTile >> shift;
  const uint32_t box_bytes = (uint32_t)rows * kHeadDim * 2;
  uint32_t n = 0;
  // 32 boxes' page ids, a lane each, from box `first` of request `of` on
  int of = -1, first = 0, id = 0;
  for (; tiles > 0; next_item(p, kept, c)) {
    const int* ids = p.table + (int64_t)c.b * p.table_stride;
    for (; c.t < c.tiles && tiles > 0; ++c.t, --tiles, ++n) {
      const int box0 = c.t * boxes;  // box number in the item
      const int valid = min(boxes, max(0, (c.len - c.t * kTile + rows - 1) >> shift));
      if (of != c.b || box0 < first || box0 + boxes > first + 32) {
        of = c.b;
        first = box0;
        const int64_t token = (int64_t)(first + lane) * rows;
        id = token < c.len ? ids[token >> p.pool.page_shift] : -1;
      }
      const int s = n % kStages;
      if (n >= kStages && !wait_warp(empty + 8 * s, (n / kStages - 1) & 1, abort, p.status)) return n;
      if (elect_one()) mbar_arrive_expect_tx(full + 8 * s, 2 * valid * box_bytes);
      for (int i = 0; i < valid; ++i) {
        const int page = __shfl_sync(kAll, id, box0 - first + i);
        const int row = ((box0 + i) << shift) & (p.pool.page_size - 1);
        const uint32_t dst = stages + s * kStageBytes + i * box_bytes;
        if (elect_one()) {  // (lanes that issue side by side take turns, one copy after the other)
          tma_page(dst, &p.k_map, row, c.h, page, full + 8 * s);
          tma_page(dst + kStageBytes / 2, &p.v_map, row, c.h, page, full + 8 * s);
        }
      }
    }
  }
  return n;
}

// What a consumer warp keeps of its item: queries 8 nt + 2 (lane % 4) and the next one (rows of S^T, columns of O^T).
template <int NT>
struct State {
  float m[NT][2], l[NT][2];  // l: this lane's own tokens
  float o[NT][8][4];         // [query tile][16 channels][fragment]
};

template <bool F16>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (F16) mma_f16(d, a, b0, b1);
  else mma_bf16(d, a, b0, b1);
}

// An item's query rows on their way: 8 lanes a row, four rows at a time.
template <int NT>
struct Queries {
  uint4 lo[NT][2], hi[NT][2];
  LaneAngles angles;
};

template <int NT>
__device__ __forceinline__ void fetch_queries(const PagesDecodeParams& p, int b, int h, Queries<NT>& x) {
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

// Rotated, and through shared memory into the first product's operands.
template <bool F16, int NT>
__device__ __forceinline__ void stage_queries(const PagesDecodeParams& p, Queries<NT>& x, uint32_t mine,
                                              uint32_t (&qf)[NT][16]) {
  const int lane = threadIdx.x % 32;
  const LaneChannels at = lane_channels(p.rot, lane % 8, p.rot.table != nullptr);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (at.turns) rotate_lane<F16>(x.lo[nt][i], x.hi[nt][i], x.angles, p.rot.interleaved != 0);
      const uint32_t row = mine + (lane / 8 + 4 * i) * kQRowBytes;
      st_shared16(row + at.lo * 2, x.lo[nt][i]);
      st_shared16(row + at.hi * 2, x.hi[nt][i]);
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // 32 channels: two k-steps of two 8-channel halves
      uint32_t f[4];
      ldsm_x4(f, mine + (lane % 8) * kQRowBytes + (4 * j + lane / 8) * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) qf[nt][4 * j + i] = f[i];
    }
    __syncwarp();
  }
}

// 16-byte chunk of a tile's row: boxes of `rows` (16 or 32) rows, first halves before second halves.
__device__ __forceinline__ uint32_t tile_chunk(uint32_t tile, int rows, int r, int chunk) {
  const int box = r & ~(rows - 1);
  return tile + box * kHeadDim * 2 + (chunk / 8) * rows * 128 + swizzled(r - box, chunk % 8);
}

// The new token of a decode step: into its page, and over row r of the stage's tile (which may hold what was there).  Not
// where the request has grown past its table: its new token has no place there, and the last row is a token's own.
template <bool F16>
__device__ __forceinline__ void place_new_token(const PagesDecodeParams& p, const Cursor& c, uint32_t kt, uint32_t vt, int rows,
                                                int r) {
  const int lane = threadIdx.x % 32;
  if (lane < 16) {
    const int i = lane % 8;
    const bool is_v = lane >= 8;
    const Rows& in = is_v ? p.v : p.k;
    const LaneChannels at = lane_channels(p.rot, i, p.rot.table != nullptr && !is_v);
    const uint16_t* src = in.data + c.b * in.token_stride + c.h * in.head_stride;
    const int given = p.lengths[c.b], last = c.len - 1;
    uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
    if (at.turns) rotate_lane<F16>(lo, hi, lane_angles(p.rot, i, c.b), p.rot.interleaved != 0);
    if (given == c.len) {
      st_shared16(tile_chunk(is_v ? vt : kt, rows, r, at.lo / 8), lo);
      st_shared16(tile_chunk(is_v ? vt : kt, rows, r, at.hi / 8), hi);
      const int page = p.table[(int64_t)c.b * p.table_stride + (last >> p.pool.page_shift)];
      if (page >= 0 && page < p.pool.num_pages) {
        uint16_t* dst = (is_v ? p.pool.v : p.pool.k) + page_row(p.pool, page, last & (p.pool.page_size - 1), c.h);
        *reinterpret_cast<uint4*>(dst + at.lo) = lo;
        *reinterpret_cast<uint4*>(dst + at.hi) = hi;
      }
    }
  }
  __syncwarp();
}

// A tile of 32 tokens, of which the first `seen` belong to the request.
template <bool F16, int NT>
__device__ __forceinline__ void attend_tile(State<NT>& st, const uint32_t (&qf)[NT][16], uint32_t kt, uint32_t vt, int rows,
                                            int seen, float c) {
  const int lane = threadIdx.x % 32;
  float s[2][NT][4], s2[2][NT][4];  // [16 tokens][query tile]; a chain of products for each half of the channels
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[mt][nt][i] = s2[mt][nt][i] = 0.f;
  // rows are 16 (a page's 16 tokens a box) or 32: token 16 mt + r lies in box mt, row r, or in the box's row 16 mt + r
  const uint32_t second = rows == 16 ? 16 * kHeadDim * 2 : 16 * 128, half = rows * 128;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      uint32_t a[4], a2[4];
      const uint32_t at = kt + mt * second + swizzled(lane % 16, 2 * ks + lane / 16);
      ldsm_x4(a, at);
      ldsm_x4(a2, at + half);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma16<F16>(s[mt][nt], a, qf[nt][2 * ks], qf[nt][2 * ks + 1]);
        mma16<F16>(s2[mt][nt], a2, qf[nt][8 + 2 * ks], qf[nt][8 + 2 * ks + 1]);
      }
    }
  }
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[mt][nt][i] += s2[mt][nt][i];
  const int g = lane / 4;
  uint32_t pf[2][NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (seen < kTile) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * mt + g + 8 * (i / 2) >= seen) s[mt][nt][i] = -INFINITY;
    }
    float top[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) top[j] = fmaxf(fmaxf(s[0][nt][j], s[0][nt][2 + j]), fmaxf(s[1][nt][j], s[1][nt][2 + j]));
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      top[0] = fmaxf(top[0], __shfl_xor_sync(kAll, top[0], o));
      top[1] = fmaxf(top[1], __shfl_xor_sync(kAll, top[1], o));
    }
    // a first maximum, or one far past the old: the sums so far count that much less (the same in all lanes of a column)
    const bool moved = (top[0] - st.m[nt][0]) * c > kRescale || (top[1] - st.m[nt][1]) * c > kRescale;
    if (__any_sync(kAll, moved)) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float m = fmaxf(st.m[nt][j], top[j]);
        const float keep = m == st.m[nt][j] ? 1.f : exp2_approx((st.m[nt][j] - m) * c);
        st.m[nt][j] = m;
        st.l[nt][j] *= keep;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          st.o[nt][d][j] *= keep;
          st.o[nt][d][2 + j] *= keep;
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float m = st.m[nt][i % 2];
        s[mt][nt][i] = exp2_approx(fmaf(s[mt][nt][i] - (m == -INFINITY ? 0.f : m), c, kLift<F16>));
        st.l[nt][i % 2] += s[mt][nt][i];
      }
      pf[mt][nt][0] = movtrans(pack2<F16>(s[mt][nt][0], s[mt][nt][1]));
      pf[mt][nt][1] = movtrans(pack2<F16>(s[mt][nt][2], s[mt][nt][3]));
    }
  }
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      uint32_t a[4];
      ldsm_x4_trans(a, vt + mt * second + (d / 4) * half + swizzled(lane % 8 + 8 * (lane / 16), 2 * (d % 4) + lane / 8 % 2));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma16<F16>(st.o[nt][d], a, pf[mt][nt][0], pf[mt][nt][1]);
    }
}

// A CTA's part of the item that begins in its run (`begins`), or of the one that began before it.
__device__ __forceinline__ float* partial_of(const PagesDecodeParams& p, int cta, bool begins) {
  return p.partials + ((int64_t)cta * 2 + (begins ? 1 : 0)) * p.group * kPartialFloats;
}

// A query's sums, 16 channels of them.
struct Part {
  float m = -INFINITY, l = 0.f, o[16] = {};
};
// Adds up N rows of sums in shared memory, `apart` floats from one to the next: one maximum, then independent terms.
template <int N>
__device__ __forceinline__ Part add_rows(const float* row, int apart, int count, int channel, float cs) {
  Part a;
  float2 ml[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    ml[i] = i < count ? *reinterpret_cast<const float2*>(row + i * apart + kHeadDim) : make_float2(-INFINITY, 0.f);
    a.m = fmaxf(a.m, ml[i].x);
  }
  const float base = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i >= count) break;
    const float e = exp2_approx((ml[i].x - base) * cs);
    a.l += ml[i].y * e;
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
__device__ __forceinline__ void store_part(const Part& a, float* channels, float* ml, int channel) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4*>(channels + channel + 4 * i) =
        make_float4(a.o[4 * i], a.o[4 * i + 1], a.o[4 * i + 2], a.o[4 * i + 3]);
  if (channel == 0) *reinterpret_cast<float2*>(ml) = make_float2(a.m, a.l);
}

// out = o / l in the cache's type, and the query's log-sum-exp (o and l are lifted alike).
template <bool F16>
__device__ __forceinline__ void write_query(const PagesDecodeParams& p, int b, int h, int len, int q, int channel,
                                            const Part& a) {
  const float r = len > 0 ? 1.0f / a.l : 0.f;
  const int head = h * p.group + q;
  uint16_t* out = p.out.data + b * p.out.token_stride + head * p.out.head_stride + channel;
  uint32_t x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = pack2<F16>(a.o[2 * i] * r, a.o[2 * i + 1] * r);
  *reinterpret_cast<uint4*>(out) = make_uint4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<uint4*>(out + 8) = make_uint4(x[4], x[5], x[6], x[7]);
  if (p.lse && channel == 0)
    p.lse[(int64_t)b * p.pool.heads * p.group + head] = a.l == 0.f ? -INFINITY : a.m * p.scale + logf(a.l * (F16 ? 0x1p-7f : 1.f));
}

// Takes a number; what the CTA's threads wrote before their last barrier is visible to whoever takes a later one.
__device__ __forceinline__ uint32_t take_ticket(uint32_t* counter) {
  uint32_t n;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;\n" : "=r"(n) : "l"(counter) : "memory");
  return n;
}

// The CTA's part of an item over the CTAs [cta0, cta1] is written: whoever comes last joins them.  (Inlined: called, it
// cost launches of 10 to 30 us up to 5%.)
template <bool F16>
__device__ __forceinline__ void join_item(const PagesDecodeParams& p, int b, int h, int len, int cta0, int cta1, float* scratch,
                                       volatile int* misc, float cs) {
  const int lane = threadIdx.x % 32, mine = threadIdx.x / 8, channel = 16 * (threadIdx.x % 8);
  // up to six queries: several groups of threads share a query's parts, each takes every `subs`-th
  const int subs = max(1, kGroups / p.group);
  const bool two_levels = cta1 - cta0 >= 24 * subs;
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
      named_barrier<kConsumers * 32>(1);
      if (!misc[1]) return;
    }
    const int sub = mine / p.group, lane8 = lane % 8;
    const unsigned group_mask = 0xffu << (lane & 24);
    for (int q = subs > 1 ? mine % p.group : mine; q < p.group && (subs == 1 || sub < subs); q += kGroups) {
      Part a;
#pragma unroll 1
      for (int k0 = subs > 1 ? sub : 0; k0 < count; k0 += 8 * subs) {
        // eight parts at a time: a lane has one's m and l, all lanes 16 channels of each, of four at once
        const int k = k0 + lane8 * subs;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (k < count) ml = __ldcg(reinterpret_cast<const float2*>(part(k) + q * kPartialFloats));
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
            float top = fmaxf(a.m, ml.x);
#pragma unroll
            for (int i = 1; i < 8; i <<= 1) top = fmaxf(top, __shfl_xor_sync(group_mask, top, i));
            const float base = top == -INFINITY ? 0.f : top;
            const float keep = exp2_approx((a.m - base) * cs);
            e = exp2_approx((ml.x - base) * cs);
            float l = ml.y * e;
#pragma unroll
            for (int i = 1; i < 8; i <<= 1) l += __shfl_xor_sync(group_mask, l, i);
            a.m = top;
            a.l = a.l * keep + l;
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
        store_part(a, row, row + kHeadDim, channel);
      } else if (level == 1) {
        write_query<F16>(p, b, h, len, q, channel, a);
      } else {
        float* row = part(0) + q * kPartialFloats;
        store_part(a, row + 4, row, channel);
      }
    }
    if (subs > 1) {
      named_barrier<kConsumers * 32>(1);
      if (mine < p.group) {
        const Part a = add_rows<kGroups>(scratch + mine * kSumFloats, p.group * kSumFloats, subs, channel, cs);
        if (level == 1) {
          write_query<F16>(p, b, h, len, mine, channel, a);
        } else {
          float* row = part(0) + mine * kPartialFloats;
          store_part(a, row + 4, row, channel);
        }
      }
    }
    named_barrier<kConsumers * 32>(1);  // the scratch is free again; the joined part is written
  }
}

// The end of the CTA's part of an item: the warps' sums are added up, 8 queries at a time, 8 threads to a query; a whole
// item is written, a part goes to the workspace, and the last part's CTA joins them all.
template <bool F16, int NT>
__device__ void finish_item(const PagesDecodeParams& p, State<NT>& st, const Cursor& c, bool whole, bool begins, int tile_u0,
                            const Work& w, float* scratch, volatile int* misc, float cs) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, tq = lane % 4;
  const int mine = threadIdx.x / 8, channel = 16 * (threadIdx.x % 8);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 4; i < 32; i <<= 1) st.l[nt][j] += __shfl_xor_sync(kAll, st.l[nt][j], i);
    if (nt > 0) named_barrier<kConsumers * 32>(1);  // the first queries' sums are read
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float* row = scratch + (warp * 8 + 2 * tq + j) * kSumFloats;
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        row[16 * d + g] = st.o[nt][d][j];
        row[16 * d + 8 + g] = st.o[nt][d][2 + j];
      }
      if (g == 0) *reinterpret_cast<float2*>(row + kHeadDim) = make_float2(st.m[nt][j], st.l[nt][j]);
    }
    named_barrier<kConsumers * 32>(1);
    const int q = 8 * nt + mine;
    if (mine < 8 && q < p.group) {
      const Part a = add_rows<kConsumers>(scratch + mine * kSumFloats, 8 * kSumFloats, kConsumers, channel, cs);
      if (whole) {
        write_query<F16>(p, c.b, c.h, c.len, q, channel, a);
      } else {
        float* row = partial_of(p, blockIdx.x, begins) + q * kPartialFloats;
        store_part(a, row + 4, row, channel);
      }
    }
  }
  named_barrier<kConsumers * 32>(1);  // the scratch is free again; the part is written
  if (whole) return;
  join_item<F16>(p, c.b, c.h, c.len, w.cta_of(tile_u0), w.cta_of(tile_u0 + c.tiles - 1), scratch, misc, cs);
}

template <bool F16, int NT>
__device__ void consume(const PagesDecodeParams& p, Cursor c, const Work& w, int tiles, uint32_t base, char* smem,
                        volatile int* misc) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = base + Smem::bars, empty = full + 8 * kStages;
  const int rows = min(p.pool.page_size, kTile);
  const float cs = p.scale * kLog2e;
  float* scratch = reinterpret_cast<float*>(smem + Smem::scratch);
  const int* kept = reinterpret_cast<const int*>(smem + Smem::lengths);
  uint32_t n = 0;
  bool alive = true;  // false: a wait ran out, and the warp only keeps up with the others' barriers
  // unit of the first item's first tile
  int tile_u0 = w.u0 - w.first_unit + kItemCost;
  Queries<NT> queries;
  if (NT == 1) fetch_queries<NT>(p, c.b, c.h, queries);
  while (tiles > 0) {
    if (NT > 1) fetch_queries<NT>(p, c.b, c.h, queries);
    const bool begins = c.t == 0, whole = begins && c.tiles <= tiles;
    uint32_t qf[NT][16];
    stage_queries<F16, NT>(p, queries, base + Smem::scratch + warp * 8 * kQRowBytes, qf);
    State<NT> st;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      st.m[nt][0] = st.m[nt][1] = -INFINITY;
      st.l[nt][0] = st.l[nt][1] = 0.f;
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[nt][d][i] = 0.f;
    }
    for (; c.t < c.tiles && tiles > 0; ++c.t, --tiles, ++n) {
      if (n % kConsumers != warp) continue;
      const int s = n % kStages;
      alive = alive && wait_warp(full + 8 * s, (n / kStages) & 1, misc, p.status);
      const uint32_t kt = base + s * kStageBytes, vt = kt + kStageBytes / 2;
      const int seen = c.len - c.t * kTile;
      __syncwarp();
      if (alive && seen > 0) {
        if (seen < kTile) {
          // what follows the request's last token may be anything, and 0 times NaN is no 0
          for (int i = seen * 16 + lane; i < kTile * 16; i += 32)
            st_shared16(tile_chunk(vt, rows, i / 16, i % 16), make_uint4(0u, 0u, 0u, 0u));
        }
        if (seen <= kTile && p.store) place_new_token<F16>(p, c, kt, vt, rows, seen - 1);
        __syncwarp();
        attend_tile<F16, NT>(st, qf, kt, vt, rows, seen, cs);
        if (seen <= kTile) fence_proxy_async_shared();  // TMA writes the stage again
      }
      __syncwarp();
      // (not after a wait that ran out: the stage would be filled over a copy whose bytes are still expected)
      if (alive && lane == 0) mbar_arrive(empty + 8 * s);
    }
    const Cursor done = c;
    if (tiles > 0) {  // the next item's queries come in meanwhile
      next_item(p, kept, c);
      if (NT == 1) fetch_queries<NT>(p, c.b, c.h, queries);  // (of 16 queries they would take the sums' registers)
    }
    named_barrier<kConsumers * 32>(1);  // every warp has read its queries from the scratch
    finish_item<F16, NT>(p, st, done, whole, begins, tile_u0, w, scratch, misc, cs);
    tile_u0 += done.tiles + kItemCost;
  }
}

template <bool F16, int NT>
__global__ void __launch_bounds__(kThreads, 2) pages_decode_kernel(const __grid_constant__ PagesDecodeParams p) {
  extern __shared__ __align__(1024) char smem[];
  const uint32_t base = smem_u32(smem), full = base + Smem::bars, empty = full + 8 * kStages;
  volatile int* misc = reinterpret_cast<int*>(smem + Smem::misc);  // [0] abort, [1] last part, [8 ..] scan
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    mbar_init_fence();
    misc[0] = 0;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    prefetch_tensormap(&p.k_map);
    prefetch_tensormap(&p.v_map);
  }
  grid_launch_dependents();
  grid_dependency_wait();
  prefetch_queries(p);
  Work w;
  Cursor c;
  int* kept = reinterpret_cast<int*>(smem + Smem::lengths);
  const int tiles = find_work(p, const_cast<int*>(misc) + 8, kept, w, c);
  if (tiles == 0) return;
  uint32_t asked = 0;
  if (threadIdx.x / 32 == kConsumers) {
    fence_proxy_async_global();  // pages written by ordinary stores of earlier launches
    asked = produce(p, c, tiles, kept, base, full, empty, misc);
  } else {
    consume<F16, NT>(p, c, w, tiles, base, smem, misc);
  }
  __syncthreads();
  if (misc[0]) {  // a CTA that gave up leaves once the copies it asked for have landed
    for (uint32_t n = asked > kStages ? asked - kStages : 0; n < asked; ++n)
      drain_phase(full + 8 * (n % kStages), (n / kStages) & 1);
  }
}

template <bool F16, int NT>
cudaError_t launch(const PagesDecodeParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};  // devices whose shared-memory limit is raised
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(pages_decode_kernel<F16, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem::bytes);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_overlapped(pages_decode_kernel<F16, NT>, dim3((unsigned)decode_ctas()), kThreads, Smem::bytes, s, p);
}

}  // namespace

cudaError_t launch_pages_decode(const PagesDecodeParams& p, bool f16, cudaStream_t s) {
  if (p.group <= 8) return f16 ? launch<true, 1>(p, s) : launch<false, 1>(p, s);
  return f16 ? launch<true, 2>(p, s) : launch<false, 2>(p, s);
}

}  // namespace hg
