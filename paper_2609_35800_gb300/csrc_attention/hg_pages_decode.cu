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
#include "hg_pages_split.cuh"

namespace hg {
namespace {

constexpr int kStages = 6;
constexpr int kTile = kDecodeTile, kTileShift = 5;
static_assert(kTile == 1 << kTileShift, "tile");
constexpr int kConsumers = 3, kItemCost = kDecodeItemCost;
constexpr int kJoinCost = 24;  // a ticket and a join, in tiles
static_assert(kStages % kConsumers == 0, "a stage belongs to one warp");
constexpr int kStageBytes = 2 * kTile * kHeadDim * 2;  // keys, then values
constexpr int kQRowBytes = 272;  // a staged query row: 256 bytes, 16 more so that ldmatrix meets every bank once

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

__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, int row, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], "
      "[%6];\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(head), "r"(page), "r"(bar)
      : "memory");
}

template <bool F16>
struct Kind {
  static constexpr int kTile = hg::kTile, kConsumers = hg::kConsumers, kItemCost = hg::kItemCost, kJoinCost = hg::kJoinCost;
  static __device__ __forceinline__ int least_share(int) { return 1; }
  static constexpr int kTwoLevels = 24;
  static constexpr bool kWeighsWhole = false;
  static constexpr bool kF16 = F16;
  static constexpr float kUnlift = F16 ? 0x1p-7f : 1.f;
  static constexpr bool kUnits = false;
  static __device__ __forceinline__ float result(float x) { return x; }
  static __device__ __forceinline__ void place(float* row, int g, float first, float second) {
    row[g] = first;
    row[8 + g] = second;
  }
};

// Copies the CTA's tiles into the ring, in order; returns how many it asked for.
template <class K>
__device__ uint32_t produce(const PagesDecodeParams& p, Cursor c, int tiles, const int* kept, uint32_t stages, uint32_t full,
                            uint32_t empty, volatile int* abort) {
  const int lane = threadIdx.x % 32;
  const int shift = min(p.pool.page_shift, kTileShift), rows = 1 << shift;  // tokens of a box
  const int boxes = kTile >> shift;
  const uint32_t box_bytes = (uint32_t)rows * kHeadDim * 2;
  uint32_t n = 0;
  // 32 boxes' page ids, a lane each, from box `first` of request `of` on
  int of = -1, first = 0, id = 0;
  for (; tiles > 0; next_item<K>(p, kept, c)) {
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

template <bool F16>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (F16) mma_f16(d, a, b0, b1);
  else mma_bf16(d, a, b0, b1);
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
      next_item<Kind<F16>>(p, kept, c);
      if (NT == 1) fetch_queries<NT>(p, c.b, c.h, queries);  // (of 16 queries they would take the sums' registers)
    }
    named_barrier<kConsumers * 32>(1);  // every warp has read its queries from the scratch
    finish_item<Kind<F16>, NT>(p, st, done, whole, begins, tile_u0, w, scratch, misc, cs, 1.f);
    tile_u0 += done.tiles + kItemCost;
  }
}

template <bool F16, int NT>
__global__ void __launch_bounds__(kThreads<Kind<F16>>, 2) pages_decode_kernel(const __grid_constant__ PagesDecodeParams p) {
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
  prefetch_queries<Kind<F16>>(p);
  Work w;
  Cursor c;
  int* kept = reinterpret_cast<int*>(smem + Smem::lengths);
  const int tiles = find_work<Kind<F16>>(p, const_cast<int*>(misc) + 8, kept, reinterpret_cast<int*>(smem + Smem::scratch), w, c);
  if (tiles == 0) return;
  uint32_t asked = 0;
  if (threadIdx.x / 32 == kConsumers) {
    fence_proxy_async_global();  // pages written by ordinary stores of earlier launches
    asked = produce<Kind<F16>>(p, c, tiles, kept, base, full, empty, misc);
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
  return launch_overlapped(pages_decode_kernel<F16, NT>, dim3((unsigned)decode_ctas()), kThreads<Kind<F16>>, Smem::bytes, s, p);
}

}  // namespace

cudaError_t launch_pages_decode(const PagesDecodeParams& p, bool f16, cudaStream_t s) {
  if (p.group <= 8) return f16 ? launch<true, 1>(p, s) : launch<false, 1>(p, s);
  return f16 ? launch<true, 2>(p, s) : launch<false, 2>(p, s);
}

}  // namespace hg
