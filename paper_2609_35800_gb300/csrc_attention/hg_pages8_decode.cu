// Attention of one new token per request over an 8-bit paged cache, split over the cache's length and joined.
//
// For a request, KV head and its G queries: S_t = scale ks q.c_t with the key block's scale ks, m = max S_t, out = sum
// e^(S_t - m) vs c'_t / sum e^(S_t - m) with the value block's scale vs.  A block is 16 tokens, the height of a product's
// tile, so a scale is one factor of a fragment.  The work is divided and joined as over 16-bit pages (hg_pages_split.cuh),
// an item's fixed costs counted as 6 tiles and a join as 12 (18 shapes, geometric mean: 20.6 us; 20.7 to 20.9 with 3, 4 or
// 8, and 9 or 15).
//
// 2 G flop a byte, so the reads of the cache bound it, but an entry costs twice the instructions a byte of the 16-bit
// kernel's.  Measured: 32 requests x 8,577 tokens x 8 KV heads 86 us, 6.6 TB/s, 0.97 of a copy's rate; one request of
// 131,073 tokens 51 us (0.78: data at 7.1 TB/s from 3 to 40 us, the slowest CTA 3 us later, then the last join); 37 of 1
// to 9,001 tokens, 12 queries a KV head 23 to 25 us (14 tiles a CTA in five rounds of 2.2 us, start, sums and joins; an
// item of one tile takes a CTA 6 us, 3 with up to 8 queries); 321 tokens 6.2 us.
//
// A producer warp copies tiles of 64 tokens into a ring of six 16 KB stages with TMA, a box per page (swizzled rows of 128
// bytes; a page outside the pool reads as zeros), and their scales beside them with four-byte asynchronous copies that
// arrive on the same barrier.  (Tiles of 32 tokens: 118 us where these take 86; a warp's chain of load, products, maximum,
// exponentials and products is what it waits for, and 64 tokens are twice as much side by side.)  Three consumer warps
// take the tiles in turn, each with its own running maximum and sums, and turn codes into FP16 in registers, exactly (e4m3
// is a subset), for mma.sync m16n8k16:
//   S^T[token][query] = K . q        A = keys.  A 16-byte chunk of a row is a product's 16 channels; ldmatrix leaves
//                                    channels 4i .. 4i + 3 in a lane, where the product wants 2i, 2i + 1, 2i + 8, 2i + 9:
//                                    the queries' fragments have the same order, and a sum's order is free
//   O^T[channel][query] += V^T . P^T A = values, by ldmatrix.trans on pairs of channels; a byte permutation parts them,
//                                    rows i and i + 8 of the product are channels 2i and 2i + 1
// A BF16 query is multiplied by a power of two that brings its largest entry below 2^15, so that FP16 holds it, and
// entries down to 2^-31 of it with all their bits; the factor comes back with ks.  P is e^(S - m) 2^7 vs / u, where u is
// the largest vs so far, to a power of two: at most 2^15, as a score may be 2^8 past the running maximum; the sums O stay
// in units of u, are moved when u grows, and are multiplied by u once they are divided (before, sums of values near BF16's
// end would pass binary32's).  Below 2^-21 of the largest probability times the largest scale so far terms lose
// bits, and below 2^-32 of it they are lost to the second product.  Scores, maxima, sums and outputs are held in 32 bits.
#include <cfloat>

#include "hg_pages8.cuh"
#include "hg_pages_split.cuh"

namespace hg {
namespace {

constexpr int kStages = 6;
constexpr int kTile = kDecodeTile8, kTileShift = 6;
static_assert(kTile == 1 << kTileShift, "tile");
constexpr int kConsumers = 3, kItemCost = 6, kJoinCost = 12;
static_assert(kStages % kConsumers == 0, "a stage belongs to one warp");
constexpr int kHalfBytes = kTile * kHeadDim;   // keys; then values
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kQRowBytes = 288;  // a staged query row: 256 bytes and its factor; 8 banks on, so that four rows meet all
constexpr int kTileBlocks = kTile / kBlock8;
constexpr int kScaleLanes = 2 * kTileBlocks;
// A tile with no more tokens than this goes block by block (one token: 3.6 -> 3.0 us an item).  Not of more than 8 queries,
// where a second form of the tile's code costs the first its registers (37 requests of 1 to 9,001 tokens: 24.8 -> 27.0 us).
constexpr int kFewTokens = 32;

// Shared memory, two CTAs an SM.  The staged queries (16 rows at most) and the warps' parts that are added up at an item's
// end (8 queries at a time) take turns in one region.
struct Smem {
  static constexpr int scales = kStages * kStageBytes;  // of each stage: its keys' blocks, its values' blocks
  static constexpr int scratch = scales + kStages * kScaleLanes * 4;
  static constexpr int scratch_bytes = kConsumers * 8 * kSumFloats * 4;
  static constexpr int bars = scratch + scratch_bytes;
  static constexpr int misc = bars + 2 * kStages * 8;  // abort flag, last part, start of the CTA's work, scan
  static constexpr int lengths = misc + 128;           // the first requests' lengths
  static constexpr int bytes = lengths + 4 * kKeptLengths;
};
static_assert(Smem::scratch_bytes >= 16 * kQRowBytes, "queries are staged there too");
static_assert(Smem::scratch_bytes >= ((kConsumers + 1) * 32 + kDecodeJoinCounters / 2 * kDecodeJoinCtas + 2) * 4, "runs' starts too");
static_assert(Smem::scratch % 16 == 0 && Smem::bars % 8 == 0, "alignment");
static_assert((8 + 16 + kConsumers + 1) * 4 <= Smem::lengths - Smem::misc, "the scan's words");
static_assert(2 * (Smem::bytes + 1024) <= 228 * 1024, "two CTAs an SM");

template <bool F16>
struct Kind {
  static constexpr int kTile = hg::kTile, kConsumers = hg::kConsumers, kItemCost = hg::kItemCost, kJoinCost = hg::kJoinCost;
  // Two rounds of the warps: more parts cost their join more than they save (1,475 tokens, 4 KV heads 13.7 us at 1, 9.4 at 6,
  // 10.6 at 9), with more queries three (16 requests of 4,000 tokens, 2 KV heads, 16 queries each 21.8 us at 6, 20.0 at 9).
  static __device__ __forceinline__ int least_share(int group) { return group > 8 ? 9 : 6; }
  static constexpr int kTwoLevels = 8;  // 131,073 tokens, 38 parts of 4 queries by three groups each: 50.4 us, 51.6 at 24
  static constexpr bool kWeighsWhole = true;
  static constexpr bool kF16 = F16;
  static constexpr float kUnlift = 0x1p-7f;
  static constexpr bool kUnits = true;
  static __device__ __forceinline__ float result(float x) { return in_range<F16>(x); }
  static __device__ __forceinline__ void place(float* row, int g, float first, float second) {
    *reinterpret_cast<float2*>(row + 2 * g) = make_float2(first, second);
  }
};

__device__ __forceinline__ void tma_page8(uint32_t dst, const CUtensorMap* map, int row, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(head), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void st_shared4(uint32_t addr, float x) {
  asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(addr), "f"(x) : "memory");
}
// Four bytes, or zeros where `bytes` is 0.
__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// An arrival on `bar`, one of those it counts, once this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(bar) : "memory");
}

// Copies the CTA's tiles into the ring, in order; returns how many it asked for.
template <class K>
__device__ uint32_t produce(const Pages8DecodeParams& p, Cursor c, int tiles, const int* kept, uint32_t stages, uint32_t full,
                            uint32_t empty, volatile int* abort) {
  const int lane = threadIdx.x % 32;
  const int shift = min(p.pool.page_shift, kTileShift), rows = 1 << shift;  // tokens of a box
  const int boxes = kTile >> shift;
  const uint32_t box_bytes = (uint32_t)rows * kHeadDim;
  // the lane's scale of a tile
  const float* scales = lane < kTileBlocks ? p.pool.k_scales : p.pool.v_scales;
  const int block_row = lane % kTileBlocks * kBlock8;
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
          tma_page8(dst, &p.k_map, row, c.h, page, full + 8 * s);
          tma_page8(dst + kHalfBytes, &p.v_map, row, c.h, page, full + 8 * s);
        }
      }
      const int page = __shfl_sync(kAll, id, box0 - first + (block_row >> shift));
      if (lane < kScaleLanes) {
        const int token = c.t * kTile + block_row;
        const bool there = token < c.len && page >= 0 && page < p.pool.num_pages;
        const float* src = there ? scales + scale_at(p.pool, page, token & (p.pool.page_size - 1), c.h) : scales;
        cp_async4(stages + Smem::scales + (s * kScaleLanes + lane) * 4, src, there ? 4 : 0);
        cp_async_arrive(full + 8 * s);
      }
    }
  }
  return n;
}

// The same for pages of 16 tokens, of which a tile is four: eight copies and as many scales' addresses are what everybody
// waits for, so a lane keeps a page and its two scales, 32 pages of an item at a time and the next ones' numbers, and stores
// scales from registers (32 requests x 8,577 tokens, 8 KV heads 100 -> 89 us; 321 tokens 6.6 -> 6.0).  Larger pages lose more
// to the wait for 32 boxes' scales than they gain (pages of 64: 86 -> 89 us).
template <class K>
__device__ uint32_t produce_blocks(const Pages8DecodeParams& p, Cursor c, int tiles, const int* kept, uint32_t stages,
                                   uint32_t full, uint32_t empty, volatile int* abort) {
  constexpr uint32_t kBoxBytes = kBlock8 * kHeadDim;
  const int lane = threadIdx.x % 32;
  uint32_t n = 0;
  // the pages from `first` of request `of` on, and the head whose scales are here; the 32 pages behind them
  int of = -1, head = -1, first = 0, page = -1, next = -1;
  float ks = 0.f, vs = 0.f;
  for (; tiles > 0; next_item<K>(p, kept, c)) {
    const int* ids = p.table + (int64_t)c.b * p.table_stride;
    const int pages = (c.len + kBlock8 - 1) / kBlock8;
    for (; c.t < c.tiles && tiles > 0; ++c.t, --tiles, ++n) {
      const int at = c.t * kTileBlocks, valid = min(kTileBlocks, pages - at);
      const bool fresh = of != c.b || at < first || at + kTileBlocks > first + 32;
      if (fresh || head != c.h) {
        if (fresh) {
          page = of == c.b && at == first + 32 ? next : at + lane < pages ? ids[at + lane] : -1;
          of = c.b;
          first = at;
          next = first + 32 + lane < pages ? ids[first + 32 + lane] : -1;
        }
        head = c.h;
        const bool there = page >= 0 && page < p.pool.num_pages;
        const int64_t place = scale_at(p.pool, there ? page : 0, 0, head);
        ks = there ? p.pool.k_scales[place] : 0.f;
        vs = there ? p.pool.v_scales[place] : 0.f;
      } else if (at - first == 16 && next >= 0 && next < p.pool.num_pages) {
        const int64_t place = scale_at(p.pool, next, 0, head);
        prefetch_l2(p.pool.k_scales + place);
        prefetch_l2(p.pool.v_scales + place);
      }
      const int s = n % kStages;
      if (n >= kStages && !wait_warp(empty + 8 * s, (n / kStages - 1) & 1, abort, p.status)) return n;
      int box[kTileBlocks];
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) box[i] = __shfl_sync(kAll, page, (at - first + i) & 31);
      if (elect_one()) {
        mbar_arrive_expect_tx(full + 8 * s, 2 * max(valid, 0) * kBoxBytes);
#pragma unroll
        for (int i = 0; i < kTileBlocks; ++i) {
          if (i >= valid) break;
          const uint32_t dst = stages + s * kStageBytes + i * kBoxBytes;
          tma_page8(dst, &p.k_map, 0, c.h, box[i], full + 8 * s);
          tma_page8(dst + kHalfBytes, &p.v_map, 0, c.h, box[i], full + 8 * s);
        }
      }
      const int mine = lane - (at - first);
      if (mine >= 0 && mine < kTileBlocks) {
        const uint32_t slot = stages + Smem::scales + (s * kScaleLanes + mine) * 4;
        st_shared4(slot, ks);
        st_shared4(slot + 4 * kTileBlocks, vs);
      }
      __syncwarp();
      if (elect_one()) mbar_arrive(full + 8 * s);
    }
  }
  return n;
}

// An item's query rows on their way: eight lanes a row, the CTA's consumers side by side.
template <int NT>
constexpr int kRowsPerLane = (8 * NT + kGroups<Kind<false>> - 1) / kGroups<Kind<false>>;
template <int NT>
struct MyQueries {
  uint4 lo[kRowsPerLane<NT>], hi[kRowsPerLane<NT>];
  LaneAngles angles;  // of up to 8 queries; those of 16 would be in the sums' way, and come as the rows are turned
};

template <int NT>
__device__ __forceinline__ void fetch_my_queries(const Pages8DecodeParams& p, int b, int h, MyQueries<NT>& x) {
  const int c = threadIdx.x % 8;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr);
  const uint16_t* row = p.q.data + b * p.q.token_stride + (int64_t)h * p.group * p.q.head_stride;
#pragma unroll
  for (int i = 0; i < kRowsPerLane<NT>; ++i) {
    const int q = threadIdx.x / 8 + i * kGroups<Kind<false>>;
    x.lo[i] = x.hi[i] = make_uint4(0u, 0u, 0u, 0u);
    if (q < p.group) {
      x.lo[i] = ldg16(row + q * p.q.head_stride + at.lo);
      x.hi[i] = ldg16(row + q * p.q.head_stride + at.hi);
    }
  }
  if (NT == 1 && at.turns) x.angles = lane_angles(p.rot, c, b);
}

// Rotated, as FP16, into shared memory, once for all consumers, and from there into the first product's operands; `back`:
// what undoes each query's factor.
template <bool F16, int NT>
__device__ __forceinline__ void stage_queries(const Pages8DecodeParams& p, int b, MyQueries<NT>& x, uint32_t staged,
                                              uint32_t (&qf)[NT][16], float (&back)[NT][2]) {
  const int lane = threadIdx.x % 32;
  const LaneChannels at = lane_channels(p.rot, lane % 8, p.rot.table != nullptr);
  if (NT > 1 && at.turns) x.angles = lane_angles(p.rot, lane % 8, b);
#pragma unroll
  for (int i = 0; i < kRowsPerLane<NT>; ++i) {
    const int q = threadIdx.x / 8 + i * kGroups<Kind<F16>>;
    if (at.turns) rotate_lane<F16>(x.lo[i], x.hi[i], x.angles, p.rot.interleaved != 0);
    const uint32_t row = staged + q * kQRowBytes;
    if (!F16) {
      float v[16];
      row_values<F16>(x.lo[i], x.hi[i], nullptr, false, v);
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) top = max(top, finite_bits(v[k]));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(kAll, top, o));
      // 2^(14 - e) for a largest entry in [2^e, 2^(e + 1)), 2^126 at most
      const int field = min(127 + 14 + 127 - (int)(top >> 23), kMostField);
      const float factor = power_of_field(field);
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] *= factor;
      x.lo[i] = pack8<true>(v);
      x.hi[i] = pack8<true>(v + 8);
      if (q < 8 * NT && lane % 8 == 0)
        st_shared16(row + 256, make_uint4(__float_as_uint(inverse_of_field(field)), 0u, 0u, 0u));
    }
    if (q < 8 * NT) {
      st_shared16(row + at.lo * 2, x.lo[i]);
      st_shared16(row + at.hi * 2, x.hi[i]);
    }
  }
  named_barrier<kConsumers * 32>(1);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // a product's 16 channels, four a lane
      const uint32_t a = staged + (8 * nt + lane / 4) * kQRowBytes + (16 * j + 4 * (lane % 4)) * 2;
      asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];\n" : "=r"(qf[nt][2 * j]), "=r"(qf[nt][2 * j + 1]) : "r"(a) : "memory");
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      back[nt][j] = 1.f;
      if (!F16) back[nt][j] = __uint_as_float(ld_shared16(staged + (8 * nt + 2 * (lane % 4) + j) * kQRowBytes + 256).x);
    }
  }
}

// Byte `channel` of row r of a tile; boxes lie one after the other, so that a row's place depends on its number alone.
__device__ __forceinline__ uint32_t tile_byte(uint32_t tile, int r, int channel) {
  return tile + swizzled(r, channel / 16) + channel % 16;
}
__device__ __forceinline__ uint2 ld_shared8(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared8(uint32_t addr, uint2 v) {
  asm volatile("st.shared.v2.b32 [%0], {%1,%2};\n" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}

// The new token of a decode step, row r of the tile: its block is brought to the scale that it needs, in the pool and over
// what the stage holds.  Not where the request has grown past its table: its new token has no place there, and the last
// row is a token's own.  scales: the tile's, keys' blocks before values', which may rise.
template <bool F16>
__device__ __forceinline__ void place_new_token(const Pages8DecodeParams& p, const Cursor& c, uint32_t kt, uint32_t vt, int r,
                                                volatile float* scales) {
  if (p.lengths[c.b] != c.len) return;
  const int lane = threadIdx.x % 32, i = lane % 8;
  const bool is_v = lane / 8 == 1;
  const int last = c.len - 1, block = r / kBlock8, before = r % kBlock8;  // tokens that the block has
  const int page = page_of(p.pool, p.table + (int64_t)c.b * p.table_stride, p.table_stride, last);
  const int in_page = last & (p.pool.page_size - 1);
  const Rows& in = is_v ? p.v : p.k;
  const LaneChannels at = lane_channels(p.rot, i, p.rot.table != nullptr && !is_v);
  const uint16_t* src = in.data + c.b * in.token_stride + c.h * in.head_stride;
  float x[16];
  LaneAngles angles;
  if (at.turns) angles = lane_angles(p.rot, i, c.b);
  row_values<F16>(ldg16(src + at.lo), ldg16(src + at.hi), at.turns ? &angles : nullptr, p.rot.interleaved != 0, x);
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) top = max(top, finite_bits(x[k]));
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(kAll, top, o));
  const float old = scales[(is_v ? kTileBlocks : 0) + block];
  int field = needed_field(top);
  if (before > 0) field = max(field, stored_field(old));
  const float scale = power_of_field(field), inv = inverse_of_field(field);
  uint8_t* row = (is_v ? p.pool.v : p.pool.k) + code_row(p.pool, max(page, 0), in_page, c.h);
  if (lane < 16) {  // keys by the first eight lanes, values by the next
    const uint32_t tile = is_v ? vt : kt;
    const uint2 lo = encode8(x, inv), hi = encode8(x + 8, inv);
    st_shared8(tile_byte(tile, r, at.lo), lo);
    st_shared8(tile_byte(tile, r, at.hi), hi);
    if (page >= 0) {
      *reinterpret_cast<uint2*>(row + at.lo) = lo;
      *reinterpret_cast<uint2*>(row + at.hi) = hi;
      if (i == 0) (is_v ? p.pool.v_scales : p.pool.k_scales)[scale_at(p.pool, page, in_page, c.h)] = scale;
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {  // the block's tokens so far, a lane 8 bytes
    const float from = __shfl_sync(kAll, old, 8 * which), to = __shfl_sync(kAll, scale, 8 * which);
    if (lane == 0) scales[which * kTileBlocks + block] = to;
    if (before == 0 || from == to) continue;
    uint8_t* first = (which ? p.pool.v : p.pool.k) + code_row(p.pool, max(page, 0), in_page - before, c.h);
    const uint32_t tile = which ? vt : kt;
    for (int k = lane; k < before * 16; k += 32) {
      const uint32_t a = tile_byte(tile, r - before + k / 16, k % 16 * 8);
      const uint2 codes = recode8(ld_shared8(a), from / to);
      st_shared8(a, codes);
      if (page >= 0) *reinterpret_cast<uint2*>(first + (k / 16) * p.pool.token_stride + k % 16 * 8) = codes;
    }
  }
  __syncwarp();
}

// NB blocks, of whose tokens the first `seen` belong to the request; scales: the tile's, from the first of these blocks on.
// unit: the exponent field of u.
template <int NB, int NT>
__device__ __forceinline__ void attend_blocks(State<NT>& st, int& unit, const uint32_t (&qf)[NT][16], const float (&back)[NT][2],
                                            uint32_t kt, uint32_t vt, const volatile float* scales, int seen, float c) {
  const int lane = threadIdx.x % 32;
  float ks[NB], vs[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    ks[i] = scales[i];
    vs[i] = scales[kTileBlocks + i];
  }
  float s[NB][NT][4];
#pragma unroll
  for (int mt = 0; mt < NB; ++mt) {
    float s2[NT][4];  // a chain of products for each half of the chunks
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[mt][nt][i] = s2[nt][i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t r[4];
      ldsm_x4(r, kt + mt * kBlock8 * kHeadDim + swizzled(lane % 16, 2 * j + lane / 16));
      uint32_t a[4], b[4];
      decode4(r[0], a[0], a[2]);
      decode4(r[1], a[1], a[3]);
      decode4(r[2], b[0], b[2]);
      decode4(r[3], b[1], b[3]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma_f16(s[mt][nt], a, qf[nt][4 * j], qf[nt][4 * j + 1]);
        mma_f16(s2[nt], b, qf[nt][4 * j + 2], qf[nt][4 * j + 3]);
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // (finite: where query and key share no channel 0 times it is 0, however large they are)
      const float factor[2] = {fminf(ks[mt] * back[nt][0], FLT_MAX), fminf(ks[mt] * back[nt][1], FLT_MAX)};
#pragma unroll
      for (int i = 0; i < 4; ++i) s[mt][nt][i] = (s[mt][nt][i] + s2[nt][i]) * factor[i % 2];
    }
  }
  // a first scale of the values, or one past the old: the sums so far count that much less
  float top_scale = vs[0];
#pragma unroll
  for (int mt = 1; mt < NB; ++mt) top_scale = fmaxf(top_scale, vs[mt]);
  const int field = stored_field(top_scale);
  if (field > unit) {
    const float keep = unit > 0 ? power_of_field(unit) * inverse_of_field(field) : 0.f;
    unit = field;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[nt][d][i] *= keep;
  }
  float share[NB];
#pragma unroll
  for (int mt = 0; mt < NB; ++mt) share[mt] = vs[mt] * inverse_of_field(unit);
  const int g = lane / 4;
  uint32_t pf[NB][NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (seen < NB * kBlock8) {
#pragma unroll
      for (int mt = 0; mt < NB; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * mt + g + 8 * (i / 2) >= seen) s[mt][nt][i] = -INFINITY;
    }
    float top[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      top[j] = fmaxf(s[0][nt][j], s[0][nt][2 + j]);
#pragma unroll
      for (int mt = 1; mt < NB; ++mt) top[j] = fmaxf(top[j], fmaxf(s[mt][nt][j], s[mt][nt][2 + j]));
    }
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
    for (int mt = 0; mt < NB; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float m = st.m[nt][i % 2];
        s[mt][nt][i] = exp2_approx(fmaf(s[mt][nt][i] - (m == -INFINITY ? 0.f : m), c, kLift<true>));
        st.l[nt][i % 2] += s[mt][nt][i];
        s[mt][nt][i] *= share[mt];
      }
      pf[mt][nt][0] = movtrans(pack2<true>(s[mt][nt][0], s[mt][nt][1]));
      pf[mt][nt][1] = movtrans(pack2<true>(s[mt][nt][2], s[mt][nt][3]));
    }
  }
#pragma unroll
  for (int mt = 0; mt < NB; ++mt)
#pragma unroll
    for (int d = 0; d < 8; d += 2) {
      uint32_t r[4];
      ldsm_x4_trans(r, vt + mt * kBlock8 * kHeadDim + swizzled(lane % 16, d + lane / 16));
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = prmt(r[i], 0u, 0x3120u);  // two tokens of a channel side by side
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t a[4];
        decode4(r[2 * e], a[0], a[1]);
        decode4(r[2 * e + 1], a[2], a[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_f16(st.o[nt][d + e], a, pf[mt][nt][0], pf[mt][nt][1]);
      }
    }
}

template <bool F16, int NT>
__device__ void consume(const Pages8DecodeParams& p, Cursor c, const Work& w, int tiles, uint32_t base, char* smem,
                        volatile int* misc) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = base + Smem::bars, empty = full + 8 * kStages;
  const float cs = p.scale * kLog2e;
  float* scratch = reinterpret_cast<float*>(smem + Smem::scratch);
  const int* kept = reinterpret_cast<const int*>(smem + Smem::lengths);
  volatile float* scales = reinterpret_cast<volatile float*>(smem + Smem::scales);
  uint32_t n = 0;
  bool alive = true;  // false: a wait ran out, and the warp only keeps up with the others' barriers
  // unit of the first item's first tile
  int tile_u0 = w.u0 - w.first_unit + kItemCost;
  constexpr bool kEarly = NT == 1;  // (those of 16 queries would be in the sums' way)
  MyQueries<NT> queries;
  if (kEarly) fetch_my_queries<NT>(p, c.b, c.h, queries);
  while (tiles > 0) {
    if (!kEarly) fetch_my_queries<NT>(p, c.b, c.h, queries);
    const bool begins = c.t == 0, whole = begins && c.tiles <= tiles;
    uint32_t qf[NT][16];
    float back[NT][2];
    stage_queries<F16, NT>(p, c.b, queries, base + Smem::scratch, qf, back);
    State<NT> st;
    int unit = 0;
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
      const uint32_t kt = base + s * kStageBytes, vt = kt + kHalfBytes;
      const int seen = c.len - c.t * kTile;
      __syncwarp();
      if (alive && seen > 0) {
        volatile float* its = scales + s * kScaleLanes;
        // what follows the request's last token may be anything, and 0 times NaN is no 0
        const bool few = NT == 1 && seen <= kFewTokens;
        const int end = few ? (seen + kBlock8 - 1) & ~(kBlock8 - 1) : kTile;
        for (int i = seen * 8 + lane; i < end * 8; i += 32)
          st_shared16(vt + swizzled(i / 8, i % 8), make_uint4(0u, 0u, 0u, 0u));
        if (seen <= kTile && p.store) place_new_token<F16>(p, c, kt, vt, seen - 1, its);
        __syncwarp();
        if (few) {
#pragma unroll 1
          for (int i = 0; i < end; i += kBlock8)
            attend_blocks<1, NT>(st, unit, qf, back, kt + i * kHeadDim, vt + i * kHeadDim, its + i / kBlock8, seen - i, cs);
        } else {
          attend_blocks<kTileBlocks, NT>(st, unit, qf, back, kt, vt, its, seen, cs);
        }
        if (seen <= kTile) fence_proxy_async_shared();  // TMA writes the stage again
      }
      __syncwarp();
      // (not after a wait that ran out: the stage would be filled over a copy whose bytes are still expected)
      if (alive && lane == 0) mbar_arrive(empty + 8 * s);
    }
    const Cursor done = c;
    if (tiles > 0) {  // the next item's queries come in meanwhile
      next_item<Kind<F16>>(p, kept, c);
      if (kEarly) fetch_my_queries<NT>(p, c.b, c.h, queries);
    }
    named_barrier<kConsumers * 32>(1);  // every warp has read its queries from the scratch
    finish_item<Kind<F16>, NT>(p, st, done, whole, begins, tile_u0, w, scratch, misc, cs,
                                     unit > 0 ? power_of_field(unit) : 0.f);
    tile_u0 += done.tiles + kItemCost;
  }
}

template <bool F16, int NT>
__global__ void __launch_bounds__(kThreads<Kind<F16>>, 2) pages8_decode_kernel(const __grid_constant__ Pages8DecodeParams p) {
  extern __shared__ __align__(1024) char smem[];
  const uint32_t base = smem_u32(smem), full = base + Smem::bars, empty = full + 8 * kStages;
  volatile int* misc = reinterpret_cast<int*>(smem + Smem::misc);  // [0] abort, [1] last part, [8 ..] scan
  const bool blocks = p.pool.page_shift == kBlock8Shift;  // pages of 16 tokens
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      // the copies that are asked for, and the scales: stored (by produce_blocks), or each with a copy of its own
      mbar_init(full + 8 * i, 1 + (blocks ? 1 : kScaleLanes));
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
    asked = blocks ? produce_blocks<Kind<F16>>(p, c, tiles, kept, base, full, empty, misc)
                   : produce<Kind<F16>>(p, c, tiles, kept, base, full, empty, misc);
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
cudaError_t launch(const Pages8DecodeParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};  // devices whose shared-memory limit is raised
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(pages8_decode_kernel<F16, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem::bytes);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_overlapped(pages8_decode_kernel<F16, NT>, dim3((unsigned)decode_ctas()), kThreads<Kind<F16>>, Smem::bytes, s, p);
}

}  // namespace

cudaError_t launch_pages8_decode(const Pages8DecodeParams& p, bool f16, cudaStream_t s) {
  if (p.group <= 8) return f16 ? launch<true, 1>(p, s) : launch<false, 1>(p, s);
  return f16 ? launch<true, 2>(p, s) : launch<false, 2>(p, s);
}

}  // namespace hg
