// Attention of packed prompts on the fifth-generation tensor cores.
//
// For a prompt's query row: s_t = scale q.k_t over the keys it sees, m = max s_t, out = sum e^(s_t - m) v_t / sum
// e^(s_t - m).  4 * 128 flop a (query head, key) pair and little to read: the kernel is bound by the products, and for
// short prompts by the chain of a tile's blocks.  Measured: 2 x 8,192 causal tokens of 64 heads 1,551-1,565 TFLOP/s in short
// runs, 1,462 over seconds under the power limit (at 1,950 MHz: 4,930 flop a cycle and SM, of 7,780 that a large matrix
// product reaches).  An earlier form ran at 1,461, at 1,604 with the softmax left out and at 1,641 without loads either, so
// most of the rest is in the products as they are issued here; what holds them back is not known (shared memory's pipe is
// 42% busy with their operands).  1,460 tokens of 28 heads 25.5 us, 12 blocks of 3,000 cycles one after the other.
//
// A work item is two tiles of 128 rows of one prompt and KV head.  A tile's rows are 128 / G consecutive tokens times
// the G query heads of the KV head, so short prompts fill their tiles and a causal tile spans few tokens; both tiles use
// every key block that is loaded.  One persistent CTA per SM takes items from a counter, longest first; its warps:
//   warp 9      loads: the items' queries, then 128-key blocks of K and V into a ring, by TMA (128-byte swizzle)
//   warp 8      issues the products: S = Q K^T into tensor memory, then O += P V with P read from tensor memory
//   warps 0-3, 4-7  softmax of tile 0 and of tile 1, a thread to a row: S out of tensor memory, P back over it (so a
//               tile's next S follows its P V), O scaled there when a maximum moves, written out at the end
// While one tile's softmax runs the tensor cores work on the other tile.  Tensor memory: S 2 x 128 columns, O 2 x 128.
// What is not here because it was slower at 2 x 8,192 tokens (on short items none of it was measured): P handed over in
// halves (1,409 TFLOP/s then, 1,467 without), outputs written by a warpgroup of their own (1,387), items taken by a warp of
// its own (1,508 of 1,547: every waiting warp takes something), three or five stages of the ring (1,514 and 1,497 of 1,541
// and 1,562).
//
// Scores, maxima, sums and O are held in 32 bits; P is rounded to the inputs' type for the second product, lifted in FP16
// (kLift).  The running maximum moves when a score passes it by more than 2^8, which bounds P and makes changes of O rare.
// Where the items are fewer than the SMs can share (few rows over long keys), an item's keys are cut into pieces whose
// (m, l, O) go to the workspace, and a second kernel joins them (64 tokens after 16,000: 25 us;
// uncut, 126 blocks would follow one another).
#include <algorithm>

#include "hg_rows.cuh"
#include "hg_tcgen05.cuh"

namespace hg {
namespace {

constexpr int kBlock = kPromptBlock;        // keys of a block
constexpr int kTileRows = 128;
constexpr int kHalfBytes = 128 * 128;       // 64 channels of 128 rows
constexpr int kTileBytes = 2 * kHalfBytes;  // a tile of queries, a block of keys or of values
constexpr int kStages = 4;
constexpr int kThreads = 384;  // the last two warps have nothing to do: registers are divided by warpgroups
// Registers a thread: at launch 65,536 / 384 give 168; the softmax rows need more, the others less.
constexpr int kRowRegisters = 208, kOtherRegisters = 88;
static_assert(256 * kRowRegisters + 128 * kOtherRegisters <= kThreads * 168, "what the launch has");
constexpr int kMmaWarp = 8, kLoadWarp = 9;
constexpr uint32_t kScoreColumn = 0, kOutColumn = 256;  // + 128 for tile 1
constexpr unsigned kAll = 0xffffffffu;

// Shared memory from a 1024-byte boundary.
constexpr int kQueryOffset = 0;
constexpr int kRingOffset = 2 * kTileBytes;
constexpr int kOutOffset = kRingOffset + kStages * kTileBytes;  // half of the channels of each tile, on their way out
constexpr int kBarOffset = kOutOffset + 2 * kHalfBytes;
constexpr int kSmemBytes = kBarOffset + 512 + 1024;
enum Bar { kQueryFull = 0, kQueryFree, kScoreFull, kProbFull = kScoreFull + 2, kOutFull = kProbFull + 2,
           kStageFull = kOutFull + 2, kStageFree = kStageFull + 2, kItemFull = kStageFree + 2, kItemFree = kItemFull + 2,
           kRingFull = kItemFree + 2, kRingFree = kRingFull + kStages, kBars = kRingFree + kStages };
constexpr int kItemOffset = kBarOffset + 256;  // two Items
constexpr int kMiscOffset = kItemOffset + 2 * 64;  // abort flag, tensor memory address, copies asked for
static_assert(kBars * 8 <= 256, "barriers");

struct __align__(16) Item {
  int q0;         // first query row (token of the tensors) of the prompt
  int tok0;       // first token of tile 0, in the prompt
  int q_len, k_len, k0;
  int head;       // KV head
  int first;      // first key block
  int n[2];       // key blocks of each tile from `first` on
  int width[2];   // keys of the last of them that some row sees
  int slot;       // where the item's part goes; -1: the item is whole
  int slot_step;  // from a piece's slot to the next one's
  int none;       // no further item
};
static_assert(sizeof(Item) == 64, "items");

__device__ __forceinline__ int seen_by(const PromptParams& p, int q_len, int k_len, int tok) {
  return p.causal ? min(max(tok + 1 + k_len - q_len, 0), k_len) : k_len;
}

// The item at a shared-memory address.
__device__ __forceinline__ void read_item(Item& it, uint32_t from) {
  union {
    uint4 w[4];
    Item item;
  } x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.w[i] = ld_shared16(from + 16 * i);
  it = x.item;
}

// Item number -> work: prompt by prompt (longest first), piece by piece, tile pair by tile pair (last tokens first), heads
// innermost.  False: the piece holds no key of its tiles.
__device__ bool item_at(const PromptParams& p, int index, Item& it) {
  const int head = index % p.kv_heads, unit = index / p.kv_heads;
  int lo = 0, hi = p.prompts;  // the prompt that holds the unit
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.first_unit[mid] <= unit) lo = mid;
    else hi = mid;
  }
  const PromptRange r = p.range[lo];
  const int tiles = (r.q_len + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens), local = unit - p.first_unit[lo];
  const int piece = local / tiles, tile = local - piece * tiles;
  it.q0 = r.q0;
  it.q_len = r.q_len;
  it.k0 = r.k0;
  it.k_len = r.k_len;
  it.tok0 = (tiles - 1 - tile) * 2 * p.tile_tokens;
  it.head = head;
  it.first = piece * p.chunk;
  it.none = 0;
  int blocks = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int from = it.tok0 + t * p.tile_tokens, to = min(from + p.tile_tokens, r.q_len) - 1;  // the last row sees most
    const int seen = from < r.q_len ? seen_by(p, r.q_len, r.k_len, to) : 0;
    const int n = (seen + kBlock - 1) / kBlock;
    blocks = max(blocks, n);
    const int end = min(n, it.first + p.chunk);
    it.n[t] = max(0, end - it.first);
    it.width[t] = min(kBlock, seen - (end - 1) * kBlock);
  }
  it.slot = blocks > p.chunk ? index : -1;
  it.slot_step = tiles * p.kv_heads;
  return piece == 0 || blocks > it.first;
}

// One warp: items from the counter to the others, queries and key blocks into shared memory.  Returns the ring's fills.
__device__ void load_items(const PromptParams& p, Item it, bool some, uint32_t base, char* smem, volatile int* misc,
                           uint32_t& fills, uint32_t& queries) {
  const int lane = threadIdx.x % 32;
  const uint32_t bars = base + kBarOffset;
  Item* items = reinterpret_cast<Item*>(smem + kItemOffset);
  const uint32_t q_bytes = (uint32_t)p.group * p.tile_tokens * 128;
  fills = queries = 0;
  for (uint32_t n = 0;; ++n, some = false) {
    while (!some) {
      int index = 0;
      if (lane == 0) index = (int)gridDim.x + (int)atomicAdd(p.counters, 1u);
      index = __shfl_sync(kAll, index, 0);
      it.none = index >= p.items;
      some = it.none || item_at(p, index, it);
    }
    const uint32_t s = n & 1;
    if (n >= 2 && !wait_warp<true>(bars + 8 * (kItemFree + s), ((n >> 1) - 1) & 1, misc, p.status)) return;
    if (lane == 0) {
      items[s] = it;
      mbar_arrive(bars + 8 * (kItemFull + s));
    }
    if (it.none) return;
    const int blocks = max(it.n[0], it.n[1]);
    if (blocks == 0) continue;
    if (queries > 0 && !wait_to_fill(bars + 8 * kQueryFree, (queries - 1) & 1, misc, p.status)) return;
    if (lane == 0) {
      const uint32_t bar = bars + 8 * kQueryFull;
      mbar_arrive_expect_tx(bar, (uint32_t)((it.n[0] > 0) + (it.n[1] > 0)) * 2 * q_bytes);
      for (int t = 0; t < 2; ++t)
        if (it.n[t] > 0)
          for (int half = 0; half < 2; ++half)
            tma_load_3d(base + kQueryOffset + t * kTileBytes + half * kHalfBytes, &p.q_map, 64 * half, it.head * p.group,
                        it.q0 + it.tok0 + t * p.tile_tokens, bar);
    }
    ++queries;
    for (int j = 0; j < 2 * blocks; ++j, ++fills) {  // K, V of a block
      const uint32_t stage = fills % kStages, round = fills / kStages;
      if (round > 0 && !wait_to_fill<true>(bars + 8 * (kRingFree + stage), (round - 1) & 1, misc, p.status)) return;
      if (lane == 0) {
        misc[2] = (int)fills;
        const uint32_t bar = bars + 8 * (kRingFull + stage), dst = base + kRingOffset + stage * kTileBytes;
        mbar_arrive_expect_tx(bar, kTileBytes);
        for (int half = 0; half < 2; ++half)
          tma_load_3d(dst + half * kHalfBytes, j % 2 ? &p.v_map : &p.k_map, 64 * half, it.k0 + (it.first + j / 2) * kBlock,
                      it.head, bar);
      }
      __syncwarp();
    }
  }
}

// One warp, of which one thread issues every product.  Returns how many of the ring's blocks they have used.
template <bool F16>
__device__ uint32_t issue_products(const PromptParams& p, uint32_t base, uint32_t tmem, volatile int* misc) {
  const int lane = threadIdx.x % 32;
  const uint32_t bars = base + kBarOffset;
  const uint32_t q_operand = smem_operand(base + kQueryOffset, 16), k_operand = smem_operand(base + kRingOffset, 16);
  const uint32_t v_operand = smem_operand(base + kRingOffset, kHalfBytes), v_shape = mma_shape(F16, kHeadDim, true);
  uint32_t fill = 0, queries = 0, probs[2] = {0, 0};
  for (uint32_t n = 0;; ++n) {
    const uint32_t slot = n & 1;
    if (!wait_warp(bars + 8 * (kItemFull + slot), (n >> 1) & 1, misc, p.status)) return fill;
    Item it;
    read_item(it, base + kItemOffset + slot * 64);
    const int none = it.none, first = it.first, k_len = it.k_len;
    const int count[2] = {it.n[0], it.n[1]}, width[2] = {it.width[0], it.width[1]};
    __syncwarp();
    if (lane == 0) mbar_arrive(bars + 8 * (kItemFree + slot));
    if (none) return fill;
    const int blocks = max(count[0], count[1]);
    if (blocks == 0) continue;
    wait_data(bars + 8 * kQueryFull, queries & 1, misc, p.status);
    ++queries;

    // S of tile t and block j: 128 rows by the block's keys that any of them sees, 16 channels at a time
    auto scores = [&](int t, int j, uint32_t stage) {
      if (j >= count[t] || !elect_one()) return;
      const int keys = j == count[t] - 1 ? (width[t] + 15) & ~15 : kBlock;
      const uint32_t shape = mma_shape(F16, keys, false), q = q_operand + t * (kTileBytes >> 4);
      const uint32_t k = k_operand + stage * (kTileBytes >> 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t at = ((i / 4) * kHalfBytes + (i % 4) * 32) >> 4;
        tc_mma_ss(tmem + kScoreColumn + 128 * t, q + at, k + at, shape, i > 0);
      }
      tc_commit(bars + 8 * (kScoreFull + t));
      if (j == count[t] - 1 && count[t] == blocks && (t == 1 || count[1] < blocks)) tc_commit(bars + 8 * kQueryFree);
    };
    auto wait_fill = [&](uint32_t f) { wait_data(bars + 8 * (kRingFull + f % kStages), (f / kStages) & 1, misc, p.status); };

    // the ring holds K, V of block 0, K, V of block 1, ...: block j's K is fill + 2 j
    wait_fill(fill);
    scores(0, 0, fill % kStages);
    scores(1, 0, fill % kStages);
    if (elect_one()) tc_commit(bars + 8 * (kRingFree + fill % kStages));
    for (int j = 0; j < blocks; ++j) {
      const uint32_t fv = fill + 2 * j + 1, fk = fv + 1;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (j >= count[t]) continue;
        wait_data(bars + 8 * (kProbFull + t), probs[t] & 1, misc, p.status);
        if (t == 0 || j >= count[0]) {  // the first that reads this block's values
          wait_fill(fv);
          const int valid = k_len - (first + j) * kBlock;
          if (valid < kBlock && valid % 16 != 0) {
            // rows past the prompt's last value may be anything, and 0 times NaN is no 0: zeros up to a step's end
            const uint32_t v = base + kRingOffset + (fv % kStages) * kTileBytes;
            for (int i = lane; i < (16 - valid % 16) * 16; i += 32)
              st_shared16(v + (i / 8 % 2) * kHalfBytes + swizzled(valid + i / 16, i % 8), make_uint4(0u, 0u, 0u, 0u));
            fence_proxy_async_shared();
            __syncwarp();
          }
        }
        const uint32_t v = v_operand + (fv % kStages) * (kTileBytes >> 4), o = tmem + kOutColumn + 128 * t;
        const uint32_t prob = tmem + kScoreColumn + 128 * t;
        const int steps = j < count[t] - 1 ? kBlock / 16 : (width[t] + 15) / 16;
        tc_fence_after();
        ++probs[t];
        if (elect_one()) {
          if (steps == kBlock / 16) {
#pragma unroll
            for (int i = 0; i < kBlock / 16; ++i) tc_mma_ts(o, prob + 8 * i, v + i * (2048 >> 4), v_shape, i > 0 ? 1u : j > 0);
          } else {
            for (int i = 0; i < steps; ++i) tc_mma_ts(o, prob + 8 * i, v + i * (2048 >> 4), v_shape, j > 0 || i > 0);
          }
          if (j == count[t] - 1) tc_commit(bars + 8 * (kOutFull + t));
        }
        __syncwarp();
        if (j + 1 < count[t]) {
          wait_fill(fk);
          scores(t, j + 1, fk % kStages);
        }
      }
      if (elect_one()) {
        tc_commit(bars + 8 * (kRingFree + fv % kStages));
        if (j + 1 < blocks) tc_commit(bars + 8 * (kRingFree + fk % kStages));
      }
      __syncwarp();
    }
    fill += 2 * blocks;
  }
}

// A row's softmax so far.  Its probabilities are 2^(s c - (M + r)), c = scale log2(e): M is the maximum times c less the
// lift, rounded; r, what the rounding took, where M is so large that it shows, else 0.
struct RowSum {
  float M, r, l;
};

template <bool F16>
__device__ __forceinline__ float residual(float top, float c, float M) {
  return fabsf(M) >= 1048576.f && fabsf(M) < INFINITY ? fmaf(top, c, -M) - kLift<F16> : 0.f;
}

__device__ __forceinline__ void st_global32(void* to, const uint32_t (&x)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"l"(to), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]),
               "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
               : "memory");
}

// 64 scores of a row to probabilities, two of the type in a word; returns their sum.
template <bool F16>
__device__ __forceinline__ float half_probabilities(const uint32_t (&a)[32], const uint32_t (&b)[32], const RowSum& st, float c,
                                                    uint32_t (&prob)[32]) {
  const float shift = st.M == -INFINITY ? 0.f : -st.M;
  const uint64_t c2 = f32x2(__float_as_uint(c), __float_as_uint(c));
  const uint64_t shift2 = f32x2(__float_as_uint(shift), __float_as_uint(shift));
  uint64_t sum[2] = {0, 0};
  if (__any_sync(kAll, st.r != 0.f)) {
    const uint64_t r2 = f32x2(__float_as_uint(-st.r), __float_as_uint(-st.r));
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const uint32_t lo = k < 16 ? a[2 * k & 31] : b[2 * k & 31], hi = k < 16 ? a[(2 * k + 1) & 31] : b[(2 * k + 1) & 31];
      const uint64_t x = f32x2_add(f32x2_fma(f32x2(lo, hi), c2, shift2), r2);
      const float e = exp2_approx(__uint_as_float((uint32_t)x)), f = exp2_approx(__uint_as_float((uint32_t)(x >> 32)));
      sum[k % 2] = f32x2_add(sum[k % 2], f32x2(__float_as_uint(e), __float_as_uint(f)));
      prob[k] = pack2<F16>(e, f);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const uint32_t lo = k < 16 ? a[2 * k & 31] : b[2 * k & 31], hi = k < 16 ? a[(2 * k + 1) & 31] : b[(2 * k + 1) & 31];
      const uint64_t x = f32x2_fma(f32x2(lo, hi), c2, shift2);
      const float e = exp2_approx(__uint_as_float((uint32_t)x)), f = exp2_approx(__uint_as_float((uint32_t)(x >> 32)));
      sum[k % 2] = f32x2_add(sum[k % 2], f32x2(__float_as_uint(e), __float_as_uint(f)));
      prob[k] = pack2<F16>(e, f);
    }
  }
  sum[0] = f32x2_add(sum[0], sum[1]);
  return __uint_as_float((uint32_t)sum[0]) + __uint_as_float((uint32_t)(sum[0] >> 32));
}

// 128 threads, a row each, of tile t.
template <bool F16>
__device__ void softmax_rows(const PromptParams& p, int t, uint32_t base, uint32_t tmem, volatile int* misc) {
  const int lane = threadIdx.x % 32, row = threadIdx.x % kTileRows;
  const uint32_t bars = base + kBarOffset;
  const uint32_t mine = (uint32_t)(row / 32 * 32) << 16;  // this warp's lanes of tensor memory
  const uint32_t s_at = tmem + mine + kScoreColumn + 128 * t, o_at = tmem + mine + kOutColumn + 128 * t;
  const float c = p.scale * kLog2e;
  const int tok_of_row = row / p.group, head_of_row = row - tok_of_row * p.group;
  uint32_t scores = 0, outs = 0, stores = 0;
  for (uint32_t n = 0;; ++n) {
    const uint32_t slot = n & 1;
    // (a tile without rows waits for as long as the other tile's keys take)
    if (!wait_for_others(bars + 8 * (kItemFull + slot), (n >> 1) & 1, misc + 2, misc, p.status)) return;
    Item it;
    read_item(it, base + kItemOffset + slot * 64);
    const int blocks = t == 0 ? it.n[0] : it.n[1];
    __syncwarp();
    if (lane == 0) mbar_arrive(bars + 8 * (kItemFree + slot));
    if (it.none) return;
    const int tok = it.tok0 + t * p.tile_tokens + tok_of_row;
    const bool valid = tok_of_row < p.tile_tokens && tok < it.q_len;
    const int seen = seen_by(p, it.q_len, it.k_len, tok);
    const int limit = valid ? seen : 0x7fffffff;  // rows of nobody need no mask
    const int least = __reduce_min_sync(kAll, limit);
    RowSum st = {-INFINITY, 0.f, 0.f};
    for (int j = 0; j < blocks; ++j, ++scores) {
      wait_data(bars + 8 * (kScoreFull + t), scores & 1, misc, p.status);
      tc_fence_after();
      uint32_t w[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_load32(w[i], s_at + 32 * i);
      tmem_wait_loads();
      const int key0 = (it.first + j) * kBlock;
      if (least < key0 + kBlock) {
#pragma unroll
        for (int i = 0; i < 128; ++i)
          if (key0 + i >= limit) w[i / 32][i % 32] = 0xff800000u;  // -inf
      }
      float top[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top[i] = __uint_as_float(w[i][0]);
#pragma unroll
        for (int k = 1; k < 31; k += 2) top[i] = fmaxf(fmaxf(top[i], __uint_as_float(w[i][k])), __uint_as_float(w[i][k + 1]));
        top[i] = fmaxf(top[i], __uint_as_float(w[i][31]));
      }
      const float best = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      const float M = fmaf(best, c, -kLift<F16>);
      // each row by itself (rows of nobody hold what shared memory held, and must not change the others' rounding)
      // (by the unrounded maxima: of scores in the millions the rounded ones may be near where these are far apart)
      const float r = residual<F16>(best, c, M);
      const bool moves = valid && (M - st.M) + (r - st.r) > kRescale;
      if (__any_sync(kAll, moves)) {
        float keep = 1.f;
        if (moves) {
          keep = exp2_approx((st.M - M) + (st.r - r));
          st.M = M;
          st.r = r;
          st.l *= keep;
        }
        __syncwarp();
        if (j > 0) {
          // S of this block is complete, so P V of the one before is, and nothing writes O now
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            uint32_t o[32];
            tmem_load32(o, o_at + 32 * i);
            tmem_wait_loads();
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * keep);
            tmem_store32(o_at + 32 * i, o);
          }
        }
      }
      uint32_t prob[32];
      const float sum = half_probabilities<F16>(w[0], w[1], st, c, prob);
      tmem_store32(s_at, prob);
      st.l += sum + half_probabilities<F16>(w[2], w[3], st, c, prob);
      tmem_store32(s_at + 32, prob);
      tmem_wait_stores();
      tc_fence_before();
      mbar_arrive(bars + 8 * (kProbFull + t));
    }

    // the tile's end: about 3,500 cycles, a third of it in the two copies of a whole tile
    if (blocks > 0) {
      wait_data(bars + 8 * (kOutFull + t), outs & 1, misc, p.status);
      ++outs;
      tc_fence_after();
    }
    const bool whole = it.slot < 0;
    const int head = it.head * p.group + head_of_row;
    const int64_t token = (int64_t)it.q0 + tok;
    if (whole && valid && p.lse)
      p.lse[token * p.q_heads + head] = st.l == 0.f ? -INFINITY : ((st.M + st.r) + log2f(st.l)) * 0.69314718055994531f;
    const float scale = seen > 0 ? 1.0f / st.l : 0.f;
    uint16_t* out = p.out.data + token * p.out.token_stride + head * p.out.head_stride;
    const bool aligned = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
    float* part = p.parts + (int64_t)it.slot * kPromptPartFloats;
    const int part_row = t * kTileRows + row;
    if (!whole && valid) {
      part[part_row] = isnan(st.l) ? 0.f : st.M;  // (a piece whose scores are all NaN has no maximum, and counts)
      part[256 + part_row] = st.r;
      part[512 + part_row] = st.l;
    }
    if (whole && blocks > 0 && p.out_mapped && it.tok0 + (t + 1) * p.tile_tokens <= it.q_len) {
      // every row is somebody's: through shared memory, and one copy for each half of the channels
      const uint32_t stage = base + kOutOffset + t * kHalfBytes;
#pragma unroll 1
      for (int half = 0; half < 2; ++half, ++stores) {
        if (stores > 0) wait_data(bars + 8 * (kStageFree + t), (stores - 1) & 1, misc, p.status);
        uint32_t o[2][32];
        tmem_load32(o[0], o_at + 64 * half);
        tmem_load32(o[1], o_at + 64 * half + 32);
        tmem_wait_loads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[e] = pack2<F16>(__uint_as_float(o[k / 4][(8 * k + 2 * e) % 32]) * scale,
                              __uint_as_float(o[k / 4][(8 * k + 2 * e + 1) % 32]) * scale);
          st_shared16(stage + swizzled(row, k), make_uint4(x[0], x[1], x[2], x[3]));
        }
        fence_proxy_async_shared();
        mbar_arrive(bars + 8 * (kStageFull + t));
        if (row == 0) {
          wait_phase(bars + 8 * (kStageFull + t), stores & 1, misc, p.status);
          tma_store_3d(&p.out_map, stage, 64 * half, it.head * p.group, it.q0 + it.tok0 + t * p.tile_tokens);
          bulk_stores_read();
          mbar_arrive(bars + 8 * (kStageFree + t));
        }
        __syncwarp();
      }
      tc_fence_before();
      continue;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t o[32];
      if (blocks > 0) {
        tmem_load32(o, o_at + 32 * i);
        tmem_wait_loads();
      } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = 0u;
      }
      if (valid && whole) {
        // a lane's row lies on lines of its own, and a warp's store takes a cycle a line: 32 bytes a store where they are
        // aligned (an item's output takes about 2,700 cycles, 4,500 in stores of 16 bytes)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] = pack2<F16>(__uint_as_float(o[16 * k + 2 * e]) * scale, __uint_as_float(o[16 * k + 2 * e + 1]) * scale);
          if (aligned) {
            st_global32(out + 32 * i + 16 * k, x);
          } else {
            *reinterpret_cast<uint4*>(out + 32 * i + 16 * k) = make_uint4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<uint4*>(out + 32 * i + 16 * k + 8) = make_uint4(x[4], x[5], x[6], x[7]);
          }
        }
      } else if (valid) {
        // [channel / 4][row][4]: a warp's rows lie side by side
#pragma unroll
        for (int k = 0; k < 8; ++k)
          *reinterpret_cast<uint4*>(part + 768 + ((8 * i + k) * 256 + part_row) * 4) =
              make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
      }
      __syncwarp();
    }
    tc_fence_before();
  }
}

template <bool F16>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const __grid_constant__ PromptParams p) {
  extern __shared__ char raw[];
  char* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  const uint32_t base = smem_u32(smem), bars = base + kBarOffset;
  volatile int* misc = reinterpret_cast<int*>(smem + kMiscOffset);
  const int warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    mbar_init(bars + 8 * kQueryFull, 1);
    mbar_init(bars + 8 * kQueryFree, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(bars + 8 * (kScoreFull + t), 1);
      mbar_init(bars + 8 * (kProbFull + t), kTileRows);
      mbar_init(bars + 8 * (kOutFull + t), 1);
      mbar_init(bars + 8 * (kStageFull + t), kTileRows);
      mbar_init(bars + 8 * (kStageFree + t), 1);
      mbar_init(bars + 8 * (kItemFull + t), 1);
      mbar_init(bars + 8 * (kItemFree + t), 9);  // eight softmax warps and the one that issues
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(bars + 8 * (kRingFull + i), 1);
      mbar_init(bars + 8 * (kRingFree + i), 1);
    }
    mbar_init_fence();
    misc[0] = misc[2] = 0;
  }
  if (warp == kMmaWarp) tmem_alloc(base + kMiscOffset + 4, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)misc[1];
  Item mine;  // the first one is known from the launch's parameters alone
  bool some = false;
  if (warp == kLoadWarp) {
    const int lane = threadIdx.x % 32;  // (without a key in any prompt, or with an output that has no map, there is none)
    if (lane == 0) prefetch_tensormap(&p.q_map);
    if (lane == 1 && p.range[0].k_len > 0) prefetch_tensormap(&p.k_map);
    if (lane == 2 && p.range[0].k_len > 0) prefetch_tensormap(&p.v_map);
    if (lane == 3 && p.out_mapped) prefetch_tensormap(&p.out_map);
    some = item_at(p, blockIdx.x, mine);
  }
  grid_launch_dependents();
  grid_dependency_wait();
  uint32_t fills = 0, queries = 0;
  if (warp >= kMmaWarp) {
    set_registers_down<kOtherRegisters>();
    if (warp == kLoadWarp) {
      fence_proxy_async_global();  // inputs written by ordinary stores of earlier launches
      load_items(p, mine, some, base, smem, misc, fills, queries);
    } else if (warp == kMmaWarp) {
      fills = issue_products<F16>(p, base, tmem, misc);
    }
  } else {
    set_registers_up<kRowRegisters>();
    softmax_rows<F16>(p, warp / 4, base, tmem, misc);
    if (threadIdx.x % kTileRows == 0) bulk_stores_done();
  }
  tc_fence_before();
  __syncthreads();
  if (misc[0] && warp == kLoadWarp) {  // a CTA that gave up leaves once the copies it asked for have landed
    for (uint32_t n = fills > kStages ? fills - kStages : 0; n < fills; ++n)
      drain_phase(bars + 8 * (kRingFull + n % kStages), (n / kStages) & 1);
    if (queries > 0) drain_phase(bars + 8 * kQueryFull, (queries - 1) & 1);
  }
  if (misc[0] && warp == kMmaWarp && fills > 0)  // and its products have ended: the last commit gave a place back
    drain_phase(bars + 8 * (kRingFree + (fills - 1) % kStages), ((fills - 1) / kStages) & 1);
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_free(tmem, 512);
  }
  // the last CTA leaves the counters at zero for the next launch: no other takes an item any more
  if (threadIdx.x == 0 && atomicAdd(p.counters + 1, 1u) == gridDim.x - 1) {
    p.counters[0] = 0u;
    p.counters[1] = 0u;
  }
}

// Joins the pieces of an item: a CTA takes 32 of its 256 rows, a lane each, and 32 channels of them, four to a warp.
template <bool F16>
__global__ void __launch_bounds__(256) prompt_join_kernel(const __grid_constant__ PromptParams p) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int lane = threadIdx.x % 32, quad = blockIdx.y * 8 + threadIdx.x / 32;  // channels 4 quad ..
  const int row = (blockIdx.x % 8) * 32 + lane, head_of_kv = blockIdx.x / 8 % p.kv_heads, tile = blockIdx.x / 8 / p.kv_heads;
  int prompt = 0, next = p.prompts;
  while (next - prompt > 1) {
    const int mid = (prompt + next) / 2;
    if (p.first_tile[mid] <= tile) prompt = mid;
    else next = mid;
  }
  Item it;  // its first piece
  item_at(p, (p.first_unit[prompt] + tile - p.first_tile[prompt]) * p.kv_heads + head_of_kv, it);
  if (it.slot < 0) return;  // whole
  const int t = row / kTileRows, in_tile = row % kTileRows;
  const int tok_of_row = in_tile / p.group, tok = it.tok0 + t * p.tile_tokens + tok_of_row;
  if (tok_of_row >= p.tile_tokens || tok >= it.q_len) return;
  const int seen = seen_by(p, it.q_len, it.k_len, tok), head = it.head * p.group + in_tile % p.group;
  const int64_t token = (int64_t)it.q0 + tok;
  // pieces that hold a key of either tile were written
  const int last_tok = min(it.tok0 + 2 * p.tile_tokens, it.q_len) - 1;
  const int blocks = (seen_by(p, it.q_len, it.k_len, last_tok) + kBlock - 1) / kBlock;
  const int pieces = (blocks + p.chunk - 1) / p.chunk;
  const float* part = p.parts + (int64_t)it.slot * kPromptPartFloats;
  const int64_t step = (int64_t)it.slot_step * kPromptPartFloats;
  float M = -INFINITY, r = 0.f, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kBatch = 6;  // pieces whose reads are in flight together
#pragma unroll 1
  for (int i0 = 0; i0 < pieces; i0 += kBatch) {
    float m[kBatch], mr[kBatch], ml[kBatch];
    float4 x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float* from = part + min(i0 + i, pieces - 1) * step;
      m[i] = i0 + i < pieces ? from[row] : -INFINITY;
      mr[i] = from[256 + row];
      ml[i] = from[512 + row];
      x[i] = *reinterpret_cast<const float4*>(from + 768 + (quad * 256 + row) * 4);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      // the piece has no key that this row sees, or is none (one whose scores are all NaN has no maximum either, and counts)
      if (m[i] == -INFINITY) continue;
      float e = 1.f;
      if (m[i] > M) {
        const float keep = exp2_approx((M - m[i]) + (r - mr[i]));
        l *= keep;
        acc = make_float4(acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep);
        M = m[i];
        r = mr[i];
      } else {
        e = exp2_approx((m[i] - M) + (mr[i] - r));
      }
      l += ml[i] * e;
      acc = make_float4(acc.x + x[i].x * e, acc.y + x[i].y * e, acc.z + x[i].z * e, acc.w + x[i].w * e);
    }
  }
  const float scale = seen > 0 ? 1.0f / l : 0.f;
  uint16_t* out = p.out.data + token * p.out.token_stride + head * p.out.head_stride + 4 * quad;
  *reinterpret_cast<uint2*>(out) =
      make_uint2(pack2<F16>(acc.x * scale, acc.y * scale), pack2<F16>(acc.z * scale, acc.w * scale));
  if (p.lse && quad == 0) p.lse[token * p.q_heads + head] = l == 0.f ? -INFINITY : ((M + r) + log2f(l)) * 0.69314718055994531f;
}

template <bool F16>
cudaError_t launch(const PromptParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};  // devices whose shared-memory limit is raised
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(prompt_kernel<F16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  e = launch_overlapped(prompt_kernel<F16>, dim3((unsigned)std::min(p.items, device_sms())), kThreads, kSmemBytes, s, p);
  if (e != cudaSuccess || !p.split) return e;
  return launch_overlapped(prompt_join_kernel<F16>, dim3((unsigned)(p.tiles * p.kv_heads * 8), 4), 256, 0, s, p);
}

}  // namespace

cudaError_t launch_prompt(const PromptParams& p, bool f16, cudaStream_t s) {
  return f16 ? launch<true>(p, s) : launch<false>(p, s);
}

}  // namespace hg
