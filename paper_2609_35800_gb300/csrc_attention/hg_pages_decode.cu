// Attention of one new token per request over a paged cache, split over the cache's length and joined.
//
// For a request, KV head and its G queries: s_t = scale q.k_t, m = max s_t, out = sum e^(s_t - m) v_t / sum e^(s_t - m).
// Every key and value is used by G <= 16 queries only, 2 G flop per byte, so the kernel is bound by the reads of the
// cache; it has to keep enough of them in flight and to spread them evenly.
//
// The work is cut into tiles of 64 tokens of one (request, KV head), numbered request by request, head by head.  CTA i
// of n takes the tiles [T i / n, T (i + 1) / n): the same share for everybody whatever the requests' lengths, which the
// kernel reads on the device.  A CTA's run of tiles cuts at most two (request, head) items, its first and its last; it
// leaves their (m, l, o) in the workspace, and the last CTA to arrive at an item (a ticket, no waiting) joins its parts
// in order, so the result does not depend on who comes last.
//
// A producer warp copies tiles into a ring of three 32 KB stages with TMA, a box per page (swizzled rows; a page id
// outside the pool reads as zeros).  Each of four consumer warps takes 16 of a tile's 64 tokens, with its own running
// maximum and sums, and computes with mma.sync m16n8k16 (a tcgen05 product would have M = 128 tokens by N = 8 queries
// and its probabilities would pass through TMEM; the tensor work here is a few per cent of what mma.sync gives):
//   S^T[token][query] = K . q        A = keys (ldmatrix), B = the queries, padded to 8 or 16
//   O^T[channel][query] += V^T . P^T A = values (ldmatrix.trans), B = P^T (movmatrix of the scores' fragment)
// Scores, maxima, sums and outputs are held in 32 bits; probabilities are rounded to the cache's type for the second
// product only.  The running maximum moves when a score passes it by more than 2^8, so probabilities stay below 256.
#include "hg_rows.cuh"
#include "hg_wait.cuh"

namespace hg {
namespace {

constexpr int kTile = kDecodeTile;
constexpr int kStages = 3;
constexpr int kStageBytes = 2 * kTile * kHeadDim * 2;  // keys, then values
constexpr int kConsumers = 4;
constexpr int kThreads = (kConsumers + 1) * 32;
constexpr int kQRowBytes = 272;  // a staged query row: 256 bytes, 16 more so that ldmatrix meets every bank once
constexpr unsigned kAll = 0xffffffffu;
constexpr float kRescale = 8.0f;  // log2 of how far a score may pass the running maximum

// Shared memory from a 1024-byte boundary.  The staged queries (8 rows a warp) and the warps' parts that are added up
// at an item's end (three warps, 8 queries at a time) take turns in one region.
struct Smem {
  static constexpr int scratch = kStages * kStageBytes;
  static constexpr int scratch_bytes = 3 * 8 * (kHeadDim + 2) * 4;  // > 4 * 8 * kQRowBytes
  static constexpr int bars = scratch + ((scratch_bytes + 15) & ~15);
  static constexpr int misc = bars + 2 * kStages * 8;  // abort flag, start of the CTA's work, scan
  static constexpr int bytes = misc + 128 + 1024;
};
static_assert(Smem::scratch_bytes >= kConsumers * 8 * kQRowBytes, "queries are staged there too");

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

__device__ __forceinline__ void next_item(const PagesDecodeParams& p, Cursor& c) {
  c.t = 0;
  if (++c.h < p.pool.heads) return;
  c.h = 0;
  if (++c.b >= p.batch) return;
  c.len = request_length(p, c.b);
  c.tiles = tiles_of(c.len);
}

__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, int row, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], "
      "[%6];\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(head), "r"(page), "r"(bar)
      : "memory");
}

// The tiles [u0, u1) of the launch's `total` that this CTA, one of `ctas` that have any, takes.
struct Work {
  int64_t u0, u1, total, ctas;
  __device__ __forceinline__ int cta_of(int64_t u) const { return (int)(((u + 1) * ctas - 1) / total); }
};

// The CTA's work, and where it begins; false: none.  Every thread adds
// up the tiles of its share of the requests; the one whose share holds u0 looks for it there.
__device__ bool find_work(const PagesDecodeParams& p, int* scan, Work& w, Cursor& c) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int per = (p.batch + kThreads - 1) / kThreads;
  const int b0 = min(tid * per, p.batch), b1 = min(b0 + per, p.batch);
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += tiles_of(request_length(p, b));
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kAll, sum, o);
    if (lane >= o) sum += x;
  }
  if (lane == 31) scan[warp] = sum;
  __syncthreads();
  int before = sum - mine, all = 0;
#pragma unroll
  for (int i = 0; i < kConsumers + 1; ++i) {
    if (i < warp) before += scan[i];
    all += scan[i];
  }
  w.total = (int64_t)all * p.pool.heads;
  w.ctas = min((int64_t)gridDim.x, w.total);
  if (blockIdx.x >= w.ctas) return false;
  w.u0 = w.total * blockIdx.x / w.ctas;
  w.u1 = w.total * (blockIdx.x + 1) / w.ctas;
  const int64_t at = w.u0 - (int64_t)before * p.pool.heads;
  if (at >= 0 && at < (int64_t)mine * p.pool.heads) {
    int64_t left = at;
    int b = b0, len = 0, tiles = 0;
    for (;; ++b) {
      len = request_length(p, b);
      tiles = tiles_of(len);
      if (left < (int64_t)tiles * p.pool.heads) break;
      left -= (int64_t)tiles * p.pool.heads;
    }
    scan[8] = b;
    scan[9] = (int)(left / tiles);
    scan[10] = (int)(left % tiles);
    scan[11] = len;
    scan[12] = tiles;
  }
  __syncthreads();
  c = {scan[8], scan[9], scan[10], scan[11], scan[12]};
  return true;
}

// Copies the CTA's tiles into the ring, in order; returns how many it asked for.
__device__ uint32_t produce(const PagesDecodeParams& p, Cursor c, int64_t units, uint32_t stages, uint32_t full, uint32_t empty,
                        volatile int* abort) {
  const int lane = threadIdx.x % 32;
  const int rows = min(p.pool.page_size, kTile);  // tokens of a box
  const int boxes = kTile / rows;
  const uint32_t box_bytes = (uint32_t)rows * kHeadDim * 2;
  uint32_t n = 0;
  for (; units > 0; next_item(p, c)) {
    const int* ids = p.table + (int64_t)c.b * p.table_stride;
    // 32 page ids at a time, a lane each: that of the 64-token tiles' first box, second, ...
    int first = -1, id = 0;
    for (; c.t < c.tiles && units > 0; ++c.t, --units, ++n) {
      const int box0 = c.t * boxes;  // box number in the item
      const int valid = min(boxes, max(0, (c.len - c.t * kTile + rows - 1) / rows));
      if (first < 0 || box0 + boxes > first + 32) {
        first = box0;
        const int64_t token = (int64_t)(first + lane) * rows;
        id = token < c.len ? ids[token >> p.pool.page_shift] : -1;
      }
      const int s = n % kStages;
      if (n >= kStages && !wait_phase(empty + 8 * s, (n / kStages - 1) & 1, abort, p.status)) return n;
      if (lane == 0) mbar_arrive_expect_tx(full + 8 * s, 2 * valid * box_bytes);
      __syncwarp();
      const int page = __shfl_sync(kAll, id, (box0 - first + lane) & 31);
      if (lane < valid) {
        const int row = ((box0 + lane) * rows) & (p.pool.page_size - 1);
        const uint32_t dst = stages + s * kStageBytes + lane * box_bytes;
        tma_page(dst, &p.k_map, row, c.h, page, full + 8 * s);
        tma_page(dst + kStageBytes / 2, &p.v_map, row, c.h, page, full + 8 * s);
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

// 16 rows of 8 lanes each, rotated: the queries of the item, 8 at a time, as operands of the first product.
template <bool F16, int NT>
__device__ __forceinline__ void load_queries(const PagesDecodeParams& p, int b, int h, uint32_t mine, uint32_t (&qf)[NT][16]) {
  const int lane = threadIdx.x % 32, c = lane % 8;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr);
  LaneAngles g;
  if (at.turns) g = lane_angles(p.rot, c, b);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = lane / 8 + 4 * i, q = nt * 8 + r;
      uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
      if (q < p.group) {
        const uint16_t* src = p.q.data + b * p.q.token_stride + (int64_t)(h * p.group + q) * p.q.head_stride;
        lo = ldg16(src + at.lo);
        hi = ldg16(src + at.hi);
        if (at.turns) rotate_lane<F16>(lo, hi, g, p.rot.interleaved != 0);
      }
      st_shared16(mine + r * kQRowBytes + at.lo * 2, lo);
      st_shared16(mine + r * kQRowBytes + at.hi * 2, hi);
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

// The new token of a decode step: into its page, and over row r of the stage's tile (which may hold what was there).
template <bool F16>
__device__ __forceinline__ void place_new_token(const PagesDecodeParams& p, const Cursor& c, uint32_t kbox, uint32_t vbox,
                                                int rows, int r) {
  const int lane = threadIdx.x % 32;
  if (lane < 16) {
    const int i = lane % 8;
    const bool is_v = lane >= 8;
    const Rows& in = is_v ? p.v : p.k;
    const LaneChannels at = lane_channels(p.rot, i, p.rot.table != nullptr && !is_v);
    const uint16_t* src = in.data + c.b * in.token_stride + c.h * in.head_stride;
    uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
    if (at.turns) rotate_lane<F16>(lo, hi, lane_angles(p.rot, i, c.b), p.rot.interleaved != 0);
    const uint32_t box = is_v ? vbox : kbox;
    st_shared16(box + (at.lo / 64) * rows * 128 + swizzled(r, at.lo / 8 % 8), lo);
    st_shared16(box + (at.hi / 64) * rows * 128 + swizzled(r, at.hi / 8 % 8), hi);
    const int last = c.len - 1;
    const int page = p.table[(int64_t)c.b * p.table_stride + (last >> p.pool.page_shift)];
    if (page >= 0 && page < p.pool.num_pages) {
      uint16_t* dst = (is_v ? p.pool.v : p.pool.k) + page_row(p.pool, page, last & (p.pool.page_size - 1), c.h);
      *reinterpret_cast<uint4*>(dst + at.lo) = lo;
      *reinterpret_cast<uint4*>(dst + at.hi) = hi;
    }
  }
  __syncwarp();
}

// 16 tokens of a tile, of which the first `seen` belong to the request.
template <bool F16, int NT>
__device__ __forceinline__ void attend_slice(const PagesDecodeParams& p, State<NT>& st, const uint32_t (&qf)[NT][16], uint32_t kbox,
                                             uint32_t vbox, int rows, int r0, int seen, float c) {
  const int lane = threadIdx.x % 32;
  float s[NT][4];
  float s2[NT][4];  // two chains of products, one for each half of the channels
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[nt][i] = s2[nt][i] = 0.f;
  const int kr = r0 + lane % 16;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    uint32_t a[4], a2[4];
    ldsm_x4(a, kbox + swizzled(kr, 2 * ks + lane / 16));
    ldsm_x4(a2, kbox + rows * 128 + swizzled(kr, 2 * ks + lane / 16));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mma16<F16>(s[nt], a, qf[nt][2 * ks], qf[nt][2 * ks + 1]);
      mma16<F16>(s2[nt], a2, qf[nt][8 + 2 * ks], qf[nt][8 + 2 * ks + 1]);
    }
  }
  const int g = lane / 4;
  uint32_t pf[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[nt][i] = g + 8 * (i / 2) < seen ? s[nt][i] + s2[nt][i] : -INFINITY;
    float top[2] = {fmaxf(s[nt][0], s[nt][2]), fmaxf(s[nt][1], s[nt][3])};
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
    for (int i = 0; i < 4; ++i) {
      const float m = st.m[nt][i % 2];
      s[nt][i] = exp2_approx((s[nt][i] - (m == -INFINITY ? 0.f : m)) * c);
      st.l[nt][i % 2] += s[nt][i];
    }
    pf[nt][0] = movtrans(pack2<F16>(s[nt][0], s[nt][1]));
    pf[nt][1] = movtrans(pack2<F16>(s[nt][2], s[nt][3]));
  }
  const int vr = r0 + lane % 8 + 8 * (lane / 16);
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    uint32_t a[4];
    ldsm_x4_trans(a, vbox + (d / 4) * rows * 128 + swizzled(vr, 2 * (d % 4) + lane / 8 % 2));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mma16<F16>(st.o[nt][d], a, pf[nt][0], pf[nt][1]);
  }
}

// A CTA's part of the item that begins in its run (`begins`), or of the one that began before it.
__device__ __forceinline__ float* partial_of(const PagesDecodeParams& p, int cta, bool begins) {
  return p.partials + ((int64_t)cta * 2 + (begins ? 1 : 0)) * p.group * kPartialFloats;
}

// out = o / l in the cache's type and the log-sum-exp of a query; a lane has channels 4 lane ..
template <bool F16>
__device__ __forceinline__ void write_query(const PagesDecodeParams& p, int b, int h, int q, float m, float l, const float4& o,
                                            int len, float c) {
  const int lane = threadIdx.x % 32;
  const float r = len > 0 ? 1.0f / l : 0.f;
  const int head = h * p.group + q;
  uint16_t* out = p.out.data + b * p.out.token_stride + head * p.out.head_stride;
  *reinterpret_cast<uint2*>(out + 4 * lane) = make_uint2(pack2<F16>(o.x * r, o.y * r), pack2<F16>(o.z * r, o.w * r));
  if (p.lse && lane == 0) p.lse[(int64_t)b * p.pool.heads * p.group + head] = l == 0.f ? -INFINITY : m * p.scale + logf(l);
}

// The end of the CTA's part of an item: the four warps' sums are added up, 8 queries at a time; a whole item is
// written, a part goes to the workspace, and the last part's CTA joins them all.
template <bool F16, int NT>
__device__ void finish_item(const PagesDecodeParams& p, State<NT>& st, const Cursor& c, bool whole, bool begins,
                            int64_t item_u0, const Work& w, float* scratch, volatile int* misc, float cs) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, tq = lane % 4;
  float* slot = partial_of(p, blockIdx.x, begins);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) st.l[nt][j] += __shfl_xor_sync(kAll, st.l[nt][j], o);
    // [warp][query] m, l and 128 channels
    if (nt > 0) named_barrier<kConsumers * 32>(1);
    float* ml = scratch;
    float* o = scratch + 3 * 8 * 2;
    if (warp > 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = (warp - 1) * 8 + 2 * tq + j;
        if (g == 0) {
          ml[2 * row] = st.m[nt][j];
          ml[2 * row + 1] = st.l[nt][j];
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          o[row * kHeadDim + 16 * d + g] = st.o[nt][d][j];
          o[row * kHeadDim + 16 * d + 8 + g] = st.o[nt][d][2 + j];
        }
      }
    }
    named_barrier<kConsumers * 32>(1);
    if (warp == 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float m = st.m[nt][j], l = 0.f;
        const int q = 2 * tq + j;
#pragma unroll
        for (int w = 0; w < 3; ++w) m = fmaxf(m, ml[2 * (8 * w + q)]);
        const float base = m == -INFINITY ? 0.f : m;
        const float own = exp2_approx((st.m[nt][j] - base) * cs);
        l = st.l[nt][j] * own;
        float e[3];
#pragma unroll
        for (int w = 0; w < 3; ++w) {
          e[w] = exp2_approx((ml[2 * (8 * w + q)] - base) * cs);
          l += ml[2 * (8 * w + q) + 1] * e[w];
        }
        st.m[nt][j] = m;
        st.l[nt][j] = l;
#pragma unroll
        for (int d = 0; d < 8; ++d)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float x = st.o[nt][d][2 * half + j] * own;
#pragma unroll
            for (int w = 0; w < 3; ++w) x += o[(8 * w + q) * kHeadDim + 16 * d + 8 * half + g] * e[w];
            st.o[nt][d][2 * half + j] = x;
          }
      }
      // back through shared memory, so that a query's channels lie side by side
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          o[(2 * tq + j) * kHeadDim + 16 * d + g] = st.o[nt][d][j];
          o[(2 * tq + j) * kHeadDim + 16 * d + 8 + g] = st.o[nt][d][2 + j];
        }
      if (g == 0)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          ml[2 * (2 * tq + j)] = st.m[nt][j];
          ml[2 * (2 * tq + j) + 1] = st.l[nt][j];
        }
    }
    named_barrier<kConsumers * 32>(1);
    for (int q = warp; q < 8 && 8 * nt + q < p.group; q += kConsumers) {
      const float4 x = *reinterpret_cast<const float4*>(o + q * kHeadDim + 4 * lane);
      if (whole) {
        write_query<F16>(p, c.b, c.h, 8 * nt + q, ml[2 * q], ml[2 * q + 1], x, c.len, cs);
      } else {
        float* row = slot + (8 * nt + q) * kPartialFloats;
        *reinterpret_cast<float4*>(row + 4 + 4 * lane) = x;
        if (lane == 0) *reinterpret_cast<float2*>(row) = make_float2(ml[2 * q], ml[2 * q + 1]);
      }
    }
  }
  if (whole) {
    named_barrier<kConsumers * 32>(1);  // the scratch is free again
    return;
  }
  // ticket: the parts before it are visible to the last one
  const int cta0 = w.cta_of(item_u0), cta1 = w.cta_of(item_u0 + c.tiles - 1);
  uint32_t* counter = p.counters + (int64_t)c.b * p.pool.heads + c.h;
  __threadfence();
  named_barrier<kConsumers * 32>(1);
  if (threadIdx.x == 0) {
    const uint32_t before = atomicAdd(counter, 1u);
    misc[1] = before == (uint32_t)(cta1 - cta0);
    if (misc[1]) *counter = 0u;
    __threadfence();
  }
  named_barrier<kConsumers * 32>(1);
  if (!misc[1]) return;
  __threadfence();
  for (int q = warp; q < p.group; q += kConsumers) {
    float m = -INFINITY;
    for (int i = cta0 + lane; i <= cta1; i += 32) {
      m = fmaxf(m, __ldcg(partial_of(p, i, i == cta0) + q * kPartialFloats));
    }
    m = warp_max(m);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = cta0; i <= cta1; ++i) {
      const float* row = partial_of(p, i, i == cta0) + q * kPartialFloats;
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(row));
      const float4 x = __ldcg(reinterpret_cast<const float4*>(row + 4) + lane);
      const float e = exp2_approx((ml.x - base) * cs);
      l += ml.y * e;
      acc.x += x.x * e;
      acc.y += x.y * e;
      acc.z += x.z * e;
      acc.w += x.w * e;
    }
    write_query<F16>(p, c.b, c.h, q, m, l, acc, c.len, cs);
  }
}

template <bool F16, int NT>
__device__ void consume(const PagesDecodeParams& p, Cursor c, const Work& w, uint32_t base, char* smem, volatile int* misc) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = base + Smem::bars, empty = full + 8 * kStages;
  const int rows = min(p.pool.page_size, kTile);
  const float cs = p.scale * kLog2e;
  float* scratch = reinterpret_cast<float*>(smem + Smem::scratch);
  uint32_t n = 0;
  bool alive = true;  // false: a wait ran out, and the warp only keeps up with the others' barriers
  for (int64_t u = w.u0; u < w.u1; next_item(p, c)) {
    const int64_t item_u0 = u - c.t;
    const bool begins = item_u0 >= w.u0, whole = c.t == 0 && u + c.tiles <= w.u1;
    uint32_t qf[NT][16];
    load_queries<F16, NT>(p, c.b, c.h, base + Smem::scratch + warp * 8 * kQRowBytes, qf);
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
    for (; c.t < c.tiles && u < w.u1; ++c.t, ++u, ++n) {
      const int s = n % kStages;
      alive = alive && wait_phase(full + 8 * s, (n / kStages) & 1, misc, p.status);
      const uint32_t kt = base + s * kStageBytes, vt = kt + kStageBytes / 2;
      const int t0 = 16 * warp, seen = c.len - c.t * kTile - t0;  // of this warp's 16 tokens
      if (alive && seen > 0) {
        const uint32_t box = (uint32_t)(t0 / rows) * rows * kHeadDim * 2;
        const int r0 = t0 % rows;
        if (seen < 16) {
          // what follows the request's last token may be anything, and 0 times NaN is no 0
          for (int i = seen * 16 + lane; i < 256; i += 32) {
            const int r = r0 + i / 16, chunk = i % 16;
            st_shared16(vt + box + (chunk / 8) * rows * 128 + swizzled(r, chunk % 8), make_uint4(0u, 0u, 0u, 0u));
          }
        }
        if (seen <= 16 && p.store) place_new_token<F16>(p, c, kt + box, vt + box, rows, r0 + seen - 1);
        __syncwarp();
        attend_slice<F16, NT>(p, st, qf, kt + box, vt + box, rows, r0, seen, cs);
        if (seen <= 16) fence_proxy_async_shared();  // TMA writes the stage again
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + 8 * s);
    }
    --c.t;  // the item's last tile of this run
    named_barrier<kConsumers * 32>(1);  // every warp has read its queries from the scratch
    finish_item<F16, NT>(p, st, c, whole, begins, item_u0, w, scratch, misc, cs);
  }
}

template <bool F16, int NT>
__global__ void __launch_bounds__(kThreads, 2) pages_decode_kernel(const __grid_constant__ PagesDecodeParams p) {
  extern __shared__ char raw[];
  char* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  const uint32_t base = smem_u32(smem), full = base + Smem::bars, empty = full + 8 * kStages;
  volatile int* misc = reinterpret_cast<int*>(smem + Smem::misc);  // [0] abort, [1] last part, [8 ..] scan
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, kConsumers);
    }
    mbar_init_fence();
    misc[0] = 0;
  }
  __syncthreads();
  grid_launch_dependents();
  grid_dependency_wait();
  Work w;
  Cursor c;
  if (!find_work(p, const_cast<int*>(misc) + 8, w, c)) return;
  uint32_t asked = 0;
  if (threadIdx.x / 32 == kConsumers) {
    fence_proxy_async_global();  // pages written by ordinary stores of earlier launches
    asked = produce(p, c, w.u1 - w.u0, base, full, empty, misc);
  } else {
    consume<F16, NT>(p, c, w, base, smem, misc);
  }
  __syncthreads();
  if (misc[0]) {  // a CTA that gave up leaves once the copies it asked for have landed
    for (uint32_t n = asked > kStages ? asked - kStages : 0; n < asked; ++n)
      for (uint32_t i = 0; i < kAsyncRounds && !mbar_try_wait_sleep(full + 8 * (n % kStages), (n / kStages) & 1, kAsyncSleepNs); ++i) {
      }
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
