// New tokens into an 8-bit paged cache, with the position rotation on the way.
//
// A block is 16 tokens of one head.  Its scale s is a power of two, max(the least with amax <= 448 s over the new tokens'
// entries, the one of the tokens it has); code = e4m3(x / s).  A scale needs the whole block's entries before any code, so
// a CTA takes the new tokens of one block, KV head and of the keys or the values: 16 rows, eight lanes each, 16 channels a
// lane as hg_pages_append has them, whose largest entry passes through shared memory once.  The rows stay in registers,
// so everything is read once and written once, and the kernel is bound by memory.  The other CTAs turn queries, two heads
// of a token by eight lanes.  Measured: 21,400 tokens of 60 + 5 + 5 heads 142 us, 6.3 TB/s, 0.93 of a copy's rate (one
// head by eight lanes 161 us, four 147, six 154); 1,460 tokens of 28 + 4 + 4 heads 4.8 us on the device, 16 of one token
// each 2.7.
//
// Which blocks a launch touches is known on the device only.  Request r with n new tokens touches at most n / 16 + 2 of
// them; numbered from (begin[r] - begin[0]) / 16 + 2 r on, no two requests' numbers meet, and a CTA finds its request by
// a search in begin alone.  Numbers without a block end at once.
#include "hg_pages8.cuh"

namespace hg {
namespace {

constexpr int kThreads = 128;  // 16 rows
constexpr int kQueries = kAppend8Queries;
constexpr unsigned kAll = 0xffffffffu;

// begin[r], whatever lies there, within the call's rows.
__device__ __forceinline__ int begin_of(const Pages8AppendParams& p, int r) { return min(max(p.begin[r], 0), p.tokens); }

// The request that unit u belongs to: the last whose first unit is not above it.  32 candidates a round, a lane each.
__device__ int request_of(const Pages8AppendParams& p, int u, int begin0) {
  const int lane = threadIdx.x % 32;
  int lo = 0, n = p.requests;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, r = lo + lane * step;
    const bool below = lane * step < n && ((begin_of(p, r) - begin0) >> kBlock8Shift) + 2 * r <= u;
    const int count = __popc(__ballot_sync(kAll, below));
    const int k = max(count - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// kQueries heads of a token by eight lanes: their reads are in flight together, and the token's cosines and sines, its
// number and whether it is any request's are found out once.
template <bool F16>
__device__ __forceinline__ void turn_queries(const Pages8AppendParams& p, uint32_t cta) {
  const uint32_t parts = (p.q_heads + kQueries - 1) / kQueries, item = cta * (kThreads / 8) + threadIdx.x / 8;
  const uint32_t at_token = item / parts;
  if (at_token >= (uint32_t)p.tokens) return;
  const int token = (int)at_token, head = (int)(item - at_token * parts) * kQueries, c = threadIdx.x % 8;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr);
  const uint16_t* src = p.q.data + token * p.q.token_stride + head * p.q.head_stride;
  uint4 lo[kQueries], hi[kQueries];
#pragma unroll
  for (int i = 0; i < kQueries; ++i) {
    if (head + i >= p.q_heads) break;
    lo[i] = ldg16(src + i * p.q.head_stride + at.lo);
    hi[i] = ldg16(src + i * p.q.head_stride + at.hi);
  }
  LaneAngles angles;
  if (at.turns) angles = lane_angles(p.rot, c, token);
  if (token < p.begin[0] || token >= p.begin[p.requests]) return;
  uint16_t* dst = p.q_out.data + token * p.q_out.token_stride + head * p.q_out.head_stride;
#pragma unroll
  for (int i = 0; i < kQueries; ++i) {
    if (head + i >= p.q_heads) break;
    if (at.turns) rotate_lane<F16>(lo[i], hi[i], angles, p.rot.interleaved != 0);
    *reinterpret_cast<uint4*>(dst + i * p.q_out.head_stride + at.lo) = lo[i];
    *reinterpret_cast<uint4*>(dst + i * p.q_out.head_stride + at.hi) = hi[i];
  }
}

template <bool F16>
__global__ void __launch_bounds__(kThreads) pages8_append_kernel(const __grid_constant__ Pages8AppendParams p) {
  __shared__ uint32_t tops[kThreads / 32];
  grid_launch_dependents();
  grid_dependency_wait();
  if ((int)blockIdx.x >= p.kv_ctas) {
    turn_queries<F16>(p, blockIdx.x - p.kv_ctas);
    return;
  }
  const int unit = blockIdx.x / (2 * p.pool.heads), part = blockIdx.x - unit * 2 * p.pool.heads;
  const bool is_v = part >= p.pool.heads;
  const int head = is_v ? part - p.pool.heads : part;
  const int begin0 = begin_of(p, 0), r = request_of(p, unit, begin0);
  const int row0 = begin_of(p, r), rows = begin_of(p, r + 1) - row0;
  const int start = p.lengths[r] - rows;  // of the new tokens, in the request
  // the block, the thread's token of it and that one's row
  const int block = (start >> kBlock8Shift) + unit - (((row0 - begin0) >> kBlock8Shift) + 2 * r);
  const int first = block << kBlock8Shift, mine = first + (int)threadIdx.x / 8;
  if (rows <= 0 || first >= start + rows) return;
  const int row = row0 + mine - start;
  const bool is_new = mine >= start && mine < start + rows, is_old = mine < start;
  const int page = page_of(p.pool, p.table + (int64_t)r * p.table_stride, p.table_stride, mine);

  const int c = threadIdx.x % 8;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr && !is_v);
  const Rows &in = is_v ? p.v : p.k, &out = is_v ? p.v_out : p.k_out;
  float x[16];
  uint32_t top = 0;
  if (is_new) {
    const uint16_t* src = in.data + row * in.token_stride + head * in.head_stride;
    const uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
    LaneAngles angles;
    if (at.turns) angles = lane_angles(p.rot, c, row);
    row_values<F16>(lo, hi, at.turns ? &angles : nullptr, p.rot.interleaved != 0, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, finite_bits(x[i]));
    if (out.data) {
      uint16_t* dst = out.data + row * out.token_stride + head * out.head_stride;
      *reinterpret_cast<uint4*>(dst + at.lo) = pack8<F16>(x);
      *reinterpret_cast<uint4*>(dst + at.hi) = pack8<F16>(x + 8);
    }
  }
  // a page starts on a block's first token: the whole block has one page
  float* scale = (is_v ? p.pool.v_scales : p.pool.k_scales) + scale_at(p.pool, max(page, 0), first & (p.pool.page_size - 1), head);
  uint8_t* codes = (is_v ? p.pool.v : p.pool.k) + code_row(p.pool, max(page, 0), mine & (p.pool.page_size - 1), head);
  const float before = page >= 0 && first < start ? *scale : 0.f;
  top = __reduce_max_sync(kAll, top);
  if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
  __syncthreads();
  if (page < 0) return;
  int field = needed_field(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  if (first < start) field = max(field, stored_field(before));
  const float after = power_of_field(field);
  if (threadIdx.x == 0) *scale = after;
  if (is_new) {
    const float inv = inverse_of_field(field);
    *reinterpret_cast<uint2*>(codes + at.lo) = encode8(x, inv);
    *reinterpret_cast<uint2*>(codes + at.hi) = encode8(x + 8, inv);
  } else if (is_old && before != after) {
    uint2* at8 = reinterpret_cast<uint2*>(codes + 16 * c);
    const float ratio = before / after;
    at8[0] = recode8(at8[0], ratio);
    at8[1] = recode8(at8[1], ratio);
  }
}

}  // namespace

cudaError_t launch_pages8_append(const Pages8AppendParams& p, bool f16, cudaStream_t s) {
  Pages8AppendParams a = p;
  int64_t kv = 0, q = 0;
  if (!append8_grid(p.tokens, p.requests, p.q_heads, p.pool.heads, &kv, &q)) return cudaErrorInvalidConfiguration;
  a.kv_ctas = (int)kv;
  const dim3 grid((unsigned)(kv + q));
  return f16 ? launch_overlapped(pages8_append_kernel<true>, grid, kThreads, 0, s, a)
             : launch_overlapped(pages8_append_kernel<false>, grid, kThreads, 0, s, a);
}

}  // namespace hg
