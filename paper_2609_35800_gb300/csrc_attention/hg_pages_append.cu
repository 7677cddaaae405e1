// New tokens into a paged cache, with the position rotation on the way.
//
// Pair (a, b) of a query or key row turned by its angle t: (a cos t - b sin t, b cos t + a sin t); values are copied.
// Nothing is used twice but a token's cosines and sines, so the kernel is bound by memory: every row is read once and
// written once (a key that is wanted densely too, twice).  Eight lanes take a row, 16 channels each in two 16-byte
// loads, both halves of a pair in one lane; rows are numbered token by token (queries, keys, values), so a block's
// lanes share a token's cosines and sines through L1.  Measured: 21,400 tokens of 60 + 5 + 5 heads 148 us, 6.25 TB/s,
// 0.92 of a copy's rate (two rows a thread: 150 us); 1,460 tokens of 28 + 4 + 4 heads 5.1 us on the device.
#include "hg_rows.cuh"

namespace hg {
namespace {

constexpr int kAppendThreads = 256;

template <bool F16>
__global__ void __launch_bounds__(kAppendThreads) pages_append_kernel(const __grid_constant__ PagesAppendParams p) {
  grid_launch_dependents();
  const int rows = p.q_heads + 2 * p.pool.heads;
  const int64_t item = (int64_t)blockIdx.x * (kAppendThreads / 8) + threadIdx.x / 8;
  const int c = threadIdx.x % 8;
  const int token = (int)(item / rows);
  if (token >= p.tokens) return;
  const int row = (int)(item - (int64_t)token * rows);
  grid_dependency_wait();

  const bool is_q = row < p.q_heads, is_v = row >= p.q_heads + p.pool.heads;
  const int head = is_q ? row : is_v ? row - p.q_heads - p.pool.heads : row - p.q_heads;
  const Rows& in = is_q ? p.q : is_v ? p.v : p.k;
  const Rows& out = is_q ? p.q_out : is_v ? p.v_out : p.k_out;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr && !is_v);

  const uint16_t* src = in.data + token * in.token_stride + head * in.head_stride;
  uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
  if (at.turns) rotate_lane<F16>(lo, hi, lane_angles(p.rot, c, token), p.rot.interleaved != 0);
  if (out.data) {
    uint16_t* dst = out.data + token * out.token_stride + head * out.head_stride;
    *reinterpret_cast<uint4*>(dst + at.lo) = lo;
    *reinterpret_cast<uint4*>(dst + at.hi) = hi;
  }
  if (is_q) return;
  const int slot = p.slots[token];
  const int page = slot >> p.pool.page_shift;
  if (slot < 0 || page >= p.pool.num_pages) return;
  uint16_t* dst = (is_v ? p.pool.v : p.pool.k) + page_row(p.pool, page, slot & (p.pool.page_size - 1), head);
  *reinterpret_cast<uint4*>(dst + at.lo) = lo;
  *reinterpret_cast<uint4*>(dst + at.hi) = hi;
}

}  // namespace

cudaError_t launch_pages_append(const PagesAppendParams& p, bool f16, cudaStream_t s) {
  const int64_t rows = (int64_t)p.tokens * (p.q_heads + 2 * p.pool.heads);
  const int64_t blocks = (rows + kAppendThreads / 8 - 1) / (kAppendThreads / 8);
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks);
  return f16 ? launch_overlapped(pages_append_kernel<true>, grid, kAppendThreads, 0, s, p)
             : launch_overlapped(pages_append_kernel<false>, grid, kAppendThreads, 0, s, p);
}

}  // namespace hg
