// Attention of one new token per request over a paged cache.
#include "hg_simple.cuh"

namespace hg {
namespace {

// The new tokens' keys, rotated, and values into their pages (8 lanes a row, as in the append).
template <bool F16>
__global__ void __launch_bounds__(256) pages_store_kernel(const __grid_constant__ PagesDecodeParams p) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int item = blockIdx.x * 32 + threadIdx.x / 8, c = threadIdx.x % 8;
  const int b = item / (2 * p.pool.heads), row = item - b * 2 * p.pool.heads;
  if (b >= p.batch) return;
  const bool is_v = row >= p.pool.heads;
  const int head = is_v ? row - p.pool.heads : row;
  const Rows& in = is_v ? p.v : p.k;
  const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr && !is_v);
  const uint16_t* src = in.data + b * in.token_stride + head * in.head_stride;
  uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
  if (at.turns) rotate_lane<F16>(lo, hi, lane_angles(p.rot, c, b), p.rot.interleaved != 0);
  const int last = min(p.lengths[b], p.table_stride * p.pool.page_size) - 1;
  if (last < 0) return;
  const int page = p.table[(int64_t)b * p.table_stride + (last >> p.pool.page_shift)];
  if (page < 0 || page >= p.pool.num_pages) return;
  uint16_t* dst = (is_v ? p.pool.v : p.pool.k) + page_row(p.pool, page, last & (p.pool.page_size - 1), head);
  *reinterpret_cast<uint4*>(dst + at.lo) = lo;
  *reinterpret_cast<uint4*>(dst + at.hi) = hi;
}

template <bool F16>
__global__ void __launch_bounds__(128) pages_decode_kernel(const __grid_constant__ PagesDecodeParams p) {
  __shared__ __align__(16) uint16_t rows[4][2][kHeadDim];  // the query; the new token's key
  grid_launch_dependents();
  grid_dependency_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int heads = p.pool.heads * p.group;
  const int item = blockIdx.x * 4 + warp;
  const int b = item / heads, h = item - b * heads;
  if (b >= p.batch) return;
  const int kvh = h / p.group;
  if (lane < (p.store ? 16 : 8)) {
    const int c = lane % 8;
    const LaneChannels at = lane_channels(p.rot, c, p.rot.table != nullptr);
    const uint16_t* src = lane < 8 ? p.q.data + b * p.q.token_stride + h * p.q.head_stride
                                   : p.k.data + b * p.k.token_stride + kvh * p.k.head_stride;
    uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
    if (at.turns) rotate_lane<F16>(lo, hi, lane_angles(p.rot, c, b), p.rot.interleaved != 0);
    *reinterpret_cast<uint4*>(rows[warp][lane / 8] + at.lo) = lo;
    *reinterpret_cast<uint4*>(rows[warp][lane / 8] + at.hi) = hi;
  }
  __syncwarp();
  const float4 q = lane_channels4<F16>(rows[warp][0], lane);
  const int len = min(p.lengths[b], p.table_stride * p.pool.page_size);
  __shared__ __align__(16) uint16_t zero[kHeadDim];
  zero[threadIdx.x] = 0;
  __syncwarp();
  RowState st;
  for (int t = 0; t < len; ++t) {
    if (p.store && t == len - 1) {
      attend_key<F16>(st, q, p.scale, rows[warp][1], p.v.data + b * p.v.token_stride + kvh * p.v.head_stride, lane);
      break;
    }
    const int page = p.table[(int64_t)b * p.table_stride + (t >> p.pool.page_shift)];
    const bool inside = page >= 0 && page < p.pool.num_pages;
    const int64_t row = inside ? page_row(p.pool, page, t & (p.pool.page_size - 1), kvh) : 0;
    attend_key<F16>(st, q, p.scale, inside ? p.pool.k + row : zero, inside ? p.pool.v + row : zero, lane);
  }
  store_row<F16>(st, p.out.data + b * p.out.token_stride + h * p.out.head_stride,
                 p.lse ? p.lse + (int64_t)b * heads + h : nullptr, lane, len <= 0);
}

template <bool F16>
cudaError_t launch(const PagesDecodeParams& p, cudaStream_t s) {
  if (p.store) {
    const int items = p.batch * 2 * p.pool.heads;
    const cudaError_t e = launch_overlapped(pages_store_kernel<F16>, dim3((items + 31) / 32), 256, 0, s, p);
    if (e != cudaSuccess) return e;
  }
  const int items = p.batch * p.pool.heads * p.group;
  return launch_overlapped(pages_decode_kernel<F16>, dim3((items + 3) / 4), 128, 0, s, p);
}

}  // namespace

cudaError_t launch_pages_decode(const PagesDecodeParams& p, bool f16, cudaStream_t s) {
  return f16 ? launch<true>(p, s) : launch<false>(p, s);
}

}  // namespace hg
