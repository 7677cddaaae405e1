// Attention of one new token per request over an 8-bit paged cache.
//
// For a request, KV head and its G queries: S_t = scale ks q.c_t with the key block's scale ks, m = max S_t, out = sum e^(S_t
// - m) vs c'_t / sum e^(S_t - m) with the value block's scale vs.  A warp takes a request's query head and goes through its
// tokens one by one with a running maximum and sum, four channels a lane.
#include "hg_pages8.cuh"

namespace hg {
namespace {

constexpr int kThreads = 128;
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
  return x;
}

// The row of a head, turned, four channels a lane, through shared memory; 16 channels of it in lanes below 8.
template <bool F16>
__device__ __forceinline__ void load_row(const Rows& rows, const Rotation& rot, bool turns, int b, int head, float* staged,
                                         bool rounded, float (&x)[4]) {
  const int lane = threadIdx.x % 32;
  if (lane < 8) {
    const LaneChannels at = lane_channels(rot, lane, turns && rot.table != nullptr);
    const uint16_t* src = rows.data + b * rows.token_stride + head * rows.head_stride;
    const uint4 lo = ldg16(src + at.lo), hi = ldg16(src + at.hi);
    LaneAngles angles;
    if (at.turns) angles = lane_angles(rot, lane, b);
    float v[16];
    row_values<F16>(lo, hi, at.turns ? &angles : nullptr, rot.interleaved != 0, v);
    for (int i = 0; i < 16; ++i) {
      if (rounded) {
        const float2 f = unpack2<F16>(pack2<F16>(v[i], 0.f));
        v[i] = f.x;
      }
      staged[(i < 8 ? at.lo + i : at.hi + i - 8)] = v[i];
    }
  }
  __syncwarp();
  for (int i = 0; i < 4; ++i) x[i] = staged[4 * lane + i];
  __syncwarp();
}

// The row as a block of its own holds it.
__device__ __forceinline__ void held(float (&x)[4]) {
  uint32_t top = 0;
  for (int i = 0; i < 4; ++i) top = max(top, finite_bits(x[i]));
  const int field = needed_field(__reduce_max_sync(kAll, top));
  const float inv = inverse_of_field(field), s = power_of_field(field);
  for (int i = 0; i < 4; i += 2) {
    const float2 f = half2_bits_to_float2(decode2(encode2(x[i], x[i + 1], inv)));
    x[i] = f.x * s;
    x[i + 1] = f.y * s;
  }
}

template <bool F16>
__global__ void __launch_bounds__(kThreads) pages8_decode_kernel(const __grid_constant__ Pages8DecodeParams p) {
  __shared__ float staged[kThreads / 32][128];
  grid_launch_dependents();
  grid_dependency_wait();
  const int item = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, lane = threadIdx.x % 32;
  const int heads = p.group * p.pool.heads;
  const int b = item / heads, qh = item - b * heads, h = qh / p.group;
  if (b >= p.batch) return;
  float* mine = staged[threadIdx.x / 32];
  const int cap = p.table_stride << p.pool.page_shift, given = p.lengths[b], len = min(max(given, 0), cap);
  const int* table = p.table + (int64_t)b * p.table_stride;
  float q[4];
  load_row<F16>(p.q, p.rot, true, b, qh, mine, true, q);
  float m = -INFINITY, l = 0.f, o[4] = {};
  for (int t = 0; t < len; ++t) {
    const int page = page_of(p.pool, table, p.table_stride, t), at = t & (p.pool.page_size - 1);
    float k[4] = {}, v[4] = {};
    if (page >= 0) {
      const int64_t row = code_row(p.pool, page, at, h) + 4 * lane, block = scale_at(p.pool, page, at, h);
      const uint32_t kc = *reinterpret_cast<const uint32_t*>(p.pool.k + row), vc = *reinterpret_cast<const uint32_t*>(p.pool.v + row);
      const float ks = p.pool.k_scales[block], vs = p.pool.v_scales[block];
      for (int i = 0; i < 4; i += 2) {
        const float2 a = half2_bits_to_float2(decode2(kc >> 8 * i & 0xffffu)), c = half2_bits_to_float2(decode2(vc >> 8 * i & 0xffffu));
        k[i] = a.x * ks;
        k[i + 1] = a.y * ks;
        v[i] = c.x * vs;
        v[i + 1] = c.y * vs;
      }
    } else if (p.store && t == given - 1) {  // it has no block to be in
      load_row<F16>(p.k, p.rot, true, b, h, mine, false, k);
      load_row<F16>(p.v, p.rot, false, b, h, mine, false, v);
      held(k);
      held(v);
    }
    const float s = warp_sum(q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3]) * p.scale;
    const float top = fmaxf(m, s), keep = expf(m - top), e = expf(s - top);
    m = top;
    l = l * keep + e;
    for (int i = 0; i < 4; ++i) o[i] = o[i] * keep + e * v[i];
  }
  const float r = len > 0 ? 1.f / l : 0.f;
  uint16_t* out = p.out.data + b * p.out.token_stride + qh * p.out.head_stride + 4 * lane;
  for (int i = 0; i < 4; ++i) o[i] = in_range<F16>(o[i] * r);
  *reinterpret_cast<uint2*>(out) = make_uint2(pack2<F16>(o[0], o[1]), pack2<F16>(o[2], o[3]));
  if (p.lse && lane == 0) p.lse[(int64_t)b * heads + qh] = len > 0 ? m + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t launch_pages8_decode(const Pages8DecodeParams& p, bool f16, cudaStream_t s) {
  if (p.store) {
    Pages8AppendParams a = {};
    a.pool = p.pool;
    a.rot = p.rot;
    a.tokens = a.requests = p.batch;
    a.k = p.k;
    a.v = p.v;
    a.table = p.table;
    a.table_stride = p.table_stride;
    a.lengths = p.lengths;
    const cudaError_t e = launch_pages8_append(a, f16, s);
    if (e != cudaSuccess) return e;
  }
  const int64_t warps = (int64_t)p.batch * p.group * p.pool.heads, blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks);
  return f16 ? launch_overlapped(pages8_decode_kernel<true>, grid, kThreads, 0, s, p)
             : launch_overlapped(pages8_decode_kernel<false>, grid, kThreads, 0, s, p);
}

}  // namespace hg
