// Tokens of an 8-bit paged cache as dense 16-bit rows: code * scale, rounded once.
//
// Every code is read once and every entry written once, three bytes an entry, so the kernel is bound by memory.  Eight
// lanes take a token's row of one head, 16 codes a lane in one load and 32 bytes out.  A CTA takes 32 tokens and four of
// the heads' keys and values, so that a token's request and page are looked up once for all of them, and reads all four
// rows before it stores the first.  Measured: 24 requests of 1 to 8,577 tokens, 8 heads 26.8 us, 6.05 TB/s, 0.89 of a
// copy's rate (31 us with the stores between the reads and a clamp for every entry); 16,064 tokens of 4 heads 8.0 us.
#include "hg_pages8.cuh"

namespace hg {
namespace {

constexpr int kThreads = 256, kTokens = kThreads / 8;
constexpr int kRowsPerCta = 4;  // heads of the keys or the values

// The last request that begins at the row or before it, 32 candidates a round; the first where none does.
__device__ __forceinline__ int request_of(const Pages8DequantizeParams& p, int row) {
  const int lane = threadIdx.x % 32;
  int r = 0;
  for (int n = p.requests; n > 1;) {
    const int step = (n + 31) / 32;
    const bool below = lane * step < n && p.begin[r + lane * step] <= row;
    const int k = max(__popc(__ballot_sync(0xffffffffu, below)) - 1, 0);
    r += k * step;
    n = min(step, n - k * step);
  }
  return r;
}

// code * scale towards zero, its last bit set where something is left: rounding that to 16 bits rounds the product itself,
// 28 bits of it, once (24 requests of 8,577 tokens, 8 heads: 197 us, 187 with powers of two).  What is left is found 2^24
// higher where it could be below binary32's end.
__device__ __forceinline__ float product_to_odd(float code, float scale) {
  const float x = __fmul_rz(code, scale), lift = scale < 1.f ? 0x1p24f : 1.f;
  const bool more = __fmaf_rn(code, scale * lift, -(x * lift)) != 0.f;
  return more ? __uint_as_float(__float_as_uint(x) | 1u) : x;
}

template <bool F16>
__global__ void __launch_bounds__(kThreads) pages8_dequantize_kernel(const __grid_constant__ Pages8DequantizeParams p) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int row0 = blockIdx.x * kTokens + threadIdx.x / 32 * 4;  // of the warp
  const int row = row0 + threadIdx.x % 32 / 8, c = threadIdx.x % 8;
  int r = request_of(p, row0);
  if (r + 1 < p.requests && p.begin[r + 1] <= row) {  // a later one than the warp's first row's
    ++r;
    for (int n = p.requests - r; n > 1;) {
      const int half = n / 2;
      const bool right = p.begin[r + half] <= row;
      r += right ? half : 0;
      n = right ? n - half : half;
    }
  }
  if (row >= p.tokens || row < p.begin[0] || row >= p.begin[p.requests]) return;
  const int token = row - p.begin[r];
  const int page = page_of(p.pool, p.table + (int64_t)r * p.table_stride, p.table_stride, token);
  const int in_page = token & (p.pool.page_size - 1);
  const int parts = p.pool.heads * ((p.k_out.data ? 1 : 0) + (p.v_out.data ? 1 : 0));
  uint4 codes[kRowsPerCta];
  float scale[kRowsPerCta];
#pragma unroll
  for (int i = 0; i < kRowsPerCta; ++i) {  // every read before the first store
    const int part = blockIdx.y * kRowsPerCta + i;
    const bool is_v = !p.k_out.data || part >= p.pool.heads;
    const int head = part >= p.pool.heads ? part - p.pool.heads : part;
    codes[i] = make_uint4(0u, 0u, 0u, 0u);
    scale[i] = 0.f;
    if (part >= parts || page < 0) continue;
    codes[i] = ldg16((is_v ? p.pool.v : p.pool.k) + code_row(p.pool, page, in_page, head) + 16 * c);
    scale[i] = (is_v ? p.pool.v_scales : p.pool.k_scales)[scale_at(p.pool, page, in_page, head)];
  }
#pragma unroll
  for (int i = 0; i < kRowsPerCta; ++i) {
    const int part = blockIdx.y * kRowsPerCta + i;
    if (part >= parts) break;
    const bool is_v = !p.k_out.data || part >= p.pool.heads;
    const int head = part >= p.pool.heads ? part - p.pool.heads : part;
    const Rows& out = is_v ? p.v_out : p.k_out;
    float x[16];
    decode8(make_uint2(codes[i].x, codes[i].y), x);
    decode8(make_uint2(codes[i].z, codes[i].w), x + 8);
    if ((__float_as_uint(scale[i]) & 0x7fffffu) == 0) {  // a power of two: exact
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] *= scale[i];
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = product_to_odd(x[k], scale[i]);
    }
    if (!(scale[i] * 448.f <= kMost16<F16>)) {  // the largest code would be out of the type's range
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = in_range<F16>(x[k]);
    }
    uint16_t* dst = out.data + row * out.token_stride + head * out.head_stride + 16 * c;
    store16(dst, pack8<F16>(x), pack8<F16>(x + 8));
  }
}

}  // namespace

cudaError_t launch_pages8_dequantize(const Pages8DequantizeParams& p, bool f16, cudaStream_t s) {
  const int parts = p.pool.heads * ((p.k_out.data ? 1 : 0) + (p.v_out.data ? 1 : 0));
  const dim3 grid((unsigned)((p.tokens + (int64_t)kTokens - 1) / kTokens), (unsigned)((parts + kRowsPerCta - 1) / kRowsPerCta));
  return f16 ? launch_overlapped(pages8_dequantize_kernel<true>, grid, kThreads, 0, s, p)
             : launch_overlapped(pages8_dequantize_kernel<false>, grid, kThreads, 0, s, p);
}

}  // namespace hg
