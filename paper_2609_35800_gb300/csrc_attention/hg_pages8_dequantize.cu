// Tokens of an 8-bit paged cache as dense 16-bit rows: code * scale, rounded once.
//
// Every code is read once and every entry written once, three bytes an entry, so the kernel is bound by memory.  Eight
// lanes take a token's row of one head, 16 codes a lane in one load and 32 bytes out.  A CTA takes 32 tokens and some of
// the heads' keys and values, so that a token's request and page are looked up once for all of them.
#include "hg_pages8.cuh"

namespace hg {
namespace {

constexpr int kThreads = 256, kTokens = kThreads / 8;
constexpr int kRowsPerCta = 4;  // heads of the keys or the values

template <bool F16>
__global__ void __launch_bounds__(kThreads) pages8_dequantize_kernel(const __grid_constant__ Pages8DequantizeParams p) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int row = blockIdx.x * kTokens + threadIdx.x / 8, c = threadIdx.x % 8;
  if (row >= p.tokens || row < p.begin[0] || row >= p.begin[p.requests]) return;
  int r = 0;  // the last request that begins at the row or before it
  for (int n = p.requests; n > 1;) {
    const int half = n / 2;
    if (p.begin[r + half] <= row) {
      r += half;
      n -= half;
    } else {
      n = half;
    }
  }
  const int token = row - p.begin[r];
  const int page = page_of(p.pool, p.table + (int64_t)r * p.table_stride, p.table_stride, token);
  const int in_page = token & (p.pool.page_size - 1);
  const int parts = p.pool.heads * ((p.k_out.data ? 1 : 0) + (p.v_out.data ? 1 : 0));
#pragma unroll
  for (int i = 0; i < kRowsPerCta; ++i) {
    const int part = blockIdx.y * kRowsPerCta + i;
    if (part >= parts) break;
    const bool is_v = !p.k_out.data || part >= p.pool.heads;
    const int head = part >= p.pool.heads ? part - p.pool.heads : part;
    const Rows& out = is_v ? p.v_out : p.k_out;
    uint4 codes = make_uint4(0u, 0u, 0u, 0u);
    float scale = 0.f;
    if (page >= 0) {
      codes = *reinterpret_cast<const uint4*>((is_v ? p.pool.v : p.pool.k) + code_row(p.pool, page, in_page, head) + 16 * c);
      scale = (is_v ? p.pool.v_scales : p.pool.k_scales)[scale_at(p.pool, page, in_page, head)];
    }
    float x[16];
    decode8(make_uint2(codes.x, codes.y), x);
    decode8(make_uint2(codes.z, codes.w), x + 8);
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = in_range<F16>(x[k] * scale);
    uint16_t* dst = out.data + row * out.token_stride + head * out.head_stride + 16 * c;
    *reinterpret_cast<uint4*>(dst) = pack8<F16>(x);
    *reinterpret_cast<uint4*>(dst + 8) = pack8<F16>(x + 8);
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
