// Attention of packed prompts.
#include "hg_simple.cuh"

namespace hg {
namespace {

template <bool F16>
__global__ void __launch_bounds__(128) prompt_kernel(const __grid_constant__ PromptParams p) {
  grid_launch_dependents();
  grid_dependency_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, h = blockIdx.y;
  const int64_t row = (int64_t)blockIdx.x * 4 + warp;
  int at = 0, i = 0;
  for (; i < p.prompts && at + p.range[i].q_len <= row; ++i) at += p.range[i].q_len;
  if (i == p.prompts) return;
  const PromptRange r = p.range[i];
  const int in_prompt = (int)(row - at), token = r.q0 + in_prompt;
  const float4 q = lane_channels4<F16>(p.q.data + token * p.q.token_stride + h * p.q.head_stride, lane);
  const int seen = p.causal ? max(0, in_prompt + 1 + r.k_len - r.q_len) : r.k_len;
  const int64_t kvh = h / p.group;
  RowState st;
  for (int t = 0; t < seen; ++t)
    attend_key<F16>(st, q, p.scale, p.k.data + (r.k0 + t) * p.k.token_stride + kvh * p.k.head_stride,
                    p.v.data + (r.k0 + t) * p.v.token_stride + kvh * p.v.head_stride, lane);
  store_row<F16>(st, p.out.data + token * p.out.token_stride + h * p.out.head_stride,
                 p.lse ? p.lse + (int64_t)token * p.q_heads + h : nullptr, lane, seen <= 0);
}

}  // namespace

cudaError_t launch_prompt(const PromptParams& p, bool f16, cudaStream_t s) {
  int64_t rows = 0;
  for (int i = 0; i < p.prompts; ++i) rows += p.range[i].q_len;
  if (rows == 0) return cudaSuccess;
  const dim3 grid((unsigned)((rows + 3) / 4), (unsigned)p.q_heads);
  return f16 ? launch_overlapped(prompt_kernel<true>, grid, 128, 0, s, p)
             : launch_overlapped(prompt_kernel<false>, grid, 128, 0, s, p);
}

}  // namespace hg
