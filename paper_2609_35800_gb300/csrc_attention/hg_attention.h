// Launch parameters and launchers shared by the host code and the kernels of the 16-bit caches: paged append, paged
// decode attention and prompt attention.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "../../include/headguard.h"

namespace hg {

constexpr int kHeadDim = 128;
constexpr int kMaxGroup = 16;
constexpr int kMaxKvHeads = 64;
constexpr size_t kAttnHeaderBytes = 512;  // workspace header: status word at byte 0, as the packed cache's has
constexpr float kLog2e = 1.4426950408889634f;

// hg_rows as the kernels take them.
struct Rows {
  uint16_t* data;
  int64_t token_stride, head_stride;
};
inline Rows rows_of(const hg_rows& r) { return {static_cast<uint16_t*>(r.data), r.token_stride, r.head_stride}; }

struct Rotation {
  const float* table;  // null: no rotation
  int table_len, half;  // half = rot_dim / 2
  int interleaved;
  int end0, end1;  // first pair of the second and of the third position; both `half` with one position a token
  const int* positions;
  int position_stride;  // tokens: distance between a token's first, second and third position
};

struct PagePool {
  uint16_t *k, *v;
  int num_pages, page_size, page_shift, heads;
  int64_t page_stride, head_stride, token_stride;
};

struct PagesAppendParams {
  PagePool pool;
  Rotation rot;
  int tokens, q_heads;
  Rows q, k, v, q_out, k_out, v_out;
  const int* slots;
};

// Tokens of a tile of the paged decode; a tensor map's box covers a tile of one page, or the page where that is smaller.
constexpr int kDecodeTile = 32;
constexpr int kDecodeItemCost = 12;  // fixed costs of a (request, KV head), in tiles
// Parts of an item over many CTAs are joined 16 CTAs at a time first; two counters for each 16, ahead of the items' ones.
constexpr int kDecodeJoinCtas = 16, kDecodeJoinCounters = 128;
// A query's part in the workspace: m, l, two unused, 128 channels.
constexpr int kPartialFloats = kHeadDim + 4;

struct PagesDecodeParams {
  CUtensorMap k_map, v_map;  // the pool as [pages][heads][2][page_size][64 channels]
  PagePool pool;
  Rotation rot;
  int batch, group;
  int store;  // a decode step: k, v hold the new token, which is stored
  Rows q, k, v, out;
  const int* table;
  int table_stride;
  const int* lengths;
  float* lse;
  float scale;
  uint32_t* status;
  uint32_t* counters;  // kDecodeJoinCounters, then [batch][heads]; zero between launches
  float* partials;
};

// Prompts of one launch (they travel in its parameters).
constexpr int kPromptsPerLaunch = 256;
struct PromptRange {
  int q0, q_len, k0, k_len;
};
constexpr int kPromptBlock = 128;  // keys of a block
// An item's part in the workspace: M, r, l of its 256 rows, then their 128 channels.
constexpr int kPromptPartFloats = 3 * 256 + 256 * kHeadDim;
constexpr int kPromptParts = 608;
struct PromptParams {
  CUtensorMap q_map, k_map, v_map, out_map;  // [tokens][heads][128] (q, out), [heads][tokens][128]: boxes of 64 channels
  int out_mapped;  // out's strides allow a map
  Rows out;
  float* lse;
  int prompts, q_heads, kv_heads, group, causal;
  int tile_tokens;  // tokens of a tile: 128 / group
  int items;        // work items: pieces, tile pairs and KV heads of every prompt
  int chunk;        // key blocks of a piece
  int split;        // some item has several pieces
  float scale;
  uint32_t* status;
  uint32_t* counters;  // items taken, CTAs that have finished; zero between launches
  float* parts;
  int tiles;        // tile pairs of every prompt
  PromptRange range[kPromptsPerLaunch];  // longest first
  int first_unit[kPromptsPerLaunch];     // (piece, tile pair) number of each prompt's first
  int first_tile[kPromptsPerLaunch];     // tile pair number of each prompt's first
};

cudaError_t launch_pages_append(const PagesAppendParams& p, bool f16, cudaStream_t s);
cudaError_t launch_pages_decode(const PagesDecodeParams& p, bool f16, cudaStream_t s);
cudaError_t launch_prompt(const PromptParams& p, bool f16, cudaStream_t s);

// A launch that may be scheduled while the kernel before it on the stream still runs (the kernel waits itself).
template <class... P, class... A>
cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s,
                              const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// Streaming multiprocessors of the current device, looked up once per device.
inline int device_sms() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 152;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 152;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// CTAs of a paged decode launch: two to an SM (as many as there are counters for).
inline int decode_ctas() { return std::min(2 * device_sms(), kDecodeJoinCounters / 2 * kDecodeJoinCtas); }

}  // namespace hg
