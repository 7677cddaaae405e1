// Host checks and plans shared by the entry points of the paged caches: rows, rotations, workspaces, tensor maps.
#pragma once
#include <cmath>
#include <initializer_list>

#include <cudaTypedefs.h>

#include "hg_attention.h"

namespace hg {

constexpr int64_t kMaxStride = int64_t(1) << 38;  // elements; a tensor map's strides are below 2^40 bytes

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline hg_status of_cuda(cudaError_t e) { return e == cudaSuccess ? HG_OK : HG_ERR_CUDA; }

// One set of rows: present, aligned, strides in range.
inline hg_status check_rows(const hg_rows& r) {
  if (!r.data || r.token_stride < 0 || r.head_stride < 0 || r.token_stride >= kMaxStride || r.head_stride >= kMaxStride)
    return HG_ERR_INVALID_ARG;
  return aligned16(r.data) && r.token_stride % 8 == 0 && r.head_stride % 8 == 0 ? HG_OK : HG_ERR_ALIGNMENT;
}

inline hg_status check_all(std::initializer_list<const hg_rows*> rows) {
  hg_status first = HG_OK;
  for (const hg_rows* r : rows) {
    const hg_status st = check_rows(*r);
    if (st == HG_ERR_INVALID_ARG) return st;
    if (first == HG_OK) first = st;
  }
  return first;
}

inline hg_status check_rotation(const hg_rotation* r, const int32_t* positions) {
  if (!r) return HG_OK;
  if (!r->table || !positions || r->table_len < 1 || r->interleaved < 0 || r->interleaved > 1) return HG_ERR_INVALID_ARG;
  if (!aligned16(r->table) || !aligned4(positions)) return HG_ERR_ALIGNMENT;
  if (r->rot_dim < 16 || r->rot_dim > kHeadDim || r->rot_dim % 16 != 0) return HG_ERR_UNSUPPORTED;
  const int32_t* s = r->sections;
  if (s[0] < 0 || s[1] < 0 || s[2] < 0) return HG_ERR_INVALID_ARG;
  if (s[0] || s[1] || s[2]) {
    if (s[0] > 64 || s[1] > 64 || s[2] > 64 || s[0] + s[1] + s[2] != r->rot_dim / 2) return HG_ERR_INVALID_ARG;
    if (s[0] % 8 || s[1] % 8 || s[2] % 8) return HG_ERR_UNSUPPORTED;
  }
  return HG_OK;
}

inline Rotation rotation_of(const hg_rotation* r, const int32_t* positions, int tokens) {
  Rotation o = {};
  if (!r) return o;
  o.table = r->table;
  o.table_len = r->table_len;
  o.half = r->rot_dim / 2;
  o.interleaved = r->interleaved;
  const bool three = r->sections[0] || r->sections[1] || r->sections[2];
  o.end0 = three ? r->sections[0] : o.half;
  o.end1 = three ? r->sections[0] + r->sections[1] : o.half;
  o.positions = positions;
  o.position_stride = three ? tokens : 0;
  return o;
}

inline float scale_of(float softmax_scale) { return softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)kHeadDim); }

// cuTensorMapEncodeTiled through the runtime (no link against the driver library).
inline PFN_cuTensorMapEncodeTiled_v12000 map_encoder() {
  static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> cached{nullptr};
  PFN_cuTensorMapEncodeTiled_v12000 fn = cached.load(std::memory_order_acquire);
  if (!fn) {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    cached.store(fn, std::memory_order_release);
  }
  return fn;
}

// Decode workspace: header, the parts that CTAs leave (two each, at the largest group whatever the call's, so that the
// counters behind them lie at one place for every call), a counter per (request, KV head): of the most KV heads that a
// pool may have, so that a workspace serves every pool (256 bytes a request).
inline size_t decode_parts_bytes() { return (size_t)decode_ctas() * 2 * kMaxGroup * kPartialFloats * sizeof(float); }
inline size_t decode_workspace_bytes(int batch) {
  const size_t counters = kDecodeJoinCounters + (size_t)batch * kMaxKvHeads;
  return kAttnHeaderBytes + decode_parts_bytes() + ((counters * sizeof(uint32_t) + 255) & ~size_t(255));
}

// Queries and requests of a paged decode over `heads` KV heads.
inline hg_status decode_batch_ok(int heads, int32_t batch, int32_t num_q_heads) {
  if (batch < 0 || num_q_heads < 1 || num_q_heads % heads != 0) return HG_ERR_INVALID_ARG;
  if (num_q_heads / heads > kMaxGroup || batch > (1 << 20)) return HG_ERR_UNSUPPORTED;
  return HG_OK;
}

// The kernels number tokens, and tiles and fixed costs of every request and head, in 32 bits.
inline bool decode_table_ok(const PoolShape& pool, int32_t batch, int32_t table_stride) {
  const int64_t capacity = (int64_t)table_stride * pool.page_size;
  return capacity <= INT32_MAX &&
         (capacity / kDecodeTile + 1 + kDecodeItemCost) * pool.heads <= INT32_MAX / std::max(batch, 1);
}

// A pool's geometry and strides in elements, checked; strides are multiples of `align`.
inline hg_status check_shape(const hg_page_shape* s, int align, PoolShape* pool) {
  if (s->dtype != HG_DTYPE_BF16 && s->dtype != HG_DTYPE_F16) return HG_ERR_INVALID_ARG;
  if (s->num_pages < 1 || s->num_kv_heads < 1 || s->page_size < 1) return HG_ERR_INVALID_ARG;
  if (s->page_stride < 0 || s->head_stride < 0 || s->token_stride < 0) return HG_ERR_INVALID_ARG;
  if (s->head_dim != kHeadDim || s->num_kv_heads > kMaxKvHeads) return HG_ERR_UNSUPPORTED;
  if (s->page_size < 16 || s->page_size > 256 || (s->page_size & (s->page_size - 1))) return HG_ERR_UNSUPPORTED;
  if ((int64_t)s->num_pages * s->page_size > INT32_MAX) return HG_ERR_UNSUPPORTED;
  int64_t token = s->token_stride, head = s->head_stride, page = s->page_stride;
  if (token == 0 && head == 0 && page == 0) {
    token = kHeadDim;
    head = token * s->page_size;
    page = head * s->num_kv_heads;
  }
  if (token < kHeadDim || (s->num_kv_heads > 1 && head < kHeadDim) || (s->num_pages > 1 && page < kHeadDim))
    return HG_ERR_INVALID_ARG;
  if (token >= kMaxStride || head >= kMaxStride || page >= kMaxStride) return HG_ERR_UNSUPPORTED;
  if (token % align || head % align || page % align) return HG_ERR_ALIGNMENT;
  int shift = 0;
  while ((1 << shift) < s->page_size) ++shift;
  *pool = {s->num_pages, s->page_size, shift, s->num_kv_heads, page, head, token};
  return HG_OK;
}

}  // namespace hg
