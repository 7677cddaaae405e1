// C ABI of the 8-bit paged caches and of page tables built on the GPU.  Every argument is checked here, on the host,
// before anything is enqueued.
#include <cstring>
#include <mutex>
#include <new>
#include <utility>

#include "hg_checks.h"

struct hg_pages8 {
  hg::PagePool8 pool;
  int dtype;
  // tensor maps, encoded by the first decode call
  std::mutex mutex;
  std::atomic<bool> mapped{false};
  CUtensorMap k_map, v_map;
};

namespace {

using namespace hg;

constexpr int kMaxRows = 1 << 30;  // tokens and requests of a call: their sums stay in 32 bits

// begin, table and what else says where a call's tokens lie.
hg_status check_places(int32_t requests, const int32_t* begin, const int32_t* page_table, int32_t table_stride,
                       const PoolShape& pool) {
  if (!begin || table_stride < 0 || (table_stride > 0 && !page_table)) return HG_ERR_INVALID_ARG;
  if (!aligned4(begin) || !aligned4(page_table)) return HG_ERR_ALIGNMENT;
  return (int64_t)table_stride * pool.page_size > INT32_MAX ? HG_ERR_UNSUPPORTED : HG_OK;
}

// A pool as [pages][heads][page_size][128]: a box is a tile's tokens of one page and head, a row the swizzle's span.
CUresult encode_pages8(PFN_cuTensorMapEncodeTiled_v12000 encode, CUtensorMap* map, void* data, const PagePool8& p) {
  const cuuint64_t dims[4] = {(cuuint64_t)kHeadDim, (cuuint64_t)p.page_size, (cuuint64_t)p.heads, (cuuint64_t)p.num_pages};
  // the stride of an axis of length 1 is never taken
  const cuuint64_t strides[3] = {(cuuint64_t)p.token_stride, p.heads > 1 ? (cuuint64_t)p.head_stride : 128,
                                 p.num_pages > 1 ? (cuuint64_t)p.page_stride : 128};
  const cuuint32_t box[4] = {kHeadDim, (cuuint32_t)std::min(p.page_size, kDecodeTile8), 1, 1};
  const cuuint32_t steps[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, data, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

hg_status map_pages8(hg_pages8* p) {
  if (p->mapped.load(std::memory_order_acquire)) return HG_OK;
  const PFN_cuTensorMapEncodeTiled_v12000 encode = map_encoder();
  if (!encode) return HG_ERR_CUDA;
  std::lock_guard<std::mutex> lock(p->mutex);
  if (p->mapped.load(std::memory_order_relaxed)) return HG_OK;
  if (encode_pages8(encode, &p->k_map, p->pool.k, p->pool) != CUDA_SUCCESS ||
      encode_pages8(encode, &p->v_map, p->pool.v, p->pool) != CUDA_SUCCESS)
    return HG_ERR_CUDA;
  p->mapped.store(true, std::memory_order_release);
  return HG_OK;
}

bool share_memory(const int32_t* a, int64_t n, const int32_t* b, int64_t m) { return a < b + m && b < a + n; }

hg_status pages8_decode(const hg_pages8* pages, int32_t batch, int32_t num_q_heads, const hg_attention_io* io,
                        const hg_rotation* rotation, const int32_t* positions, const int32_t* page_table,
                        int32_t table_stride, const int32_t* lengths, float* lse, float softmax_scale, void* ws,
                        size_t ws_bytes, bool store, cudaStream_t stream) {
  if (!pages) return HG_ERR_INVALID_ARG;
  hg_status st = decode_batch_ok(pages->pool.heads, batch, num_q_heads);
  if (st != HG_OK) return st;
  if (!io || table_stride < 0 || !(softmax_scale == softmax_scale)) return HG_ERR_INVALID_ARG;
  if (batch == 0) return HG_OK;
  if ((table_stride > 0 && !page_table) || !lengths || !ws) return HG_ERR_INVALID_ARG;
  if (!decode_table_ok(pages->pool, batch, table_stride)) return HG_ERR_UNSUPPORTED;
  st = store ? check_all({&io->q, &io->k, &io->v, &io->out}) : check_all({&io->q, &io->out});
  if (st != HG_OK) return st;
  st = check_rotation(rotation, positions);
  if (st != HG_OK) return st;
  if (!aligned4(page_table) || !aligned4(lengths) || !aligned4(lse) || !aligned16(ws)) return HG_ERR_ALIGNMENT;
  if (ws_bytes < decode_workspace_bytes(batch)) return HG_ERR_WORKSPACE_TOO_SMALL;
  st = map_pages8(const_cast<hg_pages8*>(pages));
  if (st != HG_OK) return st;
  Pages8DecodeParams p;
  std::memset(&p, 0, sizeof p);
  p.k_map = pages->k_map;
  p.v_map = pages->v_map;
  p.pool = pages->pool;
  p.rot = rotation_of(rotation, positions, batch);
  p.batch = batch;
  p.group = num_q_heads / pages->pool.heads;
  p.store = store ? 1 : 0;
  p.q = rows_of(io->q);
  p.out = rows_of(io->out);
  if (store) {
    p.k = rows_of(io->k);
    p.v = rows_of(io->v);
  }
  p.table = page_table;
  p.table_stride = table_stride;
  p.lengths = lengths;
  p.lse = lse;
  p.scale = scale_of(softmax_scale);
  char* w = static_cast<char*>(ws);
  p.status = reinterpret_cast<uint32_t*>(w);
  p.partials = reinterpret_cast<float*>(w + kAttnHeaderBytes);
  p.counters = reinterpret_cast<uint32_t*>(w + kAttnHeaderBytes + decode_parts_bytes());
  return of_cuda(launch_pages8_decode(p, pages->dtype == HG_DTYPE_F16, stream));
}

}  // namespace

extern "C" {

hg_status hg_pages8_create(const hg_page_shape* s, void* k_pages, void* v_pages, float* k_scales, float* v_scales,
                           hg_pages8** out) {
  if (!s || !k_pages || !v_pages || !k_scales || !v_scales || !out) return HG_ERR_INVALID_ARG;
  PoolShape shape;
  const hg_status st = check_shape(s, 16, &shape);
  if (st != HG_OK) return st;
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned4(k_scales) || !aligned4(v_scales)) return HG_ERR_ALIGNMENT;
  hg_pages8* p = new (std::nothrow) hg_pages8();
  if (!p) return HG_ERR_CUDA;
  static_cast<PoolShape&>(p->pool) = shape;
  p->pool.k = static_cast<uint8_t*>(k_pages);
  p->pool.v = static_cast<uint8_t*>(v_pages);
  p->pool.k_scales = k_scales;
  p->pool.v_scales = v_scales;
  p->dtype = s->dtype;
  *out = p;
  return HG_OK;
}

void hg_pages8_destroy(hg_pages8* pages) { delete pages; }

hg_status hg_pages8_append(const hg_pages8* pages, int32_t num_tokens, int32_t num_requests, int32_t num_q_heads,
                           const hg_append_io* io, const hg_rotation* rotation, const int32_t* positions,
                           const int32_t* begin, const int32_t* page_table, int32_t table_stride, const int32_t* lengths,
                           hg_stream_t stream) {
  if (!pages || num_tokens < 0 || num_requests < 0 || num_q_heads < 0 || !io) return HG_ERR_INVALID_ARG;
  if (num_q_heads > kMaxGroup * kMaxKvHeads || num_tokens > kMaxRows || num_requests > kMaxRows / 4)
    return HG_ERR_UNSUPPORTED;
  if (num_tokens == 0 || num_requests == 0) return HG_OK;
  int64_t kv = 0, q = 0;
  if (!append8_grid(num_tokens, num_requests, num_q_heads, pages->pool.heads, &kv, &q)) return HG_ERR_UNSUPPORTED;
  if (!lengths) return HG_ERR_INVALID_ARG;
  hg_status st = check_places(num_requests, begin, page_table, table_stride, pages->pool);
  if (st != HG_OK) return st;
  const hg_rows none = io->k;  // stands in for an absent set, which is not checked
  st = check_all({&io->k, &io->v, num_q_heads ? &io->q : &none, num_q_heads ? &io->q_out : &none,
                  io->k_out.data ? &io->k_out : &none, io->v_out.data ? &io->v_out : &none});
  if (st != HG_OK) return st;
  st = check_rotation(rotation, positions);
  if (st != HG_OK) return st;
  if (!aligned4(lengths)) return HG_ERR_ALIGNMENT;
  Pages8AppendParams p;
  std::memset(&p, 0, sizeof p);
  p.pool = pages->pool;
  p.rot = rotation_of(rotation, positions, num_tokens);
  p.tokens = num_tokens;
  p.requests = num_requests;
  p.q_heads = num_q_heads;
  p.q = rows_of(io->q);
  p.k = rows_of(io->k);
  p.v = rows_of(io->v);
  p.q_out = rows_of(io->q_out);
  p.k_out = rows_of(io->k_out);
  p.v_out = rows_of(io->v_out);
  p.begin = begin;
  p.table = page_table;
  p.table_stride = table_stride;
  p.lengths = lengths;
  return of_cuda(launch_pages8_append(p, pages->dtype == HG_DTYPE_F16, reinterpret_cast<cudaStream_t>(stream)));
}

hg_status hg_pages8_dequantize(const hg_pages8* pages, int32_t num_rows, int32_t num_requests, const int32_t* begin,
                               const int32_t* page_table, int32_t table_stride, const hg_rows* k_out,
                               const hg_rows* v_out, hg_stream_t stream) {
  const hg_rows none = {nullptr, 0, 0};
  const hg_rows &k = k_out ? *k_out : none, &v = v_out ? *v_out : none;
  if (!pages || num_rows < 0 || num_requests < 0 || (!k.data && !v.data)) return HG_ERR_INVALID_ARG;
  if (num_rows > kMaxRows || num_requests > kMaxRows) return HG_ERR_UNSUPPORTED;
  if (num_rows == 0 || num_requests == 0) return HG_OK;
  hg_status st = check_places(num_requests, begin, page_table, table_stride, pages->pool);
  if (st != HG_OK) return st;
  st = check_all({k.data ? &k : &v, v.data ? &v : &k});
  if (st != HG_OK) return st;
  Pages8DequantizeParams p;
  std::memset(&p, 0, sizeof p);
  p.pool = pages->pool;
  p.tokens = num_rows;
  p.requests = num_requests;
  p.k_out = rows_of(k);
  p.v_out = rows_of(v);
  p.begin = begin;
  p.table = page_table;
  p.table_stride = table_stride;
  return of_cuda(launch_pages8_dequantize(p, pages->dtype == HG_DTYPE_F16, reinterpret_cast<cudaStream_t>(stream)));
}

hg_status hg_pages8_decode_workspace_size(const hg_pages8* pages, int32_t batch, int32_t num_q_heads, size_t* bytes) {
  if (!bytes || !pages) return HG_ERR_INVALID_ARG;
  const hg_status st = decode_batch_ok(pages->pool.heads, batch, num_q_heads);
  if (st != HG_OK) return st;
  *bytes = decode_workspace_bytes(batch);
  return HG_OK;
}

hg_status hg_pages8_decode_attention(const hg_pages8* pages, int32_t batch, int32_t num_q_heads,
                                     const hg_attention_io* io, const int32_t* page_table, int32_t table_stride,
                                     const int32_t* lengths, float* lse, float softmax_scale, void* workspace,
                                     size_t workspace_bytes, hg_stream_t stream) {
  return pages8_decode(pages, batch, num_q_heads, io, nullptr, nullptr, page_table, table_stride, lengths, lse,
                       softmax_scale, workspace, workspace_bytes, false, reinterpret_cast<cudaStream_t>(stream));
}

hg_status hg_pages8_decode_step(const hg_pages8* pages, int32_t batch, int32_t num_q_heads, const hg_attention_io* io,
                                const hg_rotation* rotation, const int32_t* positions, const int32_t* page_table,
                                int32_t table_stride, const int32_t* lengths, float* lse, float softmax_scale,
                                void* workspace, size_t workspace_bytes, hg_stream_t stream) {
  return pages8_decode(pages, batch, num_q_heads, io, rotation, positions, page_table, table_stride, lengths, lse,
                       softmax_scale, workspace, workspace_bytes, true, reinterpret_cast<cudaStream_t>(stream));
}

hg_status hg_pages_plan(int32_t batch, int32_t page_size, int32_t* page_table, int32_t table_stride, const int32_t* cached,
                        const int32_t* new_tokens, int32_t* free_pages, int32_t free_capacity, const int32_t* free_count,
                        int32_t max_tokens, int32_t* lengths, int32_t* begin, int32_t* slots, int32_t* positions,
                        int32_t* counts, hg_stream_t stream) {
  if (batch < 0 || page_size < 1 || table_stride < 0 || free_capacity < 0 || max_tokens < 0) return HG_ERR_INVALID_ARG;
  if (!free_count || !begin || !counts || (free_capacity > 0 && !free_pages) || (max_tokens > 0 && !slots))
    return HG_ERR_INVALID_ARG;
  if (batch > 0 && (!cached || !new_tokens || !lengths || (table_stride > 0 && !page_table))) return HG_ERR_INVALID_ARG;
  if (batch > kPlanMaxBatch || page_size < 16 || page_size > 256 || (page_size & (page_size - 1)))
    return HG_ERR_UNSUPPORTED;
  if ((int64_t)table_stride * page_size > INT32_MAX || (int64_t)batch * table_stride > INT32_MAX || max_tokens > kMaxRows)
    return HG_ERR_UNSUPPORTED;
  for (const int32_t* x : {static_cast<const int32_t*>(page_table), cached, new_tokens, static_cast<const int32_t*>(free_pages),
                           free_count, static_cast<const int32_t*>(lengths), static_cast<const int32_t*>(begin),
                           static_cast<const int32_t*>(slots), static_cast<const int32_t*>(positions),
                           static_cast<const int32_t*>(counts)})
    if (!aligned4(x)) return HG_ERR_ALIGNMENT;
  PagesPlanParams p;
  std::memset(&p, 0, sizeof p);
  p.batch = batch;
  while ((1 << p.page_shift) < page_size) ++p.page_shift;
  p.table = page_table;
  p.table_stride = table_stride;
  p.cached = cached;
  p.new_tokens = new_tokens;
  p.free_pages = free_pages;
  p.free_capacity = free_capacity;
  p.free_count = free_count;
  p.tokens = max_tokens;
  p.lengths = lengths;
  p.begin = begin;
  p.slots = slots;
  p.positions = positions;
  p.counts = counts;
  for (const auto& out : {std::make_pair(lengths, batch), std::make_pair(counts, 4)})
    if (share_memory(out.first, out.second, cached, batch) || share_memory(out.first, out.second, new_tokens, batch) ||
        share_memory(out.first, out.second, free_count, 1))
      p.in_place = 1;
  return of_cuda(launch_pages_plan(p, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
