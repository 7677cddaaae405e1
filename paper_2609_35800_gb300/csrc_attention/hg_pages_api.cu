// C ABI of the 16-bit caches: page pools, append, paged decode attention, prompt attention.  Every argument is checked
// here, on the host, before anything is enqueued.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include <new>

#include <cudaTypedefs.h>

#include "hg_attention.h"

struct hg_pages {
  hg::PagePool pool;
  int dtype;
  // tensor maps, encoded by the first decode call
  std::mutex mutex;
  std::atomic<bool> mapped{false};
  CUtensorMap k_map, v_map;
};

namespace {

using namespace hg;

constexpr double kPromptSplitGain = 8;  // blocks by which the longest item has to pass the even share
constexpr int kPromptLeastChunk = 4;
constexpr int64_t kMaxStride = int64_t(1) << 38;  // elements; a tensor map's strides are below 2^40 bytes

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
hg_status of_cuda(cudaError_t e) { return e == cudaSuccess ? HG_OK : HG_ERR_CUDA; }

// One set of rows: present, aligned, strides in range.
hg_status check_rows(const hg_rows& r) {
  if (!r.data || r.token_stride < 0 || r.head_stride < 0 || r.token_stride >= kMaxStride || r.head_stride >= kMaxStride)
    return HG_ERR_INVALID_ARG;
  return aligned16(r.data) && r.token_stride % 8 == 0 && r.head_stride % 8 == 0 ? HG_OK : HG_ERR_ALIGNMENT;
}

hg_status check_all(std::initializer_list<const hg_rows*> rows) {
  hg_status first = HG_OK;
  for (const hg_rows* r : rows) {
    const hg_status st = check_rows(*r);
    if (st == HG_ERR_INVALID_ARG) return st;
    if (first == HG_OK) first = st;
  }
  return first;
}

hg_status check_rotation(const hg_rotation* r, const int32_t* positions) {
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

Rotation rotation_of(const hg_rotation* r, const int32_t* positions, int tokens) {
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

float scale_of(float softmax_scale) { return softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)kHeadDim); }

// cuTensorMapEncodeTiled through the runtime (no link against the driver library).
PFN_cuTensorMapEncodeTiled_v12000 map_encoder() {
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

// A page pool as [pages][heads][2][page_size][64]: both halves of a row's channels as rows of 128 bytes, the span of
// the swizzle.  A box is a tile's tokens of one page and head: first halves, then second halves.
CUresult encode_pages(PFN_cuTensorMapEncodeTiled_v12000 encode, CUtensorMap* map, void* data, const PagePool& p, bool f16) {
  const cuuint64_t dims[5] = {64, (cuuint64_t)p.page_size, 2, (cuuint64_t)p.heads, (cuuint64_t)p.num_pages};
  // the stride of an axis of length 1 is never taken
  const cuuint64_t strides[4] = {(cuuint64_t)p.token_stride * 2, 128, p.heads > 1 ? (cuuint64_t)p.head_stride * 2 : 256,
                                 p.num_pages > 1 ? (cuuint64_t)p.page_stride * 2 : 256};
  const cuuint32_t box[5] = {64, (cuuint32_t)std::min(p.page_size, kDecodeTile), 2, 1, 1};
  const cuuint32_t steps[5] = {1, 1, 1, 1, 1};
  return encode(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, data, dims, strides, box,
                steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// Rows of a prompt's tensor: [a][b][128] in boxes of box_a x box_b x 64 channels.
CUresult encode_rows(PFN_cuTensorMapEncodeTiled_v12000 encode, CUtensorMap* map, void* data, int a, int64_t stride_a, int box_a,
                     int b, int64_t stride_b, int box_b, bool f16) {
  const cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)b, (cuuint64_t)a};
  const cuuint64_t strides[2] = {b > 1 ? (cuuint64_t)stride_b * 2 : 256, a > 1 ? (cuuint64_t)stride_a * 2 : 256};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_b, (cuuint32_t)box_a};
  const cuuint32_t steps[3] = {1, 1, 1};
  return encode(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, data, dims, strides, box,
                steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// A stride that is taken has to reach past the row (a tensor map has no broadcast axis).
bool rows_mappable(const hg_rows& r, int tokens, int heads) {
  return (tokens <= 1 || r.token_stride >= kHeadDim) && (heads <= 1 || r.head_stride >= kHeadDim);
}

// Pieces, tile pairs and heads of the launch's prompts, in blocks of kPromptBlock keys a piece at most `chunk`.
int64_t count_items(PromptParams* p) {
  int64_t units = 0, all = 0;
  for (int i = 0; i < p->prompts; ++i) {
    const PromptRange& r = p->range[i];
    p->first_unit[i] = (int)std::min<int64_t>(units, INT32_MAX);
    p->first_tile[i] = (int)std::min<int64_t>(all, INT32_MAX);
    const int64_t tiles = (r.q_len + 2 * p->tile_tokens - 1) / (2 * p->tile_tokens);
    const int64_t blocks = (r.k_len + kPromptBlock - 1) / kPromptBlock;
    units += tiles * std::max<int64_t>(1, (blocks + p->chunk - 1) / p->chunk);
    all += tiles;
  }
  p->tiles = (int)std::min<int64_t>(all, INT32_MAX);
  return units * p->kv_heads;
}

// How the launch's keys are cut.  Uncut, the launch lasts as long as its longest item at least; cut, as long as the
// SMs' even share of all blocks, and the parts' way through memory and the join besides.  64 tokens after 16,000, 28
// heads: longest 126 blocks, share 6.6, cut 25 us.  1,460 tokens, 28 heads: longest 12, share 6.7, uncut 26 us, cut 49.
// Left out is that whole items come in rounds: 20 prompts of 8 tokens after 8,000 of 64 heads are 160 items on 152 SMs and
// take 179 us, 18 of them (144 items) 96.
hg_status plan_prompts(PromptParams* p) {
  p->tile_tokens = 128 / p->group;
  std::sort(p->range, p->range + p->prompts,
            [](const PromptRange& a, const PromptRange& b) { return a.k_len != b.k_len ? a.k_len > b.k_len : a.q0 < b.q0; });
  p->chunk = INT32_MAX / 2;
  int64_t items = count_items(p);
  double blocks = 0.;
  for (int i = 0; i < p->prompts; ++i) {
    const PromptRange& r = p->range[i];
    const double keys = p->causal ? std::max(r.k_len - 0.5 * r.q_len, 0.5 * r.k_len) : r.k_len;
    blocks += ((r.q_len + 2 * p->tile_tokens - 1) / (2 * p->tile_tokens)) * (keys / kPromptBlock);
  }
  const double share = blocks * p->kv_heads / device_sms();
  const int longest = (p->range[0].k_len + kPromptBlock - 1) / kPromptBlock;
  if (longest > share + kPromptSplitGain) {
    for (int chunk = std::max((int)share + 1, kPromptLeastChunk); chunk < longest; chunk *= 2) {
      p->chunk = chunk;
      items = count_items(p);
      if (items <= kPromptParts) {
        p->split = 1;
        break;
      }
    }
    if (!p->split) {
      p->chunk = INT32_MAX / 2;
      items = count_items(p);
    }
  }
  if (items * 8 > INT32_MAX) return HG_ERR_UNSUPPORTED;
  p->items = (int)items;
  return HG_OK;
}

// The launch of prompts [done, done + kPromptsPerLaunch) of a call: none of them may have a query, then there is none.
hg_status plan_launch(PromptParams* p, const int32_t* q_begin, const int32_t* k_begin, int num_prompts, int done) {
  const int end = std::min(num_prompts - done, kPromptsPerLaunch) + done;
  p->prompts = p->split = 0;
  for (int i = done; i < end; ++i)
    if (q_begin[i + 1] > q_begin[i])  // a prompt without a query has nothing to write
      p->range[p->prompts++] = {q_begin[i], q_begin[i + 1] - q_begin[i], k_begin[i], k_begin[i + 1] - k_begin[i]};
  return p->prompts == 0 ? HG_OK : plan_prompts(p);
}

hg_status map_pages(hg_pages* p) {
  if (p->mapped.load(std::memory_order_acquire)) return HG_OK;
  const PFN_cuTensorMapEncodeTiled_v12000 encode = map_encoder();
  if (!encode) return HG_ERR_CUDA;
  std::lock_guard<std::mutex> lock(p->mutex);
  if (p->mapped.load(std::memory_order_relaxed)) return HG_OK;
  const bool f16 = p->dtype == HG_DTYPE_F16;
  if (encode_pages(encode, &p->k_map, p->pool.k, p->pool, f16) != CUDA_SUCCESS ||
      encode_pages(encode, &p->v_map, p->pool.v, p->pool, f16) != CUDA_SUCCESS)
    return HG_ERR_CUDA;
  p->mapped.store(true, std::memory_order_release);
  return HG_OK;
}

// Decode workspace: header, the parts that CTAs leave (two each, at the largest group whatever the call's, so that the
// counters behind them lie at one place for every call), a counter per (request, KV head): of the most KV heads that a
// pool may have, so that a workspace serves every pool (256 bytes a request).
size_t decode_parts_bytes() { return (size_t)decode_ctas() * 2 * kMaxGroup * kPartialFloats * sizeof(float); }
size_t decode_workspace_bytes(int batch) {
  const size_t counters = kDecodeJoinCounters + (size_t)batch * kMaxKvHeads;
  return kAttnHeaderBytes + decode_parts_bytes() + ((counters * sizeof(uint32_t) + 255) & ~size_t(255));
}

hg_status decode_batch_ok(const hg_pages* p, int32_t batch, int32_t num_q_heads) {
  if (!p || batch < 0 || num_q_heads < 1 || num_q_heads % p->pool.heads != 0) return HG_ERR_INVALID_ARG;
  if (num_q_heads / p->pool.heads > kMaxGroup || batch > (1 << 20)) return HG_ERR_UNSUPPORTED;
  return HG_OK;
}

hg_status pages_decode(const hg_pages* pages, int32_t batch, int32_t num_q_heads, const hg_attention_io* io,
                       const hg_rotation* rotation, const int32_t* positions, const int32_t* page_table,
                       int32_t table_stride, const int32_t* lengths, float* lse, float softmax_scale, void* ws,
                       size_t ws_bytes, bool store, cudaStream_t stream) {
  hg_status st = decode_batch_ok(pages, batch, num_q_heads);
  if (st != HG_OK) return st;
  if (!io || table_stride < 0 || !(softmax_scale == softmax_scale)) return HG_ERR_INVALID_ARG;
  if (batch == 0) return HG_OK;
  if ((table_stride > 0 && !page_table) || !lengths || !ws) return HG_ERR_INVALID_ARG;
  // the kernel numbers tokens, and tiles and fixed costs of every request and head, in 32 bits
  const int64_t capacity = (int64_t)table_stride * pages->pool.page_size;
  if (capacity > INT32_MAX ||
      (capacity / kDecodeTile + 1 + kDecodeItemCost) * pages->pool.heads > INT32_MAX / std::max(batch, 1))
    return HG_ERR_UNSUPPORTED;
  st = store ? check_all({&io->q, &io->k, &io->v, &io->out}) : check_all({&io->q, &io->out});
  if (st != HG_OK) return st;
  st = check_rotation(rotation, positions);
  if (st != HG_OK) return st;
  if (!aligned4(page_table) || !aligned4(lengths) || !aligned4(lse) || !aligned16(ws)) return HG_ERR_ALIGNMENT;
  if (ws_bytes < decode_workspace_bytes(batch)) return HG_ERR_WORKSPACE_TOO_SMALL;
  st = map_pages(const_cast<hg_pages*>(pages));
  if (st != HG_OK) return st;
  PagesDecodeParams p;
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
  return of_cuda(launch_pages_decode(p, pages->dtype == HG_DTYPE_F16, stream));
}

}  // namespace

extern "C" {

hg_status hg_pages_create(const hg_page_shape* s, void* k_pages, void* v_pages, hg_pages** out) {
  if (!s || !k_pages || !v_pages || !out) return HG_ERR_INVALID_ARG;
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
  if (!aligned16(k_pages) || !aligned16(v_pages) || token % 8 || head % 8 || page % 8) return HG_ERR_ALIGNMENT;
  hg_pages* p = new (std::nothrow) hg_pages();
  if (!p) return HG_ERR_CUDA;
  int shift = 0;
  while ((1 << shift) < s->page_size) ++shift;
  p->pool = {static_cast<uint16_t*>(k_pages), static_cast<uint16_t*>(v_pages), s->num_pages, s->page_size, shift,
             s->num_kv_heads, page, head, token};
  p->dtype = s->dtype;
  *out = p;
  return HG_OK;
}

void hg_pages_destroy(hg_pages* pages) { delete pages; }

hg_status hg_pages_append(const hg_pages* pages, int32_t num_tokens, int32_t num_q_heads, const hg_append_io* io,
                          const hg_rotation* rotation, const int32_t* positions, const int32_t* slots,
                          hg_stream_t stream) {
  if (!pages || num_tokens < 0 || num_q_heads < 0 || !io) return HG_ERR_INVALID_ARG;
  if (num_q_heads > kMaxGroup * kMaxKvHeads) return HG_ERR_UNSUPPORTED;
  if (num_tokens == 0) return HG_OK;
  if (!slots) return HG_ERR_INVALID_ARG;
  const hg_rows none = io->k;  // stands in for an absent set, which is not checked
  hg_status st = check_all({&io->k, &io->v, num_q_heads ? &io->q : &none, num_q_heads ? &io->q_out : &none,
                            io->k_out.data ? &io->k_out : &none, io->v_out.data ? &io->v_out : &none});
  if (st != HG_OK) return st;
  st = check_rotation(rotation, positions);
  if (st != HG_OK) return st;
  if (!aligned4(slots)) return HG_ERR_ALIGNMENT;
  PagesAppendParams p;
  std::memset(&p, 0, sizeof p);
  p.pool = pages->pool;
  p.rot = rotation_of(rotation, positions, num_tokens);
  p.tokens = num_tokens;
  p.q_heads = num_q_heads;
  p.q = rows_of(io->q);
  p.k = rows_of(io->k);
  p.v = rows_of(io->v);
  p.q_out = rows_of(io->q_out);
  p.k_out = rows_of(io->k_out);
  p.v_out = rows_of(io->v_out);
  p.slots = slots;
  return of_cuda(launch_pages_append(p, pages->dtype == HG_DTYPE_F16, reinterpret_cast<cudaStream_t>(stream)));
}

hg_status hg_pages_decode_workspace_size(const hg_pages* pages, int32_t batch, int32_t num_q_heads, size_t* bytes) {
  if (!bytes) return HG_ERR_INVALID_ARG;
  const hg_status st = decode_batch_ok(pages, batch, num_q_heads);
  if (st != HG_OK) return st;
  *bytes = decode_workspace_bytes(batch);
  return HG_OK;
}

hg_status hg_pages_decode_attention(const hg_pages* pages, int32_t batch, int32_t num_q_heads,
                                    const hg_attention_io* io, const int32_t* page_table, int32_t table_stride,
                                    const int32_t* lengths, float* lse, float softmax_scale, void* workspace,
                                    size_t workspace_bytes, hg_stream_t stream) {
  return pages_decode(pages, batch, num_q_heads, io, nullptr, nullptr, page_table, table_stride, lengths, lse,
                      softmax_scale, workspace, workspace_bytes, false, reinterpret_cast<cudaStream_t>(stream));
}

hg_status hg_pages_decode_step(const hg_pages* pages, int32_t batch, int32_t num_q_heads, const hg_attention_io* io,
                               const hg_rotation* rotation, const int32_t* positions, const int32_t* page_table,
                               int32_t table_stride, const int32_t* lengths, float* lse, float softmax_scale,
                               void* workspace, size_t workspace_bytes, hg_stream_t stream) {
  return pages_decode(pages, batch, num_q_heads, io, rotation, positions, page_table, table_stride, lengths, lse,
                      softmax_scale, workspace, workspace_bytes, true, reinterpret_cast<cudaStream_t>(stream));
}

hg_status hg_prompt_workspace_size(size_t* bytes) {
  if (!bytes) return HG_ERR_INVALID_ARG;
  *bytes = kAttnHeaderBytes + (size_t)kPromptParts * kPromptPartFloats * sizeof(float);
  return HG_OK;
}

hg_status hg_prompt_attention(int32_t dtype, int32_t num_prompts, int32_t num_q_heads, int32_t num_kv_heads,
                              const hg_attention_io* io, const int32_t* q_begin, const int32_t* k_begin, float* lse,
                              int32_t causal, float softmax_scale, void* workspace, size_t workspace_bytes,
                              hg_stream_t stream) {
  if ((dtype != HG_DTYPE_BF16 && dtype != HG_DTYPE_F16) || num_prompts < 0 || num_kv_heads < 1 || num_q_heads < 1 ||
      num_q_heads % num_kv_heads != 0 || !io || causal < 0 || causal > 1 || !(softmax_scale == softmax_scale))
    return HG_ERR_INVALID_ARG;
  if (num_kv_heads > kMaxKvHeads || num_q_heads / num_kv_heads > kMaxGroup) return HG_ERR_UNSUPPORTED;
  if (num_prompts == 0) return HG_OK;
  if (!q_begin || !k_begin || q_begin[0] < 0 || k_begin[0] < 0) return HG_ERR_INVALID_ARG;
  for (int i = 0; i < num_prompts; ++i)
    if (q_begin[i + 1] < q_begin[i] || k_begin[i + 1] < k_begin[i]) return HG_ERR_INVALID_ARG;
  if (q_begin[num_prompts] == q_begin[0]) return HG_OK;
  // prompts without a key have no rows of k and v to point at
  const bool keys = k_begin[num_prompts] > k_begin[0];
  hg_status st = keys ? check_all({&io->q, &io->out, &io->k, &io->v}) : check_all({&io->q, &io->out});
  if (st != HG_OK) return st;
  const int rows = q_begin[num_prompts], key_rows = k_begin[num_prompts];
  if (!rows_mappable(io->q, rows, num_q_heads) ||
      (keys && (!rows_mappable(io->k, key_rows, num_kv_heads) || !rows_mappable(io->v, key_rows, num_kv_heads))))
    return HG_ERR_UNSUPPORTED;
  if (!workspace) return HG_ERR_INVALID_ARG;
  if (!aligned16(workspace) || !aligned4(lse)) return HG_ERR_ALIGNMENT;
  size_t need = 0;
  st = hg_prompt_workspace_size(&need);
  if (st != HG_OK) return st;
  if (workspace_bytes < need) return HG_ERR_WORKSPACE_TOO_SMALL;
  PromptParams p;
  std::memset(&p, 0, sizeof p);
  p.out = rows_of(io->out);
  p.lse = lse;
  p.q_heads = num_q_heads;
  p.kv_heads = num_kv_heads;
  p.group = num_q_heads / num_kv_heads;
  p.causal = causal;
  p.scale = scale_of(softmax_scale);
  char* w = static_cast<char*>(workspace);
  p.status = reinterpret_cast<uint32_t*>(w);
  p.counters = reinterpret_cast<uint32_t*>(w + 256);
  p.parts = reinterpret_cast<float*>(w + kAttnHeaderBytes);
  for (int done = 0; done < num_prompts; done += kPromptsPerLaunch) {  // what the last launch would refuse is refused here
    st = plan_launch(&p, q_begin, k_begin, num_prompts, done);
    if (st != HG_OK) return st;
  }
  const bool f16 = dtype == HG_DTYPE_F16;
  const PFN_cuTensorMapEncodeTiled_v12000 encode = map_encoder();
  if (!encode ||
      encode_rows(encode, &p.q_map, io->q.data, rows, io->q.token_stride, 128 / p.group, num_q_heads, io->q.head_stride,
                  p.group, f16) != CUDA_SUCCESS)
    return HG_ERR_CUDA;
  if (keys && (encode_rows(encode, &p.k_map, io->k.data, num_kv_heads, io->k.head_stride, 1, key_rows, io->k.token_stride,
                           kPromptBlock, f16) != CUDA_SUCCESS ||
               encode_rows(encode, &p.v_map, io->v.data, num_kv_heads, io->v.head_stride, 1, key_rows, io->v.token_stride,
                           kPromptBlock, f16) != CUDA_SUCCESS))
    return HG_ERR_CUDA;
  p.out_mapped = rows_mappable(io->out, rows, num_q_heads) &&
                 encode_rows(encode, &p.out_map, io->out.data, rows, io->out.token_stride, 128 / p.group, num_q_heads,
                             io->out.head_stride, p.group, f16) == CUDA_SUCCESS;
  for (int done = 0; done < num_prompts; done += kPromptsPerLaunch) {
    if (num_prompts > kPromptsPerLaunch) st = plan_launch(&p, q_begin, k_begin, num_prompts, done);
    if (st == HG_OK && p.prompts > 0) st = of_cuda(launch_prompt(p, f16, reinterpret_cast<cudaStream_t>(stream)));
    if (st != HG_OK) return st;
  }
  return HG_OK;
}

}  // extern "C"
