// C ABI of the key/value cache and its attention: argument checks on the host,
// then launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>

#include "ewsjf.h"
#include "ewsjf_cache.h"

namespace {

constexpr int32_t kMaxGroup = 64;              // query heads per key head
constexpr int64_t kMaxQ = (int64_t)1 << 24;    // query tokens of a batch
constexpr int64_t kMaxRead = (int64_t)1 << 31; // rows of a read
constexpr int64_t kMaxStride = (int64_t)1 << 48;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool stride_ok(int64_t s, int64_t unit = 8) { return s >= 0 && s <= kMaxStride && s % unit == 0; }
bool in_codes(int32_t dtype) { return dtype == EWSJF_E4M3_BF16 || dtype == EWSJF_E4M3_F16; }

// The outer dims' blocks follow one another without overlap, whatever their order.
bool apart(int64_t block, const int64_t* size, const int64_t* stride) {
  bool done[3] = {false, false, false};
  for (int i = 0; i < 3; ++i) {
    int best = -1;
    for (int d = 0; d < 3; ++d)
      if (!done[d] && (best < 0 || stride[d] < stride[best] || (stride[d] == stride[best] && size[d] < size[best])))
        best = d;
    done[best] = true;
    if (size[best] == 1) continue;
    if (stride[best] < block) return false;
    block = stride[best] * (size[best] - 1) + block;
  }
  return true;
}

bool page_ok(int32_t page_size, int32_t kv_heads, int32_t head_dim, int32_t dtype) {
  if (page_size < 1 || page_size > EWSJF_MAX_PAGE_SIZE || (page_size & (page_size - 1))) return false;
  if (kv_heads < 1 || kv_heads > 1024) return false;
  if (dtype != EWSJF_BF16 && dtype != EWSJF_F16 && !in_codes(dtype)) return false;
  const int32_t unit = in_codes(dtype) ? 16 : 8;
  return head_dim >= unit && head_dim <= EWSJF_MAX_HEAD_DIM && head_dim % unit == 0;
}

ewsjf_status cache_status(const ewsjf_cache* c) {
  if (c == nullptr) return EWSJF_ERR_NULL;
  if (c->data == nullptr || c->refs == nullptr || c->table == nullptr || c->length == nullptr) return EWSJF_ERR_NULL;
  if (c->layers < 1 || c->layers > 4096 || c->n_pages < 1 || c->n_pages > EWSJF_MAX_PAGES) return EWSJF_ERR_ARG;
  if (!page_ok(c->page_size, c->kv_heads, c->head_dim, c->dtype)) return EWSJF_ERR_ARG;
  if (c->n_slots < 1 || c->n_slots > (1 << 24) || c->width < 1) return EWSJF_ERR_ARG;
  if ((int64_t)c->width * c->page_size > 0x7ffff000) return EWSJF_ERR_ARG;
  const int64_t D = c->head_dim, block = ewsjf::cache_block(*c), unit = in_codes(c->dtype) ? 16 : 8;
  // a dim of size 1 may have any stride: it is never stepped over
  const bool head = c->kv_heads > 1, token = c->page_size > 1;
  const bool by_head = (!head || c->head_stride == D * c->page_size) && (!token || c->token_stride == D);
  const bool by_token = (!head || c->head_stride == D) && (!token || c->token_stride == D * c->kv_heads);
  if (!by_head && !by_token) return EWSJF_ERR_ARG;
  if (!stride_ok(c->layer_stride, unit) || !stride_ok(c->kv_stride, unit) || !stride_ok(c->page_stride, unit))
    return EWSJF_ERR_ARG;
  const int64_t size[3] = {c->layers, 2, c->n_pages}, stride[3] = {c->layer_stride, c->kv_stride, c->page_stride};
  if (!apart(block, size, stride)) return EWSJF_ERR_ARG;
  if (!aligned16(c->data)) return EWSJF_ERR_ALIGN;
  return EWSJF_OK;
}

bool beams_ok(const ewsjf_beams* b) {
  if (b->groups < 0 || b->groups > EWSJF_MAX_CACHE_BATCH || b->beams < 1 || b->beams > EWSJF_MAX_BEAMS) return false;
  if (b->groups * b->beams > EWSJF_MAX_CACHE_BATCH) return false;
  if (b->picks < 1 || b->picks > EWSJF_MAX_PICKS || b->vocab < 1 || b->vocab > EWSJF_MAX_VOCAB) return false;
  if (b->dtype != EWSJF_BF16 && b->dtype != EWSJF_F16 && b->dtype != EWSJF_F32) return false;
  return b->row_stride >= b->vocab && b->row_stride <= kMaxStride;
}

bool batch_ok(const ewsjf_cache* c, const ewsjf_batch* b) {
  if (b->n_seqs < 0 || b->n_seqs > EWSJF_MAX_CACHE_BATCH || b->n_groups < 0 || b->n_groups > b->n_seqs) return false;
  if (b->total_q < 0 || b->total_q >= kMaxQ || b->max_q < 1) return false;
  if (b->total_q > 0 && b->n_seqs == 0) return false;  // nobody's queries
  if (b->q_heads < 1 || b->q_heads % c->kv_heads || b->q_heads / c->kv_heads > kMaxGroup) return false;
  if (b->window < 0 || b->sinks < 0 || (b->window == 0 && b->sinks > 0)) return false;
  if (b->window > 0 && b->n_groups > 0) return false;
  return c->head_dim == 64 || c->head_dim == 128;
}

ewsjf_status launched(hipError_t e) { return e == hipSuccess ? EWSJF_OK : EWSJF_ERR_LAUNCH; }

ewsjf_status read_rows(const ewsjf_cache* c, int32_t layer, const int32_t* slot, const int32_t* start,
                       const int32_t* begin, int32_t n_seqs, int64_t total, bool all, void* k, void* v,
                       hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (layer < 0 || layer >= c->layers || n_seqs < 0 || n_seqs > EWSJF_MAX_CACHE_BATCH || total < 0 || total > kMaxRead)
    return EWSJF_ERR_ARG;
  if ((n_seqs > 0 || all) && total > 0 && (k == nullptr || v == nullptr)) return EWSJF_ERR_NULL;
  if (n_seqs > 0 && total > 0 && (slot == nullptr || start == nullptr)) return EWSJF_ERR_NULL;
  if (!aligned16(k) || !aligned16(v)) return EWSJF_ERR_ALIGN;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_read(*c, layer, slot, start, begin, n_seqs, total, all, k, v, stream));
}

ewsjf_status plan_status(const ewsjf_cache* c, const ewsjf_batch* b, const int32_t* slot, const int32_t* q_start,
                         const void* plan, size_t plan_bytes) {
  const ewsjf_status cs = cache_status(c);
  if (cs != EWSJF_OK) return cs;
  if (b == nullptr || plan == nullptr) return EWSJF_ERR_NULL;
  if (!batch_ok(c, b)) return EWSJF_ERR_ARG;
  if (b->n_seqs > 0 && (slot == nullptr || q_start == nullptr)) return EWSJF_ERR_NULL;
  if (!aligned16(plan)) return EWSJF_ERR_ALIGN;
  if (plan_bytes < ewsjf::attention_plan_bytes(*c, *b)) return EWSJF_ERR_WORKSPACE;
  return EWSJF_OK;
}

}  // namespace

extern "C" {

size_t ewsjf_cache_workspace_bytes(const ewsjf_cache* c) {
  return cache_status(c) == EWSJF_OK ? ewsjf::cache_ws_bytes(*c) : 0;
}

size_t ewsjf_cache_page_bytes(int32_t page_size, int32_t kv_heads, int32_t head_dim, int32_t dtype) {
  if (!page_ok(page_size, kv_heads, head_dim, dtype)) return 0;
  ewsjf_cache c = {};
  c.page_size = page_size, c.kv_heads = kv_heads, c.head_dim = head_dim, c.dtype = dtype;
  return (size_t)(ewsjf::cache_block(c) * ewsjf::cache_element_bytes(c));
}

ewsjf_status ewsjf_cache_extend(const ewsjf_cache* c, const int32_t* slot, const int32_t* tokens, int32_t n,
                                int32_t* granted, void* ws, size_t ws_bytes, hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (n < 0 || n > EWSJF_MAX_CACHE_BATCH) return EWSJF_ERR_ARG;
  if ((n > 0 && (slot == nullptr || tokens == nullptr || granted == nullptr)) || ws == nullptr) return EWSJF_ERR_NULL;
  if (!aligned16(ws)) return EWSJF_ERR_ALIGN;
  if (ws_bytes < ewsjf::cache_ws_bytes(*c)) return EWSJF_ERR_WORKSPACE;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_grow(*c, nullptr, slot, tokens, n, granted, ws, stream));
}

ewsjf_status ewsjf_cache_fork(const ewsjf_cache* c, const int32_t* parent, const int32_t* child,
                              const int32_t* tokens, int32_t n, int32_t* granted, void* ws, size_t ws_bytes,
                              hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (n < 0 || n > EWSJF_MAX_CACHE_BATCH) return EWSJF_ERR_ARG;
  if ((n > 0 && (parent == nullptr || child == nullptr || tokens == nullptr || granted == nullptr)) || ws == nullptr)
    return EWSJF_ERR_NULL;
  if (!aligned16(ws)) return EWSJF_ERR_ALIGN;
  if (ws_bytes < ewsjf::cache_ws_bytes(*c)) return EWSJF_ERR_WORKSPACE;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_grow(*c, parent, child, tokens, n, granted, ws, stream));
}

ewsjf_status ewsjf_cache_release(const ewsjf_cache* c, const int32_t* slot, const int32_t* begin, const int32_t* end,
                                 int32_t n, hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (n < 0 || n > EWSJF_MAX_CACHE_BATCH) return EWSJF_ERR_ARG;
  if ((n > 0 && slot == nullptr) || (begin == nullptr) != (end == nullptr)) return EWSJF_ERR_NULL;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_release(*c, slot, begin, end, n, stream));
}

ewsjf_status ewsjf_cache_copy(const ewsjf_cache* c, const int32_t* src, const int32_t* dst, int32_t n,
                              hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (n < 0 || n > c->n_pages) return EWSJF_ERR_ARG;
  if (n > 0 && (src == nullptr || dst == nullptr)) return EWSJF_ERR_NULL;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_copy(*c, src, dst, n, stream));
}

ewsjf_status ewsjf_cache_compact(const ewsjf_cache* c, int32_t* out_table, int32_t* out_refs, int32_t* used, void* ws,
                                 size_t ws_bytes, hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (out_table == nullptr || out_refs == nullptr || used == nullptr || ws == nullptr) return EWSJF_ERR_NULL;
  if (!aligned16(ws)) return EWSJF_ERR_ALIGN;
  if (ws_bytes < ewsjf::cache_ws_bytes(*c)) return EWSJF_ERR_WORKSPACE;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_compact(*c, out_table, out_refs, used, ws, stream));
}

ewsjf_status ewsjf_cache_append_granted(const ewsjf_cache* c, int32_t layer, const void* k, const void* v,
                                        int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                        int64_t v_head_stride, const int32_t* slot, const int32_t* q_start,
                                        const int32_t* granted, int32_t n_seqs, int64_t total, hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (layer < 0 || layer >= c->layers || n_seqs < 0 || n_seqs > EWSJF_MAX_CACHE_BATCH || total < 0 || total >= kMaxQ)
    return EWSJF_ERR_ARG;
  if (!stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) ||
      !stride_ok(v_head_stride))
    return EWSJF_ERR_ARG;
  if (n_seqs > 0 && total > 0 && (k == nullptr || v == nullptr || slot == nullptr || q_start == nullptr))
    return EWSJF_ERR_NULL;
  if (!aligned16(k) || !aligned16(v)) return EWSJF_ERR_ALIGN;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  const auto launch = in_codes(c->dtype) ? ewsjf::launch_cache_append_codes : ewsjf::launch_cache_append;
  return launched(launch(*c, layer, k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slot, q_start,
                         granted, n_seqs, total, stream));
}

ewsjf_status ewsjf_cache_append(const ewsjf_cache* c, int32_t layer, const void* k, const void* v,
                                int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                int64_t v_head_stride, const int32_t* slot, const int32_t* q_start, int32_t n_seqs,
                                int64_t total, hipStream_t stream) {
  return ewsjf_cache_append_granted(c, layer, k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slot,
                                    q_start, nullptr, n_seqs, total, stream);
}

ewsjf_status ewsjf_cache_read(const ewsjf_cache* c, int32_t layer, const int32_t* slot, const int32_t* start,
                              const int32_t* begin, int32_t n_seqs, int64_t total, void* k, void* v,
                              hipStream_t stream) {
  return read_rows(c, layer, slot, start, begin, n_seqs, total, false, k, v, stream);
}

ewsjf_status ewsjf_cache_read_all(const ewsjf_cache* c, int32_t layer, const int32_t* slot, const int32_t* start,
                                  const int32_t* begin, int32_t n_seqs, int64_t total, void* k, void* v,
                                  hipStream_t stream) {
  return read_rows(c, layer, slot, start, begin, n_seqs, total, true, k, v, stream);
}

size_t ewsjf_cache_reorder_workspace_bytes(const ewsjf_cache* c, int32_t n) {
  if (cache_status(c) != EWSJF_OK || n < 0 || n > EWSJF_MAX_CACHE_BATCH) return 0;
  return ewsjf::cache_reorder_ws_bytes(*c, n);
}

ewsjf_status ewsjf_cache_reorder(const ewsjf_cache* c, const int32_t* slot, const int32_t* parent, int32_t n,
                                 int32_t* granted, void* ws, size_t ws_bytes, hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (n < 0 || n > EWSJF_MAX_CACHE_BATCH) return EWSJF_ERR_ARG;
  if ((n > 0 && (slot == nullptr || parent == nullptr || granted == nullptr)) || ws == nullptr) return EWSJF_ERR_NULL;
  if (!aligned16(ws)) return EWSJF_ERR_ALIGN;
  if (ws_bytes < ewsjf::cache_reorder_ws_bytes(*c, n)) return EWSJF_ERR_WORKSPACE;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_cache_reorder(*c, slot, parent, n, granted, ws, stream));
}

size_t ewsjf_beam_workspace_bytes(const ewsjf_beams* b) {
  return b != nullptr && beams_ok(b) ? ewsjf::beam_ws_bytes(*b) : 0;
}

ewsjf_status ewsjf_beam_select(const ewsjf_beams* b, const void* logits, const float* score_in, const int32_t* done,
                               int32_t* parent, int32_t* token, float* score, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
  if (b == nullptr || ws == nullptr) return EWSJF_ERR_NULL;
  if (!beams_ok(b) || (done != nullptr && (b->end < 0 || b->end >= b->vocab))) return EWSJF_ERR_ARG;
  if (b->groups > 0 && (logits == nullptr || score_in == nullptr || parent == nullptr || token == nullptr ||
                        score == nullptr))
    return EWSJF_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(logits) & (b->dtype == EWSJF_F32 ? 3 : 1)) || !aligned16(ws)) return EWSJF_ERR_ALIGN;
  if (ws_bytes < ewsjf::beam_ws_bytes(*b)) return EWSJF_ERR_WORKSPACE;
  const ewsjf_status st = ewsjf::device_ok();
  if (st != EWSJF_OK) return st;
  return launched(ewsjf::launch_beam_select(*b, logits, score_in, done, parent, token, score, ws, stream));
}

size_t ewsjf_attention_plan_bytes(const ewsjf_cache* c, const ewsjf_batch* b) {
  return cache_status(c) == EWSJF_OK && b != nullptr && batch_ok(c, b) ? ewsjf::attention_plan_bytes(*c, *b) : 0;
}

size_t ewsjf_attention_workspace_bytes(const ewsjf_cache* c, const ewsjf_batch* b) {
  return cache_status(c) == EWSJF_OK && b != nullptr && batch_ok(c, b) ? ewsjf::attention_ws_bytes(*c, *b) : 0;
}

ewsjf_status ewsjf_prefix_plan(const ewsjf_cache* c, const ewsjf_batch* b, const int32_t* slot,
                               const int32_t* q_start, const int32_t* group_start, const int32_t* shared, void* plan,
                               size_t plan_bytes, hipStream_t stream) {
  ewsjf_status st = plan_status(c, b, slot, q_start, plan, plan_bytes);
  if (st != EWSJF_OK) return st;
  if (b->window != 0) return EWSJF_ERR_ARG;
  if (b->n_groups > 0 && (group_start == nullptr || shared == nullptr)) return EWSJF_ERR_NULL;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_attention_plan(*c, *b, slot, q_start, group_start, shared, plan, stream));
}

ewsjf_status ewsjf_window_plan(const ewsjf_cache* c, const ewsjf_batch* b, const int32_t* slot,
                               const int32_t* q_start, void* plan, size_t plan_bytes, hipStream_t stream) {
  ewsjf_status st = plan_status(c, b, slot, q_start, plan, plan_bytes);
  if (st != EWSJF_OK) return st;
  if (b->window < 1 || b->n_groups != 0) return EWSJF_ERR_ARG;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_attention_plan(*c, *b, slot, q_start, nullptr, nullptr, plan, stream));
}

ewsjf_status ewsjf_attention(const ewsjf_cache* c, const ewsjf_batch* b, int32_t layer, const void* q,
                             int64_t q_token_stride, int64_t q_head_stride, float scale, const void* plan, void* out,
                             float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  ewsjf_status st = cache_status(c);
  if (st != EWSJF_OK) return st;
  if (b == nullptr || plan == nullptr || ws == nullptr) return EWSJF_ERR_NULL;
  if (!batch_ok(c, b) || layer < 0 || layer >= c->layers) return EWSJF_ERR_ARG;
  if (b->total_q > 0 && (q == nullptr || out == nullptr)) return EWSJF_ERR_NULL;
  if (!stride_ok(q_token_stride) || !stride_ok(q_head_stride)) return EWSJF_ERR_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return EWSJF_ERR_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(plan) || !aligned16(ws)) return EWSJF_ERR_ALIGN;
  if (ws_bytes < ewsjf::attention_ws_bytes(*c, *b)) return EWSJF_ERR_WORKSPACE;
  if ((st = ewsjf::device_ok()) != EWSJF_OK) return st;
  return launched(ewsjf::launch_attention(*c, *b, layer, q, q_token_stride, q_head_stride, scale, plan, out, lse, ws,
                                          stream));
}

}  // extern "C"
