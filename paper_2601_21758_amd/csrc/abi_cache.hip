// C ABI of the key/value cache and its attention: argument checks on the host,
// then launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>

#include "ewsjf.h"
#include "ewsjf_cache.h"

namespace {

constexpr int32_t kMaxGroup = 64;              // query heads per key head
constexpr int64_t kMaxQ = (int64_t)1 << 24;    // query tokens of a batch
constexpr int64_t kMaxStride = (int64_t)1 << 48;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride && s % 8 == 0; }

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

ewsjf_status cache_status(const ewsjf_cache* c) {
  if (c == nullptr) return EWSJF_ERR_NULL;
  if (c->data == nullptr || c->refs == nullptr || c->table == nullptr || c->length == nullptr) return EWSJF_ERR_NULL;
  if (c->layers < 1 || c->layers > 4096 || c->n_pages < 1 || c->n_pages > EWSJF_MAX_PAGES) return EWSJF_ERR_ARG;
  if (c->page_size < 1 || c->page_size > EWSJF_MAX_PAGE_SIZE || (c->page_size & (c->page_size - 1)))
    return EWSJF_ERR_ARG;
  if (c->kv_heads < 1 || c->kv_heads > 1024) return EWSJF_ERR_ARG;
  if (c->head_dim < 8 || c->head_dim > EWSJF_MAX_HEAD_DIM || c->head_dim % 8) return EWSJF_ERR_ARG;
  if (c->dtype != EWSJF_BF16 && c->dtype != EWSJF_F16) return EWSJF_ERR_ARG;
  if (c->n_slots < 1 || c->n_slots > (1 << 24) || c->width < 1) return EWSJF_ERR_ARG;
  if ((int64_t)c->width * c->page_size > 0x7ffff000) return EWSJF_ERR_ARG;
  const int64_t D = c->head_dim, block = D * c->page_size * c->kv_heads;
  // a dim of size 1 may have any stride: it is never stepped over
  const bool head = c->kv_heads > 1, token = c->page_size > 1;
  const bool by_head = (!head || c->head_stride == D * c->page_size) && (!token || c->token_stride == D);
  const bool by_token = (!head || c->head_stride == D) && (!token || c->token_stride == D * c->kv_heads);
  if (!by_head && !by_token) return EWSJF_ERR_ARG;
  if (!stride_ok(c->layer_stride) || !stride_ok(c->kv_stride) || !stride_ok(c->page_stride)) return EWSJF_ERR_ARG;
  const int64_t size[3] = {c->layers, 2, c->n_pages}, stride[3] = {c->layer_stride, c->kv_stride, c->page_stride};
  if (!apart(block, size, stride)) return EWSJF_ERR_ARG;
  if (!aligned16(c->data)) return EWSJF_ERR_ALIGN;
  return EWSJF_OK;
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
  return launched(ewsjf::launch_cache_append(*c, layer, k, v, k_token_stride, k_head_stride, v_token_stride,
                                             v_head_stride, slot, q_start, granted, n_seqs, total, stream));
}

ewsjf_status ewsjf_cache_append(const ewsjf_cache* c, int32_t layer, const void* k, const void* v,
                                int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                int64_t v_head_stride, const int32_t* slot, const int32_t* q_start, int32_t n_seqs,
                                int64_t total, hipStream_t stream) {
  return ewsjf_cache_append_granted(c, layer, k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slot,
                                    q_start, nullptr, n_seqs, total, stream);
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
