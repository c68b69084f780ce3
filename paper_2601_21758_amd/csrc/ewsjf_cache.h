// Launch entry points of the paged key/value cache and its attention, called
// by the C ABI layer after it has validated every argument.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ewsjf.h"

namespace ewsjf {

// gfx950 is current (the C ABI's device check).
ewsjf_status device_ok();

// An element of the data is a byte of an 8-bit cache; a page's block of elements
// has the scales behind the codes there.
__host__ __device__ inline bool cache_in_codes(const ewsjf_cache& c) { return c.dtype >= EWSJF_E4M3_BF16; }
__host__ __device__ inline int cache_element_bytes(const ewsjf_cache& c) { return cache_in_codes(c) ? 1 : 2; }
__host__ __device__ inline int64_t cache_block(const ewsjf_cache& c) {
  const int64_t rows = (int64_t)c.kv_heads * c.page_size;
  return cache_in_codes(c) ? (rows * (c.head_dim + 1) + 15) / 16 * 16 : rows * c.head_dim;
}
// Largest magnitude that is quantised, 1.875 2^127 or 1.875 2^15: the next, 2^128
// or 2^16, the type does not hold.
__host__ __device__ inline float cache_most(const ewsjf_cache& c) {
  return c.dtype == EWSJF_E4M3_BF16 ? 0x1.ep127f : 0x1.ep15f;
}

size_t cache_ws_bytes(const ewsjf_cache& c);
// tokens for extend; parent != nullptr: a fork of slot[i] from parent[i].
hipError_t launch_cache_grow(const ewsjf_cache& c, const int32_t* parent, const int32_t* slot, const int32_t* tokens,
                             int32_t n, int32_t* granted, void* ws, hipStream_t stream);
hipError_t launch_cache_release(const ewsjf_cache& c, const int32_t* slot, const int32_t* begin, const int32_t* end,
                                int32_t n, hipStream_t stream);
hipError_t launch_cache_copy(const ewsjf_cache& c, const int32_t* src, const int32_t* dst, int32_t n,
                             hipStream_t stream);
hipError_t launch_cache_compact(const ewsjf_cache& c, int32_t* out_table, int32_t* out_refs, int32_t* used, void* ws,
                                hipStream_t stream);
hipError_t launch_cache_append(const ewsjf_cache& c, int32_t layer, const void* k, const void* v, int64_t k_token,
                               int64_t k_head, int64_t v_token, int64_t v_head, const int32_t* slot,
                               const int32_t* q_start, const int32_t* granted, int32_t n_seqs, int64_t total,
                               hipStream_t stream);

hipError_t launch_cache_append_codes(const ewsjf_cache& c, int32_t layer, const void* k, const void* v,
                                     int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head,
                                     const int32_t* slot, const int32_t* q_start, const int32_t* granted,
                                     int32_t n_seqs, int64_t total, hipStream_t stream);
hipError_t launch_cache_read(const ewsjf_cache& c, int32_t layer, const int32_t* slot, const int32_t* start,
                             const int32_t* begin, int32_t n_seqs, int64_t total, bool all, void* k, void* v,
                             hipStream_t stream);
size_t cache_reorder_ws_bytes(const ewsjf_cache& c, int32_t n);
hipError_t launch_cache_reorder(const ewsjf_cache& c, const int32_t* slot, const int32_t* parent, int32_t n,
                                int32_t* granted, void* ws, hipStream_t stream);

size_t beam_ws_bytes(const ewsjf_beams& b);
hipError_t launch_beam_select(const ewsjf_beams& b, const void* logits, const float* score_in, const int32_t* done,
                              int32_t* parent, int32_t* token, float* score, void* ws, hipStream_t stream);

size_t attention_plan_bytes(const ewsjf_cache& c, const ewsjf_batch& b);
size_t attention_ws_bytes(const ewsjf_cache& c, const ewsjf_batch& b);
hipError_t launch_attention_plan(const ewsjf_cache& c, const ewsjf_batch& b, const int32_t* slot,
                                 const int32_t* q_start, const int32_t* group_start, const int32_t* shared,
                                 void* plan, hipStream_t stream);
hipError_t launch_attention(const ewsjf_cache& c, const ewsjf_batch& b, int32_t layer, const void* q, int64_t q_token,
                            int64_t q_head, float scale, const void* plan, void* out, float* lse, void* ws,
                            hipStream_t stream);

}  // namespace ewsjf
