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

size_t attention_plan_bytes(const ewsjf_cache& c, const ewsjf_batch& b);
size_t attention_ws_bytes(const ewsjf_cache& c, const ewsjf_batch& b);
hipError_t launch_attention_plan(const ewsjf_cache& c, const ewsjf_batch& b, const int32_t* slot,
                                 const int32_t* q_start, const int32_t* group_start, const int32_t* shared,
                                 void* plan, hipStream_t stream);
hipError_t launch_attention(const ewsjf_cache& c, const ewsjf_batch& b, int32_t layer, const void* q, int64_t q_token,
                            int64_t q_head, float scale, const void* plan, void* out, float* lse, void* ws,
                            hipStream_t stream);

}  // namespace ewsjf
