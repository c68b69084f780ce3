// Attention over the paged key/value cache.
#include <hip/hip_runtime.h>

#include "ewsjf_cache.h"

namespace ewsjf {
namespace {

// A query token's slot (-1: none) and position.
struct Token {
  int32_t slot, pos;
};

__global__ void plan_tokens(ewsjf_cache c, const int32_t* slot, const int32_t* q_start, int64_t total, Token* plan) {
  const int s = blockIdx.x;
  int64_t a = q_start[s], e = q_start[s + 1];
  if (a < 0 || e < a || e > total) return;
  const int r = slot[s];
  const bool ok = r >= 0 && r < c.n_slots;
  int64_t n = ok ? c.length[r] : 0;
  const int64_t room = (int64_t)c.width * c.page_size;
  n = n < 0 ? 0 : n > room ? room : n;
  for (int64_t t = a + threadIdx.x; t < e; t += blockDim.x) plan[t] = Token{ok ? r : -1, (int32_t)(n - (e - t))};
}

__device__ float to_f32(__bf16 x) { return (float)x; }
__device__ float to_f32(_Float16 x) { return (float)x; }

__device__ float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ float wave_sum(float v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// One wave a query head of a token: 64 keys at a time, one key a lane, with the
// running maximum m and sum l of the softmax; then the lanes share the dims.
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_simple(ewsjf_cache c, ewsjf_batch b, const T* data, const T* q,
                                                     int64_t q_token, int64_t q_head, float scale, const Token* plan,
                                                     T* out, float* lse) {
  __shared__ float query[4][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = blockIdx.x;
  const int head = blockIdx.y * 4 + wave;
  if (head >= b.q_heads) return;
  for (int d = lane; d < D; d += 64) query[wave][d] = to_f32(q[t * q_token + head * q_head + d]);
  __builtin_amdgcn_wave_barrier();
  const Token me = plan[t];
  const int h = head / (b.q_heads / c.kv_heads);
  const int32_t* row = c.table + (int64_t)(me.slot < 0 ? 0 : me.slot) * c.width;
  const int64_t last = me.slot < 0 ? -1 : me.pos;
  float m = -3e38f, l = 0.f, o[D / 64] = {};
  for (int64_t k0 = 0; k0 <= last; k0 += 64) {
    if (b.window > 0 && k0 >= b.sinks && k0 + 63 <= last - b.window) continue;
    const int64_t j = k0 + lane;
    const bool seen = j <= last && (b.window == 0 || j > last - b.window || j < b.sinks);
    int page = seen ? row[j / c.page_size] : -1;
    if (page >= c.n_pages) page = -1;
    const T* at = data + (page < 0 ? 0 : page) * c.page_stride + h * c.head_stride + (j % c.page_size) * c.token_stride;
    float s = -INFINITY;
    if (page >= 0) {
      s = 0.f;
      for (int d = 0; d < D; ++d) s = fmaf(query[wave][d], to_f32(at[d]), s);
      s *= scale;
    }
    const float top = fmaxf(m, wave_max(s)), shrink = __expf(m - top);
    const float p = page >= 0 ? __expf(s - top) : 0.f;
    l = l * shrink + wave_sum(p);
    m = top;
    for (int d = 0; d < D / 64; ++d) o[d] *= shrink;
    const uint64_t here = __ballot(page >= 0);
    const uint64_t addr = reinterpret_cast<uint64_t>(at + c.kv_stride);
    for (int i = 0; i < 64; ++i) {
      if (!(here >> i & 1)) continue;
      const float w = __shfl(p, i);
      const T* v = reinterpret_cast<const T*>(__shfl(addr, i));
      for (int d = 0; d < D / 64; ++d) o[d] = fmaf(w, to_f32(v[d * 64 + lane]), o[d]);
    }
  }
  for (int d = 0; d < D / 64; ++d)
    out[(t * b.q_heads + head) * D + d * 64 + lane] = (T)(l > 0.f || l != l ? o[d] / l : 0.f);
  if (lse != nullptr && lane == 0) lse[t * b.q_heads + head] = l > 0.f || l != l ? m + __logf(l) : -INFINITY;
}

}  // namespace

size_t attention_plan_bytes(const ewsjf_cache& c, const ewsjf_batch& b) {
  return 256 + sizeof(Token) * (size_t)b.total_q;
}
size_t attention_ws_bytes(const ewsjf_cache& c, const ewsjf_batch& b) { return 256; }

hipError_t launch_attention_plan(const ewsjf_cache& c, const ewsjf_batch& b, const int32_t* slot,
                                 const int32_t* q_start, const int32_t* group_start, const int32_t* shared,
                                 void* plan, hipStream_t stream) {
  if (b.n_seqs == 0) return hipSuccess;
  plan_tokens<<<b.n_seqs, 256, 0, stream>>>(c, slot, q_start, b.total_q, static_cast<Token*>(plan));
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_typed(const ewsjf_cache& c, const ewsjf_batch& b, int32_t layer, const void* q, int64_t q_token,
                        int64_t q_head, float scale, const void* plan, void* out, float* lse, hipStream_t stream) {
  const T* data = static_cast<const T*>(c.data) + layer * c.layer_stride;
  attend_simple<T, D><<<dim3((unsigned)b.total_q, (b.q_heads + 3) / 4), 256, 0, stream>>>(
      c, b, data, static_cast<const T*>(q), q_token, q_head, scale, static_cast<const Token*>(plan),
      static_cast<T*>(out), lse);
  return hipGetLastError();
}

hipError_t launch_attention(const ewsjf_cache& c, const ewsjf_batch& b, int32_t layer, const void* q, int64_t q_token,
                            int64_t q_head, float scale, const void* plan, void* out, float* lse, void* ws,
                            hipStream_t stream) {
  if (b.total_q == 0 || b.n_seqs == 0) return hipSuccess;
  auto go = [&](auto run) { return run(c, b, layer, q, q_token, q_head, scale, plan, out, lse, stream); };
  if (c.dtype == EWSJF_BF16) return c.head_dim == 64 ? go(launch_typed<__bf16, 64>) : go(launch_typed<__bf16, 128>);
  return c.head_dim == 64 ? go(launch_typed<_Float16, 64>) : go(launch_typed<_Float16, 128>);
}

}  // namespace ewsjf
