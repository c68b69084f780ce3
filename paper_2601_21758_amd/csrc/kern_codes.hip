// Keys and values of an 8-bit cache: quantised as they are written, read back.
//
// A row is a head's elements x of one token.  With top = max |x| and 2^e the
// smallest power of two with top <= 448 2^e, the codes are x / 2^e rounded to
// e4m3 and the row's scale byte is e + 127.  A power of two loses nothing against
// any other scale (codes are floating point: their relative step is the same
// everywhere, and 448 2^e >= top > 224 2^e leaves 14 binades below), divides
// exactly, and makes the values exact in 16 bits: four significant bits.
//
// Both are bound by memory: a token of H heads of D moves 2 H (3 D + 1) bytes.
// 28,000 tokens of 8 heads of 128, 0.17 GB: written in 46 us, 3.8 TB/s; 85,000
// tokens, 0.52 GB, read in 108 us, 4.8 TB/s; eight tokens, 4 us either way.
#include <hip/hip_runtime.h>

#include "ewsjf_cache.h"
#include "ewsjf_codes.h"

namespace ewsjf {
namespace {

constexpr int kThreads = 256;
// Most tokens of a workgroup, and rows of a thread that are on their way.  28,000 tokens of 8 heads of 128: appends of 8
// tokens 46 us, of 16 50, of 4 48; with 2 rows 54, with 8 49; reads 30 us, with 16 tokens 32, with one row 36.
constexpr int kTokens = 8;
constexpr int kRows = 4;
constexpr int kFewSeqs = kThreads - 1;  // sequences whose starts a workgroup reads at once
constexpr int kMostGrid = 65536;

// Where a workgroup's tokens lie, in bytes: (head 0, token) in the layer's keys,
// its scale byte, and the token's row of k and v outside; at < 0: nowhere.
struct Place {
  int64_t at, scale, k, v;
};
constexpr int64_t kNowhere = -1, kNoRow = -2;  // a read's row is 0 there, or stays as it is

// Starts and slots of few sequences in LDS: a token's sequence is found without a
// chain of loads.
struct Seqs {
  int32_t start[kFewSeqs + 1], slot[kFewSeqs + 1];
  __device__ void take(const int32_t*& slots, const int32_t*& starts, int n_seqs) {
    if (n_seqs > kFewSeqs) return;
    if ((int)threadIdx.x <= n_seqs) start[threadIdx.x] = starts[threadIdx.x];
    if ((int)threadIdx.x < n_seqs) slot[threadIdx.x] = slots[threadIdx.x];
    starts = start, slots = slot;
  }
};

__device__ int last_at_most(const int32_t* key, int n, int64_t v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (key[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ Place place_of(const ewsjf_cache& c, int64_t page, int pos) {
  const int in = pos & (c.page_size - 1), bytes = cache_element_bytes(c);
  const int64_t block = page * c.page_stride;
  return Place{(block + in * c.token_stride) * bytes, block + (int64_t)c.kv_heads * c.page_size * c.head_dim + in, 0, 0};
}

// Token t's place, as the cache's append finds it: what is not granted, not
// held or shared with other rows is not written.
__device__ Place written_place(const ewsjf_cache& c, const int32_t* slot, const int32_t* q_start,
                               const int32_t* granted, int n_seqs, int64_t t) {
  const Place nowhere{kNowhere, 0, 0, 0};
  const int i = last_at_most(q_start, n_seqs, t), s = slot[i], a = q_start[i], e = q_start[i + 1];
  if (s < 0 || s >= c.n_slots || t < a || t >= e || (granted != nullptr && granted[i] == 0)) return nowhere;
  const int shift = __builtin_ctz(c.page_size), have = c.length[s] < 0 ? 0 : c.length[s], pos = have - (int)(e - t);
  if (pos < 0 || pos >> shift >= c.width) return nowhere;
  const int page = c.table[(int64_t)s * c.width + (pos >> shift)];
  if (page < 0 || page >= c.n_pages) return nowhere;
  if (granted == nullptr && pos >> shift < have >> shift && c.refs[page] > 1) return nowhere;
  return place_of(c, page, pos);
}

// Row t's place of a read; all: a row that no sequence has is 0 too.
__device__ Place read_place(const ewsjf_cache& c, const int32_t* slot, const int32_t* start, const int32_t* begin,
                            int n_seqs, int64_t t, bool all) {
  const Place nowhere{kNowhere, 0, 0, 0}, no_row{all ? kNowhere : kNoRow, 0, 0, 0};
  if (n_seqs == 0) return no_row;
  const int i = last_at_most(start, n_seqs, t), s = slot[i];
  const int64_t a = start[i], e = start[i + 1];
  if (t < a || t >= e) return no_row;
  if (s < 0 || s >= c.n_slots) return nowhere;
  const int64_t pos = (begin != nullptr ? begin[i] : 0) + t - a;
  const int shift = __builtin_ctz(c.page_size);
  if (pos < 0 || pos >= c.length[s] || pos >> shift >= c.width) return nowhere;
  const int page = c.table[(int64_t)s * c.width + (pos >> shift)];
  if (page < 0 || page >= c.n_pages) return nowhere;
  return place_of(c, page, (int)pos);
}

// The rows of a workgroup's tokens that a thread has: token, then keys or
// values, then head, `each` rows on at a time without a division.
struct Row {
  int token, part;  // part: the head, behind all heads for values
  int tokens_on, parts_on, parts;
  __device__ Row(int first, int each, int heads) {
    parts = 2 * heads;
    token = first / parts, part = first - token * parts;
    tokens_on = each / parts, parts_on = each - tokens_on * parts;
  }
  __device__ void next() {
    token += tokens_on, part += parts_on;
    if (part >= parts) part -= parts, ++token;
  }
};

// e + 127 of a row whose largest magnitude is `top`.  448 = 1.75 2^8: with top = f 2^k, e is k - 8, one more if f > 1.75.
__device__ int scale_byte(float top) {
  const int up = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8;
  return up < 127 - 117 ? 127 - 117 : up;
}

// The bits of a magnitude in 16 bits, in its order, and back.
__device__ uint32_t bits_of(float y, __bf16) { return __float_as_uint(y) >> 16; }
__device__ uint32_t bits_of(float y, _Float16) { return __builtin_bit_cast(uint16_t, (_Float16)y); }
__device__ float value_of(uint32_t bits, __bf16) { return __uint_as_float(bits << 16); }
__device__ float value_of(uint32_t bits, _Float16) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }

// The largest magnitude of eight numbers of 16 bits, as bits; a NaN is above all.
__device__ uint32_t largest(const uint4& w) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  auto size = [](uint32_t x) { return __builtin_bit_cast(u16x2, x & 0x7fff7fffu); };
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(size(w.x), size(w.y)),
                                            __builtin_elementwise_max(size(w.z), size(w.w)));
  return m[0] > m[1] ? m[0] : m[1];
}

template <int Control>
__device__ uint32_t moved_max(uint32_t v) {
  const uint32_t o = __builtin_amdgcn_update_dpp(v, v, Control, 0xf, 0xf, false);
  return o > v ? o : v;
}
// Over a row's lanes, a power of two up to 32 that the wave is divided into.
__device__ uint32_t row_max(uint32_t v, int lanes) {
  if (lanes > 1) v = moved_max<0xb1>(v);   // the neighbour,
  if (lanes > 2) v = moved_max<0x4e>(v);   // two away,
  if (lanes > 4) v = moved_max<0x141>(v);  // the other half of eight,
  if (lanes > 8) v = moved_max<0x140>(v);  // of sixteen
  if (lanes > 16) {
    const uint32_t o = __shfl_xor(v, 16);
    v = o > v ? o : v;
  }
  return v;
}

// Lanes of a row, 8 elements each: a power of two, so that a row's lanes are a group of a wave.
__host__ __device__ int lanes_of(int head_dim) {
  int g = 1;
  while (8 * g < head_dim) g *= 2;
  return g;
}

template <typename T, int kRows>
__global__ __launch_bounds__(kThreads) void append_codes(ewsjf_cache c, int layer, const T* k, const T* v,
                                                         int64_t k_token, int64_t k_head, int64_t v_token,
                                                         int64_t v_head, const int32_t* slot, const int32_t* q_start,
                                                         const int32_t* granted, int n_seqs, int64_t total,
                                                         int tokens) {
  __shared__ Place place[kTokens];
  const int lanes = lanes_of(c.head_dim), each = kThreads / lanes;
  const int lane = threadIdx.x & (lanes - 1), d = lane * 8;
  const bool busy = d < c.head_dim;
  char* data = static_cast<char*>(c.data) + layer * c.layer_stride;
  const float most = cache_most(c);
  __shared__ Seqs seqs;
  seqs.take(slot, q_start, n_seqs);
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < total; t0 += (int64_t)gridDim.x * tokens) {
    const int n = total - t0 < tokens ? (int)(total - t0) : tokens;
    __syncthreads();
    if ((int)threadIdx.x < n) {
      const int64_t t = t0 + threadIdx.x;
      Place p = written_place(c, slot, q_start, granted, n_seqs, t);
      p.k = t * k_token, p.v = t * v_token;
      place[threadIdx.x] = p;
    }
    __syncthreads();
    for (Row r(threadIdx.x / lanes, each, c.kv_heads); r.token < n;) {
      vec8<T> in[kRows];
      int64_t to[kRows], scale[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const bool there = r.token < n;
        const Place p = place[there ? r.token : 0];
        const bool x = r.part >= c.kv_heads;
        const int h = r.part - (x ? c.kv_heads : 0);
        const int64_t plane = x ? c.kv_stride : 0;
        // a block has less than 2^31 bytes
        to[u] = there && p.at >= 0 ? plane + p.at + (uint32_t)h * (uint32_t)c.head_stride + d : -1;
        scale[u] = plane + p.scale + (uint32_t)h * (uint32_t)c.page_size;
        const T* from = to[u] < 0 ? k : (x ? v + p.v + h * v_head : k + p.k + h * k_head) + d;
        in[u] = *reinterpret_cast<const vec8<T>*>(busy ? from : k);
        r.next();
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const uint4 w = busy ? __builtin_bit_cast(uint4, in[u]) : make_uint4(0, 0, 0, 0);
        uint32_t top = row_max(largest(w), lanes);  // of the magnitudes' bits
        const vec8<T> x8 = __builtin_bit_cast(vec8<T>, w);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = (float)x8[j];
        if (top > bits_of(most, T())) {  // a magnitude that is cut off, or a NaN
          float size = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            y[j] = y[j] > most ? most : y[j] < -most ? -most : y[j];  // a NaN stays
            size = fabsf(y[j]) > size ? fabsf(y[j]) : size;           // and does not count
          }
          top = row_max(bits_of(size, T()), lanes);
        }
        const int byte = scale_byte(value_of(top, T()));
        const float inv = scale_of(254 - byte);  // 2^-e
        uint32_t lo = 0, hi = 0;
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * inv, y[5] * inv, hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * inv, y[7] * inv, hi, true);
        if (to[u] < 0) continue;
        if (busy) *reinterpret_cast<uint2*>(data + to[u]) = make_uint2(lo, hi);
        if (lane == 0) data[scale[u]] = (char)byte;
      }
    }
  }
}

template <typename T, bool Codes, int kRows>
__global__ __launch_bounds__(kThreads) void read_tokens(ewsjf_cache c, int layer, const int32_t* slot,
                                                        const int32_t* start, const int32_t* begin, int n_seqs,
                                                        int64_t total, bool all, T* k, T* v, int tokens) {
  constexpr int kBytes = Codes ? 1 : 2;
  __shared__ Place place[kTokens];
  const int lanes = lanes_of(c.head_dim), each = kThreads / lanes;
  const int d = (threadIdx.x & (lanes - 1)) * 8;
  const char* data = static_cast<const char*>(c.data) + layer * c.layer_stride * kBytes;
  __shared__ Seqs seqs;
  if (n_seqs > 0) seqs.take(slot, start, n_seqs);
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < total; t0 += (int64_t)gridDim.x * tokens) {
    const int n = total - t0 < tokens ? (int)(total - t0) : tokens;
    __syncthreads();
    if ((int)threadIdx.x < n) {
      const int64_t t = t0 + threadIdx.x;
      Place p = read_place(c, slot, start, begin, n_seqs, t, all);
      p.k = p.v = t * (c.kv_heads * c.head_dim);
      place[threadIdx.x] = p;
    }
    __syncthreads();
    for (Row r(threadIdx.x / lanes, each, c.kv_heads); r.token < n;) {
      uint4 in[kRows];
      uint8_t scale[kRows];
      bool held[kRows];
      T* to[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const bool there = r.token < n && d < c.head_dim;
        const Place p = place[there ? r.token : 0];
        const bool x = r.part >= c.kv_heads;
        const uint32_t h = r.part - (x ? c.kv_heads : 0);
        const int64_t plane = x ? c.kv_stride * kBytes : 0;
        held[u] = there && p.at >= 0;
        to[u] = there && p.at != kNoRow ? (x ? v : k) + p.k + h * c.head_dim + d : nullptr;
        const char* at = data + (held[u] ? plane + p.at + (h * (uint32_t)c.head_stride + d) * kBytes : 0);
        if (Codes) {
          const uint2 codes = *reinterpret_cast<const uint2*>(at);
          in[u] = make_uint4(codes.x, codes.y, 0, 0);
          scale[u] = (uint8_t)data[held[u] ? plane + p.scale + h * (uint32_t)c.page_size : 0];
        } else {
          in[u] = *reinterpret_cast<const uint4*>(at);
        }
        r.next();
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        vec8<T> y = Codes ? values_of(make_uint2(in[u].x, in[u].y), scale_of(scale[u]), T()) : __builtin_bit_cast(vec8<T>, in[u]);
        if (!held[u]) y = vec8<T>{};
        if (to[u] != nullptr) *reinterpret_cast<vec8<T>*>(to[u]) = y;
      }
    }
  }
}

// Tokens of a workgroup: as many as leave the chip four workgroups a CU.
int tokens_each(int64_t total) {
  const int64_t n = total / 1024;
  return n < 1 ? 1 : n > kTokens ? kTokens : (int)n;
}
// A thread has one row of a workgroup's tokens at most.
bool one_pass(const ewsjf_cache& c, int tokens) { return tokens * 2 * c.kv_heads * lanes_of(c.head_dim) <= kThreads; }
unsigned grid_of(int64_t total, int tokens) {
  const int64_t n = (total + tokens - 1) / tokens;
  return (unsigned)(n < kMostGrid ? n : kMostGrid);
}

}  // namespace

hipError_t launch_cache_append_codes(const ewsjf_cache& c, int32_t layer, const void* k, const void* v,
                                     int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head,
                                     const int32_t* slot, const int32_t* q_start, const int32_t* granted,
                                     int32_t n_seqs, int64_t total, hipStream_t stream) {
  if (n_seqs == 0 || total == 0) return hipSuccess;
  const int tokens = tokens_each(total);
  auto go = [&](auto type, auto kernel) {
    using T = decltype(type);
    kernel<<<grid_of(total, tokens), kThreads, 0, stream>>>(
        c, layer, static_cast<const T*>(k), static_cast<const T*>(v), k_token, k_head, v_token, v_head, slot, q_start,
        granted, n_seqs, total, tokens);
  };
  const bool one = one_pass(c, tokens);
  if (c.dtype == EWSJF_E4M3_BF16) go(__bf16(), one ? append_codes<__bf16, 1> : append_codes<__bf16, kRows>);
  else go(_Float16(), one ? append_codes<_Float16, 1> : append_codes<_Float16, kRows>);
  return hipGetLastError();
}

hipError_t launch_cache_read(const ewsjf_cache& c, int32_t layer, const int32_t* slot, const int32_t* start,
                             const int32_t* begin, int32_t n_seqs, int64_t total, bool all, void* k, void* v,
                             hipStream_t stream) {
  if ((n_seqs == 0 && !all) || total == 0) return hipSuccess;
  const int tokens = tokens_each(total);
  auto go = [&](auto type, auto one, auto many) {
    using T = decltype(type);
    (one_pass(c, tokens) ? one : many)<<<grid_of(total, tokens), kThreads, 0, stream>>>(
        c, layer, slot, start, begin, n_seqs, total, all, static_cast<T*>(k), static_cast<T*>(v), tokens);
  };
  if (c.dtype == EWSJF_E4M3_BF16) go(__bf16(), read_tokens<__bf16, true, 1>, read_tokens<__bf16, true, kRows>);
  else if (c.dtype == EWSJF_E4M3_F16) go(_Float16(), read_tokens<_Float16, true, 1>, read_tokens<_Float16, true, kRows>);
  else if (c.dtype == EWSJF_BF16) go(__bf16(), read_tokens<__bf16, false, 1>, read_tokens<__bf16, false, kRows>);
  else go(_Float16(), read_tokens<_Float16, false, 1>, read_tokens<_Float16, false, kRows>);
  return hipGetLastError();
}

}  // namespace ewsjf
