// The next tokens of a beam search: the best candidates of each group of beams.
//
// Two kernels.  The first takes a segment of a row's logits into registers, once,
// and leaves the sum of their exponentials and the segment's best `picks`; the
// second, a workgroup a group, joins the sums, scores what is left and ranks it.
//
// Scores are compared across rows, so the logarithms of the sums have to be
// right far beyond the logits' own 8 to 24 bits: with sums in binary32 (errors of
// 1e-7) about one step of 64 groups of eight beams in a hundred would rank two
// candidates the wrong way round.  Exponentials are taken in binary64 to 2e-13:
//   e^x = 2^(n / 256) e^r, n = round(256 x / ln 2), |r| <= ln 2 / 512,
// 2^(n / 256) an exponent and one of 256 numbers in LDS, e^r three terms.
// binary64 adds and fused products run at binary32's rate here.
#include <hip/hip_runtime.h>

#include "ewsjf_cache.h"

namespace ewsjf {
namespace {

constexpr int kThreads = 256;      // of a segment's workgroup
constexpr int kJoinThreads = 1024; // of a group's
constexpr int kMostFound = 2048;   // candidates that a workgroup ranks at once
constexpr int kWanted = 512;       // workgroups that a launch should have
constexpr int kVocabBits = 22, kRowBits = 5;
static_assert(EWSJF_MAX_VOCAB <= 1 << kVocabBits && EWSJF_MAX_BEAMS <= 1 << kRowBits, "a candidate's place is 59 bits");
static_assert(EWSJF_MAX_PICKS <= 64, "thresholds are taken over the lanes of a wave");

// What a segment leaves: sum exp(x) = sum * exp(base).
struct Part {
  double sum, base;
};

struct Sizes {
  int vectors;   // 16-byte pieces of a thread
  int segments;  // of a row
};

Sizes sizes_of(const ewsjf_beams& b) {
  const int in = b.dtype == EWSJF_F32 ? 4 : 8;                 // elements of a piece
  const int64_t pieces = (b.vocab + in - 1 + in - 1) / in;     // of a row that begins anywhere in one
  Sizes s{8, 0};
  for (;; s.vectors /= 2) {
    s.segments = (int)((pieces + kThreads * s.vectors - 1) / (kThreads * s.vectors));
    if (s.vectors == 1 || (int64_t)b.groups * b.beams * s.segments >= kWanted) return s;
  }
}

struct Work {
  Part* part;      // [rows][segments]
  uint64_t* best;  // [rows][segments][picks]: order32(x) << 32 | ~token, 0 for none
  size_t bytes;
};

Work work_of(const ewsjf_beams& b, const Sizes& s, void* base) {
  Work w;
  const size_t parts = (size_t)b.groups * b.beams * s.segments;
  const size_t first = (parts * sizeof(Part) + 255) & ~size_t(255);
  w.part = static_cast<Part*>(base);
  w.best = reinterpret_cast<uint64_t*>(static_cast<char*>(base) + first);
  w.bytes = first + parts * b.picks * sizeof(uint64_t) + 256;
  return w;
}

// Whole numbers in the order of the values; -0 is 0.
__device__ uint32_t order32(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ float value32(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ uint64_t order64(double x) {
  const uint64_t b = __double_as_longlong(x + 0.);
  return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ double value64(uint64_t o) { return __longlong_as_double(o >> 63 ? o & ~(1ull << 63) : ~o); }

// The largest threshold that at least n of the wave's values (M a lane) reach.
template <int Bits, int M, typename K>
__device__ K wave_threshold(const K (&key)[M], int n) {
  K t = 0;
#pragma unroll 1
  for (int bit = 8 * sizeof(K) - 1; bit >= (int)(8 * sizeof(K)) - Bits; --bit) {
    const K next = t | (K)1 << bit;
    int count = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) count += __popcll(__ballot(key[i] >= next));
    if (count >= n) t = next;
  }
  return t;
}

template <typename K>
__device__ K wave_max(K v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const K o = __shfl_xor(v, d);
    if (o > v) v = o;
  }
  return v;
}
__device__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Descending order of n entries in LDS, room up to the next power of two.
template <int Threads, typename Entry, typename Above>
__device__ void sort_entries(Entry* entry, int n, const Entry& none, Above above) {
  int size = 2;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += Threads) entry[i] = none;
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      __syncthreads();
      for (int i = threadIdx.x; i < size / 2; i += Threads) {
        const int a = i / j * 2 * j + i % j, b = a + j;
        const bool down = (a & k) == 0;
        const Entry x = entry[a], y = entry[b];
        if (above(y, x) == down) entry[a] = y, entry[b] = x;
      }
    }
  __syncthreads();
}

// ---------------------------------------------------------------------------
// Segments
// ---------------------------------------------------------------------------
// The largest magnitudes, as whole numbers: of a word, of each half of it.
__device__ uint32_t larger32(uint32_t a, const uint4& v) {
  const uint32_t m = 0x7fffffffu;
  return max(max(max(a, v.x & m), max(v.y & m, v.z & m)), v.w & m);
}
__device__ uint32_t larger16(uint32_t a, const uint4& v) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  auto halves = [](uint32_t x) { return __builtin_bit_cast(u16x2, x & 0x7fff7fffu); };
  const u16x2 x = __builtin_elementwise_max(halves(v.x), halves(v.y));
  const u16x2 y = __builtin_elementwise_max(halves(v.z), halves(v.w));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_elementwise_max(x, y)));
}

template <typename T>
struct Piece;  // 16 bytes of logits
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ uint32_t larger(uint32_t a, const uint4& v) { return larger32(a, v); }
  static __device__ bool has_nan(uint32_t a) { return a > 0x7f800000u; }
  static constexpr uint32_t kNone = 0xff800000u;
  static __device__ float at(const uint4& v, int i) { return __uint_as_float((&v.x)[i]); }
};
template <>
struct Piece<__bf16> {
  static constexpr int N = 8;
  static __device__ uint32_t larger(uint32_t a, const uint4& v) { return larger16(a, v); }
  static __device__ bool has_nan(uint32_t a) { return a >> 16 > 0x7f80u || (a & 0xffffu) > 0x7f80u; }
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ float at(const uint4& v, int i) {
    const uint32_t w = (&v.x)[i / 2];
    return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
  }
};
template <>
struct Piece<_Float16> {
  static constexpr int N = 8;
  static __device__ uint32_t larger(uint32_t a, const uint4& v) { return larger16(a, v); }
  static __device__ bool has_nan(uint32_t a) { return a >> 16 > 0x7c00u || (a & 0xffffu) > 0x7c00u; }
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static __device__ float at(const uint4& v, int i) {
    union {
      uint16_t bits;
      _Float16 x;
    } u;
    u.bits = (uint16_t)((&v.x)[i / 2] >> (i % 2 * 16));
    return (float)u.x;
  }
};

constexpr double kPerLn2 = 369.3299304675746;  // 256 / ln 2
constexpr double kLn2Part = 0.0027076061740622863;  // ln 2 / 256
constexpr double kRound = 6755399441055744.;  // 1.5 2^52: a sum with it is rounded to a whole number, in its low bits

// Workgroup (segment, row).
template <typename T, int NV>
__global__ __launch_bounds__(kThreads) void take_segments(ewsjf_beams b, const T* logits, const float* score_in,
                                                          const int32_t* done, Work w, int segments) {
  using P = Piece<T>;
  constexpr int N = P::N;
  __shared__ double power[256];
  __shared__ uint64_t found[kMostFound];
  __shared__ double sums[kThreads / 64];
  __shared__ float tops[kThreads / 64];
  __shared__ uint32_t least[kThreads / 64];
  __shared__ int count;
  const int row = blockIdx.y, seg = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // rows without candidates are not read
  if (!(score_in[row] > -INFINITY) || (done != nullptr && done[row] != 0)) return;
  const T* x = logits + row * b.row_stride;
  const int skew = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));  // elements of the first piece before the row
  uint4 v[NV];
  const int piece0 = seg * kThreads * NV + threadIdx.x;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t first = (int64_t)(piece0 + i * kThreads) * N - skew;  // token of the piece's first element
    v[i] = make_uint4(P::kNone, P::kNone, P::kNone, P::kNone);
    if (first >= 0 && first + N <= b.vocab) {
      v[i] = *reinterpret_cast<const uint4*>(x + first);
    } else {
      T part[N];
      *reinterpret_cast<uint4*>(part) = v[i];
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (first + j >= 0 && first + j < b.vocab) part[j] = x[first + j];
      v[i] = *reinterpret_cast<const uint4*>(part);
    }
  }
  power[threadIdx.x] = exp2(threadIdx.x / 256.);
  if (threadIdx.x == 0) count = 0;

  // NaN become -inf: the maximum of a signalling NaN and a number is a NaN.
  uint32_t largest = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) largest = P::larger(largest, v[i]);
  if (P::has_nan(largest)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      T part[N];
      *reinterpret_cast<uint4*>(part) = v[i];
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (!(P::at(v[i], j) >= -INFINITY)) part[j] = (T)-INFINITY;
      v[i] = *reinterpret_cast<const uint4*>(part);
    }
  }

  float most[NV], ref;
  double sum, base;
  uint32_t bar;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    most[i] = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) most[i] = fmaxf(most[i], P::at(v[i], j));
    top = fmaxf(top, most[i]);
  }
  constexpr int kBits = __is_same(T, __bf16) ? 16 : 32;
  if (b.picks <= 32 || NV == 1) {
    const uint32_t key[1] = {order32(top)};
    bar = wave_threshold<kBits>(key, b.picks);
  } else {
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) key[i] = order32(most[i]);
    bar = wave_threshold<kBits>(key, b.picks);
  }
  top = wave_max(top);
  if (lane == 0) tops[wave] = top, least[wave] = bar;
  __syncthreads();
  ref = tops[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) ref = fmaxf(ref, tops[i]);
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) bar = least[i] > bar ? least[i] : bar;
  sum = 0., base = ref;
  if (ref == INFINITY) {  // the entries of +inf share the row
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) sum += P::at(v[i], j) == INFINITY ? 1. : 0.;
  } else if (fabsf(ref) < 1e6f) {
    const int from = (int)rint(ref * kPerLn2) >> 8;
    base = from * 0.6931471805599453;
    const float low = ref - 600.f;  // e^-600 of the largest: nothing, and within a binary64's exponents
    double more = 0.;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double y = fmaxf(P::at(v[i], j), low);
        const double t = fma(y, kPerLn2, kRound);
        const int n = (int)__double_as_longlong(t);
        const double r = fma(y, kPerLn2, -(t - kRound));  // in [-1/2, 1/2]
        constexpr double c1 = kLn2Part, c2 = c1 * c1 / 2, c3 = c1 * c1 * c1 / 6;
        const double p = fma(fma(c3, r, c2), r, c1) * r;
        const uint64_t bits = __double_as_longlong(power[n & 255]);
        const uint32_t hi = (uint32_t)(bits >> 32) + ((uint32_t)((n >> 8) - from) << 20);
        const double e = __longlong_as_double((uint64_t)hi << 32 | (uint32_t)bits);
        sum += e;
        more = fma(e, p, more);
      }
    sum += more;
  } else if (ref > -INFINITY) {  // logits so far out that their multiples pass 32 bits
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float y = P::at(v[i], j);
        if (y > -INFINITY) sum += exp((double)y - ref);
      }
  }
  sum = wave_sum(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = sums[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) sum += sums[i];

  // The candidates.
  const float bound = bar > order32(-INFINITY) ? value32(bar) : -INFINITY;  // numbers below are no values
  auto token_of = [&](int i, int j) { return (uint32_t)((piece0 + i * kThreads) * N + j - skew); };
  auto key_of = [&](float y, uint32_t token) { return (uint64_t)order32(y) << 32 | (uint32_t)~token; };
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (most[i] >= bound && most[i] > -INFINITY)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float y = P::at(v[i], j);
        if (y >= bound && y > -INFINITY) {
          const int at = atomicAdd(&count, 1);
          if (at < kMostFound) found[at] = key_of(y, token_of(i, j));
        }
      }
  __syncthreads();
  const int n = count;
  const int64_t out = (int64_t)row * segments + seg;
  if (threadIdx.x == 0) w.part[out] = Part{sum, base};
  uint64_t* best = w.best + out * b.picks;
  if (n <= kThreads) {  // the usual case: an entry a thread, ranked against the others
    const uint64_t mine = (int)threadIdx.x < n ? found[threadIdx.x] : 0;
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += found[i] > mine;
    if ((int)threadIdx.x < n && rank < b.picks) best[rank] = mine;
  } else if (n <= kMostFound) {
    sort_entries<kThreads>(found, n, (uint64_t)0, [](uint64_t p, uint64_t q) { return p > q; });
    if ((int)threadIdx.x < b.picks) best[threadIdx.x] = found[threadIdx.x];
  } else {  // a plateau of equal logits: one pass over the registers a pick
    uint64_t last = ~0ull;
    for (int k = 0; k < b.picks; ++k) {
      uint64_t mine = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float y = P::at(v[i], j);
          const uint64_t key = y > -INFINITY ? key_of(y, token_of(i, j)) : 0;
          if (key < last && key > mine) mine = key;
        }
      mine = wave_max(mine);
      __syncthreads();
      if (lane == 0) found[wave] = mine;
      __syncthreads();
      for (int i = 0; i < kThreads / 64; ++i) mine = found[i] > mine ? found[i] : mine;
      if (threadIdx.x == 0) best[k] = mine;
      last = mine;
    }
  }
  for (int k = n + threadIdx.x; k < b.picks; k += kThreads) best[k] = 0;
}

// ---------------------------------------------------------------------------
// Groups
// ---------------------------------------------------------------------------
// A candidate: its score, then its place, row, logit and token, both in ascending
// numbers.
struct Entry {
  uint64_t score, place;
};
__device__ bool above(const Entry& a, const Entry& b) {
  return a.score != b.score ? a.score > b.score : a.place > b.place;
}

__global__ __launch_bounds__(kJoinThreads) void join_groups(ewsjf_beams b, const float* score_in, const int32_t* done,
                                                            Work w, int segments, int32_t* parent, int32_t* token,
                                                            float* score) {
  constexpr int kWaves = kJoinThreads / 64;
  __shared__ Entry found[kMostFound];
  __shared__ double base[EWSJF_MAX_BEAMS];  // score of a logit of 0
  __shared__ int kind[EWSJF_MAX_BEAMS];     // 0: no candidates, 1: logits, 2: entries of +inf alone, 3: at its end
  __shared__ uint64_t least[kWaves];
  __shared__ Entry tops[kWaves];
  __shared__ int count;
  const int group = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) count = 0;
  for (int r = wave; r < b.beams; r += kWaves) {
    const int row = group * b.beams + r;
    const float s = score_in[row];
    if (!(s > -INFINITY) || (done != nullptr && done[row] != 0)) {
      if (lane == 0) base[r] = s, kind[r] = s > -INFINITY ? 3 : 0;
      continue;
    }
    const Part* part = w.part + (int64_t)row * segments;
    double top = -INFINITY;
    for (int i = lane; i < segments; i += 64) top = fmax(top, part[i].base);
    top = wave_max(top);
    double sum = 0.;
    for (int i = lane; i < segments; i += 64) {
      const Part p = part[i];
      if (p.base == top) sum += p.sum;
      else if (p.base > -INFINITY) sum += p.sum * exp(p.base - top);
    }
    sum = wave_sum(sum);
    if (lane == 0) {
      base[r] = top == INFINITY ? s - log(sum) : s - (top + log(sum));
      kind[r] = top == INFINITY ? 2 : top > -INFINITY ? 1 : 0;
    }
  }
  __syncthreads();

  const int each = segments * b.picks, all = b.beams * each;
  const uint64_t* best = w.best + (int64_t)group * all;
  // Candidate c of the group's; place 0: none.
  auto entry_of = [&](int c) {
    const int r = c / each, k = kind[r];
    Entry e{0, 0};
    const uint64_t before = (uint64_t)((1 << kRowBits) - 1 - r) << (32 + kVocabBits);
    const uint32_t last = (1u << kVocabBits) - 1;
    if (k == 3) {
      if (c == r * each) e = Entry{order64(base[r]), before | 1ull << (31 + kVocabBits) | (last - b.end)};
    } else if (k != 0) {
      const uint64_t key = best[c];
      const uint32_t o = (uint32_t)(key >> 32), v = ~(uint32_t)key;
      const float x = value32(o);
      if (key != 0 && (k == 1 || x == INFINITY))
        e = Entry{order64(k == 1 ? base[r] + x : base[r]), before | (uint64_t)o << kVocabBits | (last - v)};
    }
    return e;
  };
  auto none = [](const Entry& e) { return e.place == 0; };

  uint64_t high[2] = {0, 0};  // a thread's two highest scores
  for (int c = threadIdx.x; c < all; c += kJoinThreads) {
    const Entry e = entry_of(c);
    if (e.score > high[0]) high[1] = high[0], high[0] = e.score;
    else if (e.score > high[1]) high[1] = e.score;
  }
  uint64_t bar = wave_threshold<64>(high, b.picks);
  if (lane == 0) least[wave] = bar;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) bar = least[i] > bar ? least[i] : bar;
  for (int c = threadIdx.x; c < all; c += kJoinThreads) {
    const Entry e = entry_of(c);
    if (!none(e) && e.score >= bar) {
      const int at = atomicAdd(&count, 1);
      if (at < kMostFound) found[at] = e;
    }
  }
  __syncthreads();
  const int n = count;
  auto write = [&](int rank, const Entry& e) {
    const int64_t at = (int64_t)group * b.picks + rank;
    const bool there = !none(e);
    const int r = (1 << kRowBits) - 1 - (int)(e.place >> (32 + kVocabBits));
    parent[at] = there ? group * b.beams + r : -1;
    token[at] = there ? (1 << kVocabBits) - 1 - (int)(e.place & ((1u << kVocabBits) - 1)) : -1;
    score[at] = there ? (float)value64(e.score) : -INFINITY;
  };
  if (n <= kJoinThreads / 4) {
    const Entry mine = (int)threadIdx.x < n ? found[threadIdx.x] : Entry{0, 0};
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += above(found[i], mine);
    if ((int)threadIdx.x < n && rank < b.picks) write(rank, mine);
  } else if (n <= kMostFound) {
    sort_entries<kJoinThreads>(found, n, Entry{0, 0}, above);
    if ((int)threadIdx.x < b.picks) write(threadIdx.x, found[threadIdx.x]);
  } else {  // a plateau of equal scores: one pass over the candidates a pick
    Entry last{~0ull, ~0ull};
    for (int k = 0; k < b.picks; ++k) {
      Entry mine{0, 0};
      for (int c = threadIdx.x; c < all; c += kJoinThreads) {
        const Entry e = entry_of(c);
        if (above(last, e) && above(e, mine)) mine = e;
      }
#pragma unroll
      for (int d = 32; d; d >>= 1) {
        const Entry o{(uint64_t)__shfl_xor(mine.score, d), (uint64_t)__shfl_xor(mine.place, d)};
        if (above(o, mine)) mine = o;
      }
      __syncthreads();
      if (lane == 0) tops[wave] = mine;
      __syncthreads();
      for (int i = 0; i < kWaves; ++i)
        if (above(tops[i], mine)) mine = tops[i];
      if (threadIdx.x == 0) write(k, mine);
      last = mine;
    }
  }
  for (int k = n + threadIdx.x; k < b.picks; k += kJoinThreads) write(k, Entry{0, 0});
}

template <typename T>
void launch_segments(const ewsjf_beams& b, const void* logits, const float* score_in, const int32_t* done,
                     const Work& w, const Sizes& s, hipStream_t stream) {
  auto kernel = s.vectors == 8   ? take_segments<T, 8>
                : s.vectors == 4 ? take_segments<T, 4>
                : s.vectors == 2 ? take_segments<T, 2>
                                 : take_segments<T, 1>;
  kernel<<<dim3(s.segments, b.groups * b.beams), kThreads, 0, stream>>>(b, static_cast<const T*>(logits), score_in,
                                                                        done, w, s.segments);
}

}  // namespace

size_t beam_ws_bytes(const ewsjf_beams& b) { return work_of(b, sizes_of(b), nullptr).bytes; }

hipError_t launch_beam_select(const ewsjf_beams& b, const void* logits, const float* score_in, const int32_t* done,
                              int32_t* parent, int32_t* token, float* score, void* ws, hipStream_t stream) {
  if (b.groups == 0) return hipSuccess;
  const Sizes s = sizes_of(b);
  const Work w = work_of(b, s, ws);
  if (b.dtype == EWSJF_F32) launch_segments<float>(b, logits, score_in, done, w, s, stream);
  else if (b.dtype == EWSJF_BF16) launch_segments<__bf16>(b, logits, score_in, done, w, s, stream);
  else launch_segments<_Float16>(b, logits, score_in, done, w, s, stream);
  join_groups<<<b.groups, kJoinThreads, 0, stream>>>(b, score_in, done, w, s.segments, parent, token, score);
  return hipGetLastError();
}

}  // namespace ewsjf
