// The next tokens of a beam search: the best candidates of each group of beams.
//
// Two kernels.  The first takes a segment of a row's logits into registers, once,
// and leaves the sum of their exponentials and the segment's best `picks`; the
// second, a workgroup a group, joins the sums, scores what is left and ranks it.
//
// Scores are compared across rows, so the logarithms of the sums have to be
// right far beyond the logits' own 8 to 24 bits: with sums right to 1e-7, about
// one call in a hundred with 64 groups of eight beams would rank two candidates the
// wrong way round.  So exponentials are taken to 5e-10 and summed in binary64:
//   e^x = 2^(n / 256) e^r, n = round(256 x / ln 2), |r| <= ln 2 / 512,
// 2^(n / 256) an exponent and one of 256 numbers in LDS, e^r - 1 two terms in
// binary32 (the third is at most 4e-10, of the sign of r).  binary64 adds and
// fused products take 4.7 cycles of a SIMD, as integers and binary32's fused
// products of three registers do (4.5); binary32 with two registers takes 2.6.
#include <hip/hip_runtime.h>

#include "ewsjf_cache.h"

namespace ewsjf {
namespace {

constexpr int kThreads = 256;      // of a segment's workgroup
constexpr int kWaves = kThreads / 64;
constexpr int kWavePieces = 128;   // pieces with candidates that a wave keeps: above its threshold less than picks, at it picks
constexpr int kListed = kWaves * (EWSJF_MAX_PICKS - 1) * 8 + kWaves * EWSJF_MAX_PICKS;  // candidates of a segment, at most
constexpr int kJoinThreads = 1024; // of a group's workgroup
constexpr int kMostFound = 2048;   // candidates of a group that are ranked at once
constexpr int kWanted = 512;       // workgroups that a launch should have: a thread has as many pieces as leave them
constexpr int kVocabBits = 22, kRowBits = 5;
static_assert(EWSJF_MAX_VOCAB <= 1 << kVocabBits && EWSJF_MAX_BEAMS <= 1 << kRowBits, "a candidate's place is 59 bits");
static_assert(EWSJF_MAX_PICKS <= 64, "thresholds are taken over the lanes of a wave");
static_assert(kWavePieces >= 2 * EWSJF_MAX_PICKS - 1, "a wave keeps all pieces with candidates");

// What a segment leaves: sum exp(x) = sum * exp(base).
struct Part {
  double sum, base;
};

struct Sizes {
  int vectors;   // 16-byte pieces of a thread
  int segments;  // of a row
};

// skew: elements that a row's first piece has before it, at most (the workspace is sized for any).
Sizes sizes_of(const ewsjf_beams& b, int skew) {
  const int in = b.dtype == EWSJF_F32 ? 4 : 8;  // elements of a piece
  auto segments = [&](int vectors, int skew) {
    const int64_t pieces = (b.vocab + skew + in - 1) / in;
    return (int)((pieces + kThreads * vectors - 1) / (kThreads * vectors));
  };
  int vectors = 8;
  while (vectors > 1 && (int64_t)b.groups * b.beams * segments(vectors, in - 1) < kWanted) vectors /= 2;
  return Sizes{vectors, segments(vectors, skew < 0 ? in - 1 : skew)};
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
#pragma unroll  // rolled, a call of 4 rows takes 5.7 + 7.1 us for 5.2 + 6.5; two bits a step, three thresholds at once, 5.5 + 7.1
  for (int bit = 8 * sizeof(K) - 1; bit >= (int)(8 * sizeof(K)) - Bits; --bit) {
    const K next = t | (K)1 << bit;
    int count = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) count += __popcll(__ballot(key[i] >= next));
    if (count >= n) t = next;
  }
  return t;
}

// Lanes below this one whose bit is set.
__device__ int bits_below(uint64_t bits) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
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
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
template <typename F>
__device__ u32x4 each_word(u32x4 v, F f) { return u32x4{f(v.x), f(v.y), f(v.z), f(v.w)}; }
// 16 bytes of logits.  `order`: a word's logits as whole numbers in their order, with a sign; a NaN without one is above
// infinity, one with a sign below all.  `clamp`: to at least the negative `low`, a NaN with a sign among them.
__device__ uint32_t order_of(uint32_t w, float) { return w ^ ((uint32_t)((int32_t)w >> 31) & 0x7fffffffu); }
typedef __attribute__((ext_vector_type(2))) int16_t i16x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
__device__ uint32_t order16(uint32_t w) {
  const i16x2 sign = __builtin_bit_cast(i16x2, w) >> 15;
  return w ^ (__builtin_bit_cast(uint32_t, sign) & 0x7fff7fffu);
}
__device__ uint32_t max16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
// Halves that are NaN become those of `none`.
__device__ uint32_t without_nan16(uint32_t w, uint32_t inf, uint32_t none) {
  const uint32_t nan = ((w & 0x7fff7fffu) + (0x7fffu - inf) * 0x10001u) & 0x80008000u, mask = (nan >> 15) * 0xffffu;
  return (w & ~mask) | (none & mask);
}
// The larger half of an ordered word, in the upper half.
__device__ int32_t upper(uint32_t w) { return max((int32_t)w, (int32_t)(w << 16)) & (int32_t)0xffff0000; }
__device__ uint32_t clamp16(uint32_t w, uint32_t low) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, w), __builtin_bit_cast(u16x2, low)));
}

template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xff800000u;
  static constexpr int32_t kInf = 0x7f800000;
  static __device__ float at(u32x4 v, int i) { return __uint_as_float(v[i]); }
  static __device__ int32_t largest(u32x4 v) {
    return max(max((int32_t)order_of(v.x, 0.f), (int32_t)order_of(v.y, 0.f)),
               max((int32_t)order_of(v.z, 0.f), (int32_t)order_of(v.w, 0.f)));
  }
  static __device__ float value(int32_t order) { return __uint_as_float(order_of((uint32_t)order, 0.f)); }
  static __device__ uint32_t low_of(float low) { return __float_as_uint(low); }
  static __device__ uint32_t clamp(uint32_t w, uint32_t low) { return min(w, low); }
  static __device__ uint32_t without_nan(uint32_t w) { return (w & 0x7fffffffu) > 0x7f800000u ? kNone : w; }
};
template <>
struct Piece<__bf16> {
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;
  static constexpr int32_t kInf = 0x7f800000;
  static __device__ float at(u32x4 v, int i) {
    const uint32_t w = v[i / 2];
    return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
  }
  static __device__ int32_t largest(u32x4 v) {
    return upper(max16(max16(order16(v.x), order16(v.y)), max16(order16(v.z), order16(v.w))));
  }
  static __device__ float value(int32_t order) { return __uint_as_float(order16((uint32_t)order & 0xffff0000u)); }
  static __device__ uint32_t low_of(float low) { return (__float_as_uint(low) >> 16) * 0x10001u; }
  static __device__ uint32_t clamp(uint32_t w, uint32_t low) { return clamp16(w, low); }
  static __device__ uint32_t without_nan(uint32_t w) { return without_nan16(w, 0x7f80u, kNone); }
};
template <>
struct Piece<_Float16> {
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static constexpr int32_t kInf = 0x7c000000;
  static __device__ float half(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
  static __device__ float at(u32x4 v, int i) { return half(v[i / 2] >> (i % 2 * 16)); }
  static __device__ int32_t largest(u32x4 v) {
    return upper(max16(max16(order16(v.x), order16(v.y)), max16(order16(v.z), order16(v.w))));
  }
  static __device__ float value(int32_t order) { return half(order16((uint32_t)order) >> 16); }
  static __device__ uint32_t low_of(float low) { return __builtin_bit_cast(uint16_t, (_Float16)low) * 0x10001u; }
  static __device__ uint32_t clamp(uint32_t w, uint32_t low) { return clamp16(w, low); }
  static __device__ uint32_t without_nan(uint32_t w) { return without_nan16(w, 0x7c00u, kNone); }
};

// A value in its type's order, as `largest` gives it.
template <typename T>
__device__ int32_t order_in(float y) {
  if constexpr (sizeof(T) == 4) return (int32_t)order_of(__float_as_uint(y), 0.f);
  else return (int32_t)(order16(__builtin_bit_cast(uint16_t, (T)y)) << 16);
}

// The exponentials of a wave's logits.
struct alignas(16) PowerTable {
  double at[256];
};
// 2^(i / 256), by its series, less i in the bits that `Powers` adds it to.
constexpr PowerTable power_table() {
  PowerTable t{};
  for (int i = 0; i < 256; ++i) {
    const double x = i * 0.0027076061740622863;
    double sum = 0.;
    for (int k = 24; k >= 1; --k) sum = (sum + 1.) * x / k;
    t.at[i] = sum + 1.;
  }
  return t;
}
__device__ const PowerTable kPowers = power_table();

struct Powers {
  static constexpr double kPerLn2 = 369.3299304675746;  // 256 / ln 2
  static constexpr float kHigh = (float)kPerLn2, kLow = (float)(kPerLn2 - (double)kHigh);
  static constexpr double kStep = 0.0027076061740622863;  // ln 2 / 256
  static constexpr float kOne = (float)kStep, kTwo = (float)(kStep * kStep / 2);
  // Sums with `round`, 1.5 2^23, are rounded to whole numbers, n in their low bits.  Those bits, 12 to the left, add n >> 8 to
  // a binary64's exponent and n & 255 below it, which the table's numbers have less; the others, of 1.5 2^23, leave the word.
  static __device__ double entry(int i) {
    const uint64_t b = __double_as_longlong(kPowers.at[i]);
    return __longlong_as_double(b - ((uint64_t)i << 44));
  }
  static constexpr float round = 12582912.f;
  const double* table;
  double sum = 0., more = 0.;
  struct Term {
    double two;  // the table's number
    uint32_t bits;
    float p;     // e^r - 1 with r in steps
  };

  __device__ Term ask(float y) const {
    const float t = fmaf(y, kHigh, round);
    const uint32_t bits = __float_as_uint(t);
    const double two = table[bits & 255];
    const float r = fmaf(y, kLow, fmaf(y, kHigh, -(t - round)));  // in [-1/2, 1/2]
    return Term{two, bits, fmaf(r, kTwo, kOne) * r};
  }
  __device__ void add(const Term& x) {
    const uint64_t e = __double_as_longlong(x.two);
    const double two = __longlong_as_double((uint64_t)((uint32_t)(e >> 32) + (x.bits << 12)) << 32 | (uint32_t)e);
    sum += two;
    more = fma(two, (double)x.p, more);
  }
};

// Keeps what follows from v from living in registers since it was last used.
__device__ void fresh(u32x4& v) { asm volatile("" : "+v"(v)); }

__device__ void fresh(double& v) { asm volatile("" : "+v"(v)); }

// Workgroup (segment, row); its waves share nothing before the end.  Bound by vector instructions: 512 rows of 131,072
// bfloat16 logits, a fifth of them of beams at their end, take 37 us, 107 MB at 2.9 TB/s, vector units busy 68% of the
// cycles: 1,363 instructions a wave of 4,096 logits, 12 for each exponential (with polynomials in binary64, 10 in all, 10%
// slower).  The loads alone take 19 us, with exponentials and maxima 27, thresholds and sums 2, pieces and ranks 8.  A chip holds
// most of these logits at once: with all of a wave's waited for before the first exponential, 47 us.
// Waves whose largest logit is finite and 500 or more in magnitude, or that have a NaN, read their logits once more, one at
// a time, and take exponentials in binary64.  512 rows with 9,999 of 10,000 logits at the type's lowest value take 121 us
// here and 30 in the second kernel, which gets a plateau of them; both kernels with -1e4 143 to 149 us, with half of the
// logits -1e4 50, with -inf 44; with one NaN a row 73, with 9,999 of 10,000 NaN 78.
// Logits are unpacked again at each use: kept unpacked they leave four waves on a SIMD, and it took 63 us.  With 16 pieces a
// thread 53 us, with four 44.
template <typename T, int NV>
__global__ __launch_bounds__(kThreads) void take_segments(ewsjf_beams b, const T* logits, const float* score_in,
                                                          const int32_t* done, Work w, int segments) {
  using P = Piece<T>;
  constexpr int N = P::N;
  __shared__ double power[256];
  __shared__ uint64_t found[kListed];
  __shared__ u32x4 pieces[kWaves][kWavePieces];  // that hold a wave's candidates,
  __shared__ int firsts[kWaves][kWavePieces];    // and their first tokens
  __shared__ Part parts[kWaves];
  __shared__ int bars[kWaves], plains[kWaves];
  __shared__ int count;
  const int row = blockIdx.y, seg = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // rows without candidates are not read
  if (!(score_in[row] > -INFINITY) || (done != nullptr && done[row] != 0)) return;
  const T* x = logits + row * b.row_stride;
  const int skew = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));  // elements of the first piece before the row
  power[threadIdx.x] = Powers::entry(threadIdx.x);  // waited for before the logits are on their way
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  const int piece0 = seg * kThreads * NV + wave * 64 * NV + lane;
  auto token_of = [&](int i) { return (piece0 + i * 64) * N - skew; };  // of piece i's first element
  // Loads without a branch, so that each is waited for alone: pieces that do not lie within the row take what lies here, and
  // are put together afterwards.
  auto within = [&](int first) { return first >= 0 && first + N <= b.vocab; };
  u32x4 v[NV];
  bool all = true;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int first = token_of(i);
    const bool in = within(first);
    v[i] = *(const __attribute__((address_space(1))) u32x4*)(in ? (uintptr_t)(x + first) : (uintptr_t)kPowers.at);
    all &= in;
  }
  if (!__all(all)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int first = token_of(i);
      if (within(first)) continue;
      constexpr int kBits = 8 * sizeof(T), kIn = 32 / kBits;
      auto word = [&](int k) {
        uint32_t word = P::kNone;
#pragma unroll
        for (int j = 0; j < kIn; ++j) {
          const int at = first + k * kIn + j;
          if (at >= 0 && at < b.vocab) {
            const uint32_t mask = kBits == 32 ? ~0u : 0xffffu << (j * 16);
            uint32_t bits;
            if constexpr (kBits == 32) bits = reinterpret_cast<const uint32_t*>(x)[at];
            else bits = reinterpret_cast<const uint16_t*>(x)[at];
            word = (word & ~mask) | bits << (j * (kBits % 32));
          }
        }
        return word;
      };
      v[i] = u32x4{word(0), word(1), word(2), word(3)};
    }
  }

  auto largest = [](u32x4 v) {
    const int32_t most = P::largest(v);
    return most == order_in<T>(-0.f) ? 0 : most;  // -0 is 0
  };
  // Piece after piece, as they come: its largest, the exponentials.
  int32_t most[NV], top = INT32_MIN;
  Powers powers{power};
  {
    const uint32_t low = P::low_of(-600.f);  // e^-600 of a row whose largest is above -500: nothing
    constexpr int kAhead = 4;                // numbers of the table that are on their way
    typename Powers::Term term[2][kAhead];
    u32x4 held;
#pragma unroll
    for (int k = 0; k <= NV * N / kAhead; ++k) {
      if (k < NV * N / kAhead) {
        const int i = k * kAhead / N;
        if (k * kAhead % N == 0) {
          fresh(v[i]);
          most[i] = largest(v[i]);
          top = max(top, most[i]);
          held = v[i];
          fresh(held);
          held = each_word(held, [&](uint32_t w) { return P::clamp(w, low); });
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) term[k % 2][j] = powers.ask(P::at(held, (k * kAhead + j) % N));
      }
      if (k > 0)
#pragma unroll
        for (int j = 0; j < kAhead; ++j) powers.add(term[(k - 1) % 2][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  fresh(powers.sum), fresh(powers.more);  // not put off until they are used
  const bool nan = __any(top > P::kInf);
  if (nan) {
    top = INT32_MIN;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = each_word(v[i], [](uint32_t w) { return P::without_nan(w); });
      most[i] = largest(v[i]);
      top = max(top, most[i]);
    }
  }
  // A value that at least `picks` of the wave's logits reach: over the lanes' largest, for many picks over the pieces'
  // largest or all logits.
  constexpr int kBits = 8 * sizeof(T);
  constexpr uint32_t kSign = 0x80000000u;
  uint32_t bar;
  if (b.picks <= 32) {
    const uint32_t key[1] = {(uint32_t)top ^ kSign};
    bar = wave_threshold<kBits>(key, b.picks);
  } else if (NV == 1) {
    uint32_t key[N];
#pragma unroll
    for (int j = 0; j < N; ++j) key[j] = order32(P::at(v[0], j));
    bar = wave_threshold<32>(key, b.picks);
    const float y = value32(bar);  // back to the type's own order
    bar = y >= -3.4028234e38f ? (uint32_t)order_in<T>(y) ^ kSign : 0;
  } else {
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) key[i] = (uint32_t)most[i] ^ kSign;
    bar = wave_threshold<kBits>(key, b.picks);
  }
  top = wave_max(top);
  const float ref = P::value(top);

  // The sum of the exponentials; of others than plain ones relative to e^ref.
  const bool plain = !nan && fabsf(ref) < 500.f;
  double sum = 0.;
  if (plain) {
    sum = powers.sum + powers.more;
  } else if (ref > -INFINITY) {  // a NaN, far logits, or entries of +inf, which share the row: read once more
#pragma unroll 1
    for (int i = 0; i < NV; ++i)
#pragma unroll 1
      for (int j = 0; j < N; ++j) {
        const int at = token_of(i) + j;
        const float y = at >= 0 && at < b.vocab ? (float)x[at] : -INFINITY;
        if (y > -INFINITY) sum += ref == INFINITY ? (y == INFINITY ? 1. : 0.) : exp((double)y - ref);
      }
  }
  sum = wave_sum(sum);

  // The pieces with candidates, none of -inf alone.
  auto own_of = [&](uint32_t bar) { return max((int32_t)(bar ^ kSign), order_in<T>(-INFINITY) + 1); };
  int32_t own = own_of(bar);
  int n = 0, reach = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) reach += __popcll(__ballot(most[i] >= own));
  const bool many = reach > kListed / kWaves / 8;  // lanes with more than one, or a plateau
  if (many && b.picks <= 32) {
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) key[i] = (uint32_t)most[i] ^ kSign;
    own = own_of(wave_threshold<kBits>(key, b.picks));
  }
  int ties = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    bool mine = most[i] >= own;
    if (many) {  // of equal pieces the first `picks`, which have the lowest tokens
      const uint64_t tied = __ballot(most[i] == own);
      mine = most[i] > own || (most[i] == own && ties + bits_below(tied) < b.picks);
      ties += __popcll(tied);
    }
    const uint64_t taken = __ballot(mine);
    if (taken) {
      const int at = n + bits_below(taken);
      if (mine) pieces[wave][at] = v[i], firsts[wave][at] = token_of(i);
      n += __popcll(taken);
    }
  }
  if (lane == 0) parts[wave] = Part{sum, ref}, plains[wave] = plain, bars[wave] = own;
  __syncthreads();

  // Together.
  const int64_t out = (int64_t)row * segments + seg;
  if (wave == 0) {
    const Part p = parts[lane % kWaves];
    double most = p.base;
    for (int d = 1; d < kWaves; d *= 2) most = fmax(most, __shfl_xor(most, d));
    const bool alike = __all(plains[lane % kWaves] || p.base == -INFINITY);
    // e^ref has the errors of the others: a row's only token has probability 1
    Powers largest{power};
    largest.add(largest.ask(alike ? (float)most : (float)p.base));
    const double unit = largest.sum + largest.more;
    double all = p.sum;
    if (!alike) {
      if (plains[lane % kWaves]) all /= unit;
      if (p.base != most) all = p.base > -INFINITY ? all * exp(p.base - most) : 0.;
    }
    for (int d = 1; d < kWaves; d *= 2) all += __shfl_xor(all, d);
    if (lane == 0) w.part[out] = Part{alike && most > -INFINITY ? all / unit : all, most};
  }
  int32_t least = bars[0];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) least = max(least, bars[i]);
  // none of -inf: numbers below are no values
  const float lowest = -3.4028234e38f, bound = least > order_in<T>(-INFINITY) ? max(P::value(least), lowest) : lowest;
  ties = 0;
  for (int k0 = 0; k0 < n * N; k0 += 64) {  // in the tokens' order
    const int k = k0 + lane < n * N ? k0 + lane : 0;
    const uint32_t word = pieces[wave][k / N][k % N * 4 / N];
    const float y = P::at(u32x4{N == 4 ? word : word >> (k % 2 * 16), 0, 0, 0}, 0);
    const uint64_t tied = __ballot(k0 + lane < n * N && y == bound);
    if (k0 + lane < n * N && (y > bound || (y == bound && ties + bits_below(tied) < b.picks)))
      found[atomicAdd(&count, 1)] = (uint64_t)order32(y) << 32 | ~(uint32_t)(firsts[wave][k / N] + k % N);
    ties += __popcll(tied);
  }
  __syncthreads();
  const int total = count;
  uint64_t* best = w.best + out * b.picks;
  for (int k = threadIdx.x; k < total; k += kThreads) {  // each candidate ranked against the others
    const uint64_t key = found[k];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < total; ++j) rank += found[j] > key;
    if (rank < b.picks) best[rank] = key;
  }
  for (int k = total + threadIdx.x; k < b.picks; k += kThreads) best[k] = 0;
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

// A workgroup a group.  Bound by latency: 8.5 us for 64 groups of 1,024 candidates, 7 us for one, half of them the loads, the
// logarithms and the threshold that come one after the other; 14 us for one group of 20,000 candidates, 40 with all of them
// looked at and sorted where more than 512 reach the first threshold.
__global__ __launch_bounds__(kJoinThreads) void join_groups(ewsjf_beams b, const float* score_in, const int32_t* done,
                                                            Work w, int segments, int32_t* parent, int32_t* token,
                                                            float* score) {
  constexpr int kWaves = kJoinThreads / 64, kHeld = 2;  // candidates that a thread holds
  __shared__ Entry found[kMostFound];
  __shared__ double base[EWSJF_MAX_BEAMS];  // score of a logit of 0
  __shared__ int kind[EWSJF_MAX_BEAMS];     // 0: no candidates, 1: logits, 2: entries of +inf alone, 3: at its end
  __shared__ uint32_t least[kWaves], share[kWaves];
  __shared__ Entry tops[kWaves];
  __shared__ int count;
  const int group = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int each = segments * b.picks, lists = b.beams * segments, all = lists * b.picks;
  const uint64_t* best = w.best + (int64_t)group * all;
  // Of few candidates all are looked at.  Else of each list, which is in order, the first `heads`, for a threshold, and
  // then as many as reach it, by a team of threads a list.
  const bool few = all <= kHeld * kJoinThreads;
  const int heads = few ? b.picks : lists < kHeld * kJoinThreads ? kHeld * kJoinThreads / lists : 1;
  auto sample = [&](int i) { return few ? i : i / heads * b.picks + i % heads; };
  const int samples = lists * heads;
  uint64_t key[kHeld];  // asked for before anything waits
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = threadIdx.x + i * kJoinThreads;
    key[i] = c < samples ? best[sample(c)] : 0;
  }
  if (threadIdx.x == 0) count = 0;
  for (int r = wave; r < b.beams; r += kWaves) {
    const int row = group * b.beams + r;
    const float s = score_in[row];
    if (!(s > -INFINITY) || (done != nullptr && done[row] != 0)) {
      if (lane == 0) base[r] = s, kind[r] = s > -INFINITY ? 3 : 0;
      continue;
    }
    const Part* part = w.part + (int64_t)row * segments;
    Part p{0., -INFINITY};
    if (lane < segments) p = part[lane];
    double top = p.base;
    for (int i = lane + 64; i < segments; i += 64) top = fmax(top, part[i].base);
    for (int d = 1; d < 64 && d < segments; d *= 2) top = fmax(top, __shfl_xor(top, d));
    double sum = 0.;
    for (int i = lane;;) {
      if (p.base == top) sum += p.sum;
      else if (p.base > -INFINITY) sum += p.sum * exp(p.base - top);
      if ((i += 64) >= segments) break;
      p = part[i];
    }
    for (int d = 1; d < 64 && d < segments; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) {
      base[r] = top == INFINITY ? s - log(sum) : s - (top + log(sum));
      kind[r] = top == INFINITY ? 2 : top > -INFINITY ? 1 : 0;
    }
  }
  __syncthreads();

  // Candidate c of the group's; place 0: none.
  auto entry_of = [&](int c, uint64_t key) {
    const int r = c / each, k = kind[r];
    Entry e{0, 0};
    const uint64_t before = (uint64_t)((1 << kRowBits) - 1 - r) << (32 + kVocabBits);
    const uint32_t last = (1u << kVocabBits) - 1;
    if (k == 3) {
      if (c == r * each) e = Entry{order64(base[r]), before | 1ull << (31 + kVocabBits) | (last - b.end)};
    } else if (k != 0) {
      const uint32_t o = (uint32_t)(key >> 32), v = ~(uint32_t)key;
      const float x = value32(o);
      if (key != 0 && (k == 1 || x == INFINITY))
        e = Entry{order64(k == 1 ? base[r] + x : base[r]), before | (uint64_t)o << kVocabBits | (last - v)};
    }
    return e;
  };
  auto none = [](const Entry& e) { return e.place == 0; };
  // A value that at least `picks` of the wave's samples reach, in a score's upper half: over the lanes' two highest.
  uint32_t high[2] = {0, 0};
  auto look = [&](const Entry& e) {
    const uint32_t o = (uint32_t)(e.score >> 32);
    if (o > high[0]) high[1] = high[0], high[0] = o;
    else if (o > high[1]) high[1] = o;
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = threadIdx.x + i * kJoinThreads;
    if (c < samples) look(entry_of(sample(c), key[i]));
  }
  for (int c = threadIdx.x + kHeld * kJoinThreads; c < samples; c += kJoinThreads) look(entry_of(sample(c), best[sample(c)]));
  uint32_t bar = wave_threshold<22>(high, b.picks);  // cut to 22 bits fewer steps, and a few candidates more
  if (lane == 0) least[wave] = bar;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) bar = least[i] > bar ? least[i] : bar;
  auto keep = [&](const Entry& e) {
    if (none(e) || (uint32_t)(e.score >> 32) < bar) return false;
    const int at = atomicAdd(&count, 1);
    if (at < kMostFound) found[at] = e;
    return true;
  };
  int n;
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    if (few) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int c = threadIdx.x + i * kJoinThreads;
        if (c < all) keep(entry_of(c, key[i]));
      }
    } else {
      constexpr int kBatch = 4;  // loads on their way
      const int team = lists <= kJoinThreads / 16 ? 16 : lists <= kJoinThreads / 8 ? 8 : lists <= kJoinThreads / 4 ? 4 : 1;
      for (int l = threadIdx.x / team; l < lists; l += kJoinThreads / team) {
        bool more = true;
        for (int k0 = threadIdx.x % team; more && k0 < b.picks; k0 += kBatch * team) {
          uint64_t next[kBatch];
#pragma unroll
          for (int i = 0; i < kBatch; ++i) next[i] = best[l * b.picks + (k0 + i * team < b.picks ? k0 + i * team : 0)];
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const int k = k0 + i * team;
            more = more && k < b.picks && keep(entry_of(l * b.picks + k, next[i]));
          }
        }
      }
    }
    __syncthreads();
    n = count;
    if (n <= kMostFound / 4 || pass == 3) break;
    // More than are ranked quickly: a higher threshold, that `picks` of one wave's found reach, or a share of them of
    // every wave's.
    high[0] = high[1] = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = threadIdx.x + i * kJoinThreads;
      if (at < n && at < kMostFound) look(found[at]);
    }
    uint32_t next = wave_threshold<32>(high, b.picks);
    uint32_t common = wave_threshold<32>(high, (b.picks + kWaves - 1) / kWaves);
    if (lane == 0) least[wave] = next, share[wave] = common;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      next = least[i] > next ? least[i] : next;
      common = share[i] < common ? share[i] : common;
    }
    next = common > next ? common : next;
    if (next <= bar) break;
    bar = next;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
  }
  auto write = [&](int rank, const Entry& e) {
    const int64_t at = (int64_t)group * b.picks + rank;
    const bool there = !none(e);
    const int r = (1 << kRowBits) - 1 - (int)(e.place >> (32 + kVocabBits));
    parent[at] = there ? group * b.beams + r : -1;
    token[at] = there ? (1 << kVocabBits) - 1 - (int)(e.place & ((1u << kVocabBits) - 1)) : -1;
    score[at] = there ? (float)value64(e.score) : -INFINITY;
  };
  if (n <= kMostFound / 4) {  // each candidate ranked against the others
    if ((int)threadIdx.x < n) {
      const Entry mine = found[threadIdx.x];
      int rank = 0;
#pragma unroll 8
      for (int i = 0; i < n; ++i) rank += above(found[i], mine);
      if (rank < b.picks) write(rank, mine);
    }
  } else if (n <= kMostFound) {
    sort_entries<kJoinThreads>(found, n, Entry{0, 0}, above);
    if ((int)threadIdx.x < b.picks) write(threadIdx.x, found[threadIdx.x]);
  } else {  // a plateau of equal scores: the lists merged, a pick at a time
    Entry mine;  // the best of this thread's lists that is not picked yet
    auto renew = [&](const Entry& last) {
      mine = Entry{0, 0};
      for (int l = threadIdx.x; l < lists; l += kJoinThreads) {
        int at = 0;
        for (int end = b.picks; at < end;) {
          const int mid = (at + end) / 2, c = l * b.picks + mid;
          if (above(last, entry_of(c, best[c]))) end = mid;
          else at = mid + 1;
        }
        if (at == b.picks) continue;
        const int c = l * b.picks + at;
        const Entry e = entry_of(c, best[c]);
        if (above(e, mine)) mine = e;
      }
    };
    renew(Entry{~0ull, ~0ull});
#pragma unroll 1
    for (int k = 0; k < b.picks; ++k) {
      Entry top = mine;
#pragma unroll
      for (int d = 32; d; d >>= 1) {
        const Entry o{(uint64_t)__shfl_xor(top.score, d), (uint64_t)__shfl_xor(top.place, d)};
        if (above(o, top)) top = o;
      }
      __syncthreads();
      if (lane == 0) tops[wave] = top;
      __syncthreads();
      for (int i = 0; i < kWaves; ++i)
        if (above(tops[i], top)) top = tops[i];
      if (threadIdx.x == 0) write(k, top);
      if (!none(top) && mine.place == top.place) renew(top);
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

size_t beam_ws_bytes(const ewsjf_beams& b) { return work_of(b, sizes_of(b, -1), nullptr).bytes; }

hipError_t launch_beam_select(const ewsjf_beams& b, const void* logits, const float* score_in, const int32_t* done,
                              int32_t* parent, int32_t* token, float* score, void* ws, hipStream_t stream) {
  if (b.groups == 0) return hipSuccess;
  const int size = b.dtype == EWSJF_F32 ? 4 : 2;
  const int skew = (b.row_stride * size) % 16 || reinterpret_cast<uintptr_t>(logits) % 16 ? -1 : 0;
  const Sizes s = sizes_of(b, skew);
  const Work w = work_of(b, s, ws);
  if (b.dtype == EWSJF_F32) launch_segments<float>(b, logits, score_in, done, w, s, stream);
  else if (b.dtype == EWSJF_BF16) launch_segments<__bf16>(b, logits, score_in, done, w, s, stream);
  else launch_segments<_Float16>(b, logits, score_in, done, w, s, stream);
  join_groups<<<b.groups, kJoinThreads, 0, stream>>>(b, score_in, done, w, s.segments, parent, token, score);
  return hipGetLastError();
}

}  // namespace ewsjf
