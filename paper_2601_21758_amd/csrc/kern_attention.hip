// Attention over the paged key/value cache.
//
// A unit of work is one key head of a row tile: up to `rows` rows, a row being
// a query token and one of the G = q_heads / kv_heads query heads that read
// that key head, so the keys are read once for all of them.  The unit's keys
// are cut into tiles.  All units' tiles lie on one line (key head, then row
// tile, then key tile), and the line is cut into equal shares, one a worker: a
// share may begin or end inside a unit, whose parts are joined afterwards
// (running maximum, sum and output of a softmax join exactly, in any cut).
// So one sequence of many tokens, many sequences of few, and anything ragged
// between them all fill the chip evenly, and a worker writes at most two
// partial results.
//
// A shared prefix is a phase of its own: the group's queries of all members
// are the rows, the shared tokens the keys.
//
// Scores are computed transposed, S^T = K Q^T, with 32x32x16 matrix
// instructions: a lane then holds scores of one row (its column), so the
// softmax's maximum and sum are taken in the lane and joined once with the lane
// 32 away, and the weights P^T are in the registers as the second product's
// operand needs them, O^T = V^T P^T, when the keys are taken in the order
// 4h, .., 4h + 3, 8 + 4h, .. in which the first product leaves them (h = lane /
// 32).  V^T is read from LDS with the transposing read.
//
// With `width` the row's query heads, a unit of R rows and K keys reads R D +
// 2 K D values once and computes 4 R K D operations: R operations a byte of
// keys.  Up to 32 rows (decoding) memory is the limit, from about 200 rows on
// (prefill, many requests behind one prefix) the matrix units are; hence two
// kernels.  What they reach on the card, whose large copies run at 4.8 TB/s
// (read and written) and whose large 16-bit products at 1270 TFLOP/s:
//   one prompt of 16,384 tokens, 40 heads of 128, window 4096: 1.5 to 1.6 ms,
//   770 to 800 TFLOP/s; 256 single tokens of 32 query and 8 key heads of 128 over windows
//   of 4096: 194 us, 5.0 TB/s.
#include <hip/hip_runtime.h>

#include "ewsjf_cache.h"

namespace ewsjf {
namespace {

constexpr int kRowTile = 32;     // rows of a unit of the wave kernel
constexpr int kRowKeys = 32;     // its key tile
// Key tile of the workgroup kernel with four or eight waves of 32 rows: two
// tiles fill the LDS that a workgroup can have with all waves resident.
__host__ __device__ constexpr int block_keys(int waves) { return waves == 8 ? 128 : 64; }
constexpr int kWaves = 4;        // waves of a workgroup of the wave kernel
constexpr int kCUs = 256;
constexpr int64_t kMostJoins = 1 << 24;  // waves of a grid's row: a launch has below 2^32 threads in one
constexpr int kWholeKeys = 2048;   // of a unit that one workgroup takes whole
// Position of a shared phase's first query, past every shared key; its other tokens' do not pass 32 bits.
constexpr int kPast = 0x7fffffff - (1 << 24);
constexpr float kFloor = -3e38f;   // running maximum of a row that has seen no key
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// A row tile.  Row r is query token q0 + (row0 + r) / G and query head (row0 +
// r) % G of the key head's; it sees keys up to pos0 + (row0 + r) / G.
struct Entry {
  int32_t slot;       // row of the table, -1: no keys
  int32_t q0, row0, rows, pos0;
  int32_t lo, end;    // keys of the main run
  int32_t sink;       // keys [0, sink) come before it
  int32_t prefix;     // first row tile of the group's phase, -1: no shared keys
  int32_t prefix_row; // row of this tile's row 0 in the group
  int32_t tiles;
  int32_t pad;
};

// A worker's first tile: its unit's place in the line, the unit, the tile.
struct Start {
  int32_t place, entry, head, tile;
};

// The unit at a place of a line in columns.  Otherwise the line goes by heads:
// the row tiles of a key head, then the next head's.  In columns, each XCD's
// eighth of that list is dealt out to `columns` workers in turn, a worker's units
// following one another on the line; so at any time the workers of an XCD have
// neighbouring row tiles of one head, which read much the same keys (24 prompts
// over windows of 1024: 267 us, by heads 379).
__device__ int64_t unit_at(int64_t place, int64_t units, int columns) {
  int64_t base = 0, size = units;
  for (int x = 7; x >= 0; --x)
    if (place >= units * x / 8) {
      base = units * x / 8;
      size = units * (x + 1) / 8 - base;
      break;
    }
  int64_t k = place - base;
  const int64_t rows = size / columns, longer = size % columns;  // the first `longer` columns have one row more
  int64_t col, row;
  if (k < longer * (rows + 1)) {
    col = k / (rows + 1), row = k % (rows + 1);
  } else {
    k -= longer * (rows + 1);
    col = longer + k / rows, row = k % rows;
  }
  return base + row * columns + col;
}

// One phase of a plan.
struct Phase {
  int64_t total;    // key tiles of one key head
  int64_t share;    // tiles per worker
  int32_t entries;
  int32_t workers;
  int32_t columns;  // of unit_at
  int32_t pad;
};

struct Plan {
  Phase* phase;      // [2]: shared prefixes, the sequences' own keys
  Start* start[2];   // [workers]
  Entry* entry[2];
  int64_t* cum[2];   // tiles of one key head before a row tile
  int64_t* line;     // tiles before a place of the line in columns,
  int32_t* order;    // and its unit
  size_t bytes;
};

struct Shape {
  bool groups;  // a shared prefix is a phase of its own
  bool whole;   // a worker a unit: nothing is cut, nothing joined
  bool both;    // both phases in one kernel
  int G;
  int waves[2];  // of a workgroup that shares a unit's keys; 0: the wave kernel
  int rows[2], keys[2], workers[2], blocks[2];
  int64_t entries[2];  // most row tiles
  int kv_heads;
  int columns;         // phase 1's line in columns of this many a XCD; 0: by heads
};

Shape shape_of(const ewsjf_cache& c, const ewsjf_batch& b) {
  Shape s;
  s.G = b.q_heads / c.kv_heads;
  const int64_t most_keys = (int64_t)c.width * c.page_size;  // of a sequence: lengths are on the device
  // Sharing pays when the keys and values that each sequence would read for itself (much of it from caches) take longer
  // than the phase and the join.  32 query and 8 key heads of 128, shared against not: 16 sequences behind 1024 tokens
  // (66 MiB) 20 us against 17, 64 behind 1024 (264 MiB) 25 against 33, 16 behind 4096 (258 MiB) 26 against 34.  With at
  // most 32 rows a group, in two kernels: 4 behind 4096 (64 MiB) 40 against 31, 4 behind 16,000 (250 MiB) 64 against 65;
  // 8 of 40 heads behind 1024 (165 MiB) 34 against 22.
  const int64_t rows = b.n_groups > 0 ? b.total_q * s.G / b.n_groups : 0;
  const int64_t bytes = 4 * most_keys * b.n_seqs * c.kv_heads * c.head_dim;
  s.groups = rows > 0 && bytes > (rows > kRowTile ? (int64_t)128 << 20 : (int64_t)256 << 20);
  // rows that read the same keys: of a group on average, of a sequence
  const int64_t most[2] = {s.groups ? rows : 0, (int64_t)b.max_q * s.G};
  // One kernel for both phases, half of each CU to either, up to 100 GFLOP against shared keys: 64 sequences behind 2048
  // tokens took 59 us, as two kernels 71; 512 behind 4096, 109 against 143, behind 8192 (69 GFLOP) 158 against 174.
  // Beyond, a kernel with all of each CU and tiles of 256 rows makes up for the second one: 512 behind 16,123
  // (135 GFLOP) took 263 us, in one kernel 270.
  const double flops = 4. * b.total_q * b.q_heads * c.head_dim * most_keys;
  s.both = most[0] > kRowTile && most[1] <= kRowTile && flops < 100e9;
  for (int p = 0; p < 2; ++p) {
    s.waves[p] = most[p] <= kRowTile ? 0 : most[p] <= 128 || s.both ? 4 : 8;
    s.rows[p] = s.waves[p] ? 32 * s.waves[p] : kRowTile;
    s.keys[p] = s.waves[p] ? block_keys(s.waves[p]) : kRowKeys;
    // as many as fit the chip at once: eight waves of 256 registers a CU
    s.blocks[p] = s.waves[p] == 8 || s.both ? kCUs : 2 * kCUs;
    s.workers[p] = s.waves[p] ? s.blocks[p] : s.blocks[p] * kWaves;
    s.entries[p] = b.total_q * s.G / s.rows[p] + (p ? b.n_seqs : b.n_groups);
  }
  if (!s.groups) s.entries[0] = 0;
  s.kv_heads = c.kv_heads;
  // One token a sequence and few keys: a workgroup takes a unit sooner than a second kernel joins its parts.  32 query and
  // 8 key heads of 128, whole against cut: 16 sequences of 1024 keys 16 us against 24, 256 of 1024 189 against 187, 8 of
  // 2048 24 against 29, 128 of 2048 190 against 193, but 32 of 2048 56 against 50; 16 of 4096 45 against 52, 64 of 4096
  // 205 against 194, 128 of 4096 374 against 371, 256 of 4096 729 against 715.  With one token, no row sees less of a unit
  // than another, so no row is done again either.
  const int64_t keys = b.window > 0 && (int64_t)b.window + b.sinks < most_keys ? (int64_t)b.window + b.sinks : most_keys;
  const int64_t units = s.entries[1] * c.kv_heads;
  s.whole = !s.groups && s.waves[1] == 0 && b.max_q == 1 && keys <= kWholeKeys;
  if (s.whole) s.workers[1] = s.blocks[1] = (int)((units + 7) / 8 * 8);
  // many row tiles of long runs, and nothing to join them with
  s.columns = s.waves[1] && !s.groups ? s.workers[1] / 8 : 0;
  return s;
}

struct Carve {
  char* base;
  size_t at = 0;
  template <typename T>
  T* take(size_t n) {
    T* r = reinterpret_cast<T*>(base + at);
    at += (n * sizeof(T) + 255) & ~size_t(255);
    return r;
  }
};

Plan plan_of(const Shape& s, void* base) {
  Carve at{static_cast<char*>(base)};
  Plan p;
  p.phase = at.take<Phase>(2);
  for (int i = 0; i < 2; ++i) {
    p.start[i] = at.take<Start>(s.workers[i]);
    p.entry[i] = at.take<Entry>(s.entries[i]);
    p.cum[i] = at.take<int64_t>(s.entries[i] + 1);
  }
  p.line = at.take<int64_t>(s.columns ? s.entries[1] * s.kv_heads + 1 : 0);
  p.order = at.take<int32_t>(s.columns ? s.entries[1] * s.kv_heads + 1 : 0);
  p.bytes = at.at;
  return p;
}

// Partial results: outputs in binary32 before the division, and (maximum in
// the exponent's units, sum) of each row.  Parts of a unit that is cut go to
// the worker's slot 0 (its first unit) or 1 (its last), [worker][2][rows]; a
// whole unit's rows that still have to be joined with the other phase go to
// `whole`, [total_q][q_heads].
struct Parts {
  float* o;
  float2* ml;
  float* whole_o;
  float2* whole_ml;
};

struct Work {
  Parts part[2];
  float* lse;       // [total_q][q_heads], where the caller gives none
  int32_t* odd[2];  // of each wave: it met values that are not finite where some row does not look
  size_t bytes;
};

Work work_of(const ewsjf_cache& c, const ewsjf_batch& b, const Shape& s, void* base) {
  Carve at{static_cast<char*>(base)};
  Work w;
  for (int i = 0; i < 2; ++i) {
    const bool used = i == 1 ? !s.whole : s.groups;
    const size_t rows = used ? (size_t)s.workers[i] * 2 * s.rows[i] : 0;
    const size_t whole = s.groups ? (size_t)b.total_q * b.q_heads : 0;
    w.part[i].o = at.take<float>(rows * c.head_dim);
    w.part[i].ml = at.take<float2>(rows);
    w.part[i].whole_o = at.take<float>(whole * c.head_dim);
    w.part[i].whole_ml = at.take<float2>(whole);
    w.odd[i] = at.take<int32_t>((size_t)s.workers[i] * (s.waves[i] ? s.waves[i] : 1));
  }
  w.lse = at.take<float>((size_t)b.total_q * b.q_heads);
  w.bytes = at.at;
  return w;
}

// ---------------------------------------------------------------------------
// The plan
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;

__device__ int64_t scan(int64_t v, int64_t* sums, int64_t& total) {  // exclusive over the workgroup
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t inc = v;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  int64_t base = 0, all = 0;
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    if (i < wave) base += sums[i];
    all += sums[i];
  }
  total = all;
  return base + inc - v;
}

// The last i in [0, n) with key[i] <= v (0 if none).
template <typename T>
__device__ int last_at_most(const T* key, int n, int64_t v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (key[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Starts brought into [0, most], and into order: each at least as large as those
// before it.  So the row tiles of a batch are never more than its sizes allow.
__device__ void climb(const int32_t* from, int n, int most, int* to, int64_t* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t run = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int64_t v = i < n ? from[i] : 0;
    v = v < 0 ? 0 : v > most ? most : v;
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(v, d);
      if (lane >= d && o > v) v = o;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    int64_t all = run;
    for (int k = 0; k < kPlanThreads / 64; ++k) {
      if (k == wave) {
        if (all > v) v = all;
        if (i < n) to[i] = (int)v;
      }
      if (sums[k] > all) all = sums[k];
    }
    run = all;
  }
}

struct PlanArgs {
  const int32_t *slot, *q_start, *group_start, *shared;
  int rows[2], keys[2], workers[2], G, columns;
  bool whole;
};

// One workgroup, latency-bound: prefix sums over the row tiles and a search a
// worker.  14 us for 4 sequences, 27 us for 512 behind a prefix and 25 us for
// the 2560 units of one long prompt, as long as the smallest attention or
// longer; once a step, whatever the layers.
// Everything read from the caller's arrays is bounded here, so the other
// kernels follow the plan without checks of their own.
__global__ __launch_bounds__(kPlanThreads) void make_plan(ewsjf_cache c, ewsjf_batch b, PlanArgs a, Plan plan) {
  constexpr int kMost = EWSJF_MAX_CACHE_BATCH;
  __shared__ int64_t sums[kPlanThreads / 64];
  __shared__ int first[kMost + 1];  // first row tile of a sequence or group
  __shared__ int common[kMost];     // a group's shared tokens that count
  __shared__ int lead[kMost];       // its first member with queries and a slot
  __shared__ int members[kMost];
  __shared__ int q_from[kMost + 1];
  __shared__ int g_from[kMost + 1];
  const int n = b.n_seqs, groups = b.n_groups;
  const int64_t room = (int64_t)c.width * c.page_size;
  climb(a.q_start, n + 1, (int)b.total_q, q_from, sums);
  if (groups > 0) climb(a.group_start, groups + 1, n, g_from, sums);
  __syncthreads();
  auto q_at = [&](int i) -> int64_t { return q_from[i]; };
  auto queries = [&](int i) { return q_at(i + 1) - q_at(i); };
  auto has_slot = [&](int i) { return a.slot[i] >= 0 && a.slot[i] < c.n_slots; };
  auto tokens = [&](int i) -> int64_t {
    if (!has_slot(i)) return 0;
    const int64_t v = c.length[a.slot[i]];
    return v < 0 ? 0 : v > room ? room : v;
  };
  auto group_at = [&](int g) { return g_from[g]; };
  auto group_of = [&](int i) {  // -1: none
    if (groups == 0) return -1;
    const int g = last_at_most(g_from, groups, i);
    return group_at(g) <= i && i < group_at(g + 1) ? g : -1;
  };
  for (int g = threadIdx.x; g < groups; g += kPlanThreads) {
    const int v = a.shared[g];
    common[g] = v < 0 ? 0 : v < kPast ? v : kPast;
    lead[g] = n;
    members[g] = 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int g = group_of(i);
    if (g < 0 || queries(i) == 0 || !has_slot(i)) continue;
    const int64_t before = tokens(i) - queries(i);
    atomicMin(&common[g], (int)(before < 0 ? 0 : before));
    atomicMin(&lead[g], i);
    atomicAdd(&members[g], 1);
  }
  __syncthreads();
  for (int g = threadIdx.x; g < groups; g += kPlanThreads)
    common[g] = members[g] < 2 ? 0 : common[g] & ~15;  // nobody to share with; tiles begin at multiples of 16
  __syncthreads();

  for (int ph = 0; ph < 2; ++ph) {
    const int R = a.rows[ph], TK = a.keys[ph], owners = ph ? n : groups;
    Entry* entry = plan.entry[ph];
    // row tiles of each sequence, or of each group with shared tokens
    auto rows_of = [&](int i) -> int64_t {
      if (ph) return queries(i) * a.G;
      if (common[i] == 0) return 0;
      return (q_at(group_at(i + 1)) - q_at(group_at(i))) * a.G;
    };
    int64_t run = 0;
    // a group's first row tile is kept for phase 1, in `members`
    for (int i0 = 0; i0 < owners; i0 += kPlanThreads) {
      const int i = i0 + threadIdx.x;
      const int64_t tiles = i < owners ? (rows_of(i) + R - 1) / R : 0;
      int64_t total;
      const int64_t before = scan(tiles, sums, total);
      if (i < owners) first[i] = (int)(run + before);
      if (i < owners && ph == 0) members[i] = (int)(run + before);
      run += total;
    }
    const int E = (int)run;
    __syncthreads();
    int64_t line = 0;
    for (int e0 = 0; e0 < E; e0 += kPlanThreads) {
      const int e = e0 + threadIdx.x;
      Entry x = {};
      if (e < E) {
        // several owners without row tiles may begin where one with them does: the last one has them
        const int i = last_at_most(first, owners, e);
        const int64_t rows = rows_of(i);
        x.row0 = (e - first[i]) * R;
        x.rows = (int)(rows - x.row0 < R ? rows - x.row0 : R);
        if (ph == 0) {
          x.slot = a.slot[lead[i]];
          x.q0 = (int)q_at(group_at(i));
          x.pos0 = kPast;
          x.end = common[i];
          x.prefix = -1;
        } else {
          const int g = group_of(i);
          const int shared = g < 0 || !has_slot(i) ? 0 : common[g];
          const int64_t len = tokens(i);
          x.slot = has_slot(i) ? a.slot[i] : -1;
          x.q0 = (int)q_at(i);
          x.pos0 = (int)(len - queries(i));
          const int p0 = x.pos0 + x.row0 / a.G, p1 = x.pos0 + (x.row0 + x.rows - 1) / a.G;
          x.end = p1 + 1 > 0 ? p1 + 1 : 0;
          x.lo = shared;
          if (b.window > 0) {
            const int64_t w = (int64_t)p0 - b.window + 1;
            x.lo = w > 0 ? (int)w & ~15 : 0;
            x.sink = b.sinks < x.end ? b.sinks : x.end;
            if (x.lo <= x.sink) x.lo = x.sink = 0;  // one run of keys
          }
          x.prefix = shared > 0 ? members[g] : -1;
          x.prefix_row = shared > 0 ? (int)((q_at(i) - q_at(group_at(g))) * a.G + x.row0) : 0;
        }
        const int span = x.end > x.lo ? x.end - x.lo : 0;
        x.tiles = (((x.sink + 15) & ~15) + span + TK - 1) / TK;
        if (x.tiles == 0) x.tiles = 1;  // a tile without keys, for the rows' zeros
        entry[e] = x;
      }
      int64_t total;
      const int64_t before = scan(x.tiles, sums, total);
      if (e < E) plan.cum[ph][e] = line + before;
      line += total;
    }
    const int64_t all = line * c.kv_heads;
    // Even shares, but where a unit has many workers, its s tiles a share against T / s parts to join: one row tile of
    // 4096 keys a head took 59 us in shares of a tile (128 parts), 40 in shares of four.  0: a worker a unit.
    int64_t share = all > 0 ? (all + a.workers[ph] - 1) / a.workers[ph] : 1;
    while (8 * share * share * E < line) ++share;
    if (ph && a.whole) share = 0;
    const int active = share ? (int)((all + share - 1) / share) : E * c.kv_heads;
    if (threadIdx.x == 0) {
      plan.cum[ph][E] = line;
      plan.phase[ph] = Phase{line, share, E, active, ph ? a.columns : 0, 0};
    }
    __syncthreads();  // entries and sums are read back by other threads
    const int64_t units = (int64_t)E * c.kv_heads;
    if (ph && a.columns) {
      int64_t before = 0;
      for (int64_t k0 = 0; k0 < units; k0 += kPlanThreads) {
        const int64_t k = k0 + threadIdx.x;
        const int64_t unit = k < units ? unit_at(k, units, a.columns) : 0;
        const int tiles = k < units ? entry[unit % E].tiles : 0;
        int64_t total;
        const int64_t mine = scan(tiles, sums, total);
        if (k < units) {
          plan.line[k] = before + mine;
          plan.order[k] = (int)unit;
        }
        before += total;
      }
      __syncthreads();
    }
    for (int w = threadIdx.x; w < active; w += kPlanThreads) {
      const int64_t at = w * share;
      int64_t place, rest;
      if (share == 0) {
        place = w, rest = 0;
      } else if (ph && a.columns) {
        place = last_at_most(plan.line, (int)units, at);
        rest = at - plan.line[place];
      } else {
        const int64_t head = at / line;
        const int e = last_at_most(plan.cum[ph], E, at % line);
        place = head * E + e;
        rest = at % line - plan.cum[ph][e];
      }
      const int64_t unit = ph && a.columns ? plan.order[place] : place;
      plan.start[ph][w] = Start{(int)place, (int)(unit % E), (int)(unit / E), (int)rest};
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) short short4v;
typedef __attribute__((ext_vector_type(16))) float float16v;
template <int N>
struct Const {
  static constexpr int value = N;
};
template <typename T>
using vec8 = T __attribute__((ext_vector_type(8)));

__device__ float16v mfma(vec8<__bf16> a, vec8<__bf16> b, float16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ float16v mfma(vec8<_Float16> a, vec8<_Float16> b, float16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// The value of the lane 32 away joined with this lane's.
__device__ float pair_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ float pair_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Places in LDS of a tile's keys (16-byte chunks) and values (64-byte blocks),
// row by row, moved about within 256 bytes so that the 16 rows that one read of
// the keys touches, and the four rows of a transposing read of the values, lie
// in different banks.  Both moves are an exclusive or of the row with the
// chunk, so a lane's places differ from its first one by a constant that the
// loops apply (key_step, value_step).
template <int D>
__device__ int key_place(int key, int chunk) {
  return D == 128 ? key * 256 + ((chunk ^ (key & 15)) << 4) : key * 128 + ((chunk ^ ((key >> 1) & 7)) << 4);
}
template <int D>
__device__ int value_place(int key, int byte) {
  const int block = byte >> 6, in = byte & 63;
  return D == 128 ? key * 256 + ((block ^ (key & 3)) << 6) + in : key * 128 + ((block ^ ((key >> 1) & 1)) << 6) + in;
}

// Keeps what follows from x out of registers that live across the loop.
__device__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

__device__ uint32_t not_finite(uint32_t x, __bf16) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ uint32_t not_finite(uint32_t x, _Float16) { return ((x & 0x7c007c00u) + 0x04000400u) & 0x80008000u; }

// Global memory: a pointer read from memory does not say so by itself, and a
// load that may be from LDS waits for LDS too.
template <typename T>
using Global = __attribute__((address_space(1))) T*;
template <typename T>
__device__ Global<T> global(T* p) {
  return (Global<T>)p;
}

// What no kernel of the call writes: read by scalar loads where the index is the
// wave's.
template <typename T>
__device__ T constant(const T* p) {
  union {
    T all;
    uint32_t part[sizeof(T) / 4];
  } r;
  const auto* from = (const __attribute__((address_space(4))) uint32_t*)p;
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 4; ++i) r.part[i] = from[i];
  return r.all;
}

// The unit after a worker's present one.
__device__ void next_unit(const Plan& plan, const Phase& ph, int units, int& place, int& e, int& head) {
  ++place;
  if (ph.columns == 0) {
    if (++e == ph.entries) {
      e = 0;
      ++head;
    }
    return;
  }
  if (place >= units) return;
  const int u = constant(plan.order + place);
  head = u / ph.entries, e = u - head * ph.entries;
}

template <typename T>
struct Args {
  const T* data;  // the layer's keys
  const T* q;
  int64_t q_token, q_head;
  const int32_t* table;
  T* out;
  float* lse;
  int64_t kv_stride, page_stride, head_stride, token_stride;
  int n_pages, page_shift, width, kv_heads, G, window, sinks;
  float scale2;  // scale * log2(e)
  bool join;     // a whole unit's rows still have to be joined with the other phase
  Plan plan;
  Work work;
};

// The kernel's arguments, read again where they are used: kept in registers from
// the start they would push the loops' own scalars out.
template <typename T>
__device__ const Args<T>& arguments() {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Args<T>*)p;
}

// The softmax state and output of 32 rows, one a lane pair.
template <typename T, int D>
struct Rows {
  vec8<T> q[D / 16];
  float16v o[D / 32];
  float top, sum;  // of the scaled scores in the exponent's units, less kLift; the lane's own keys

  __device__ void clear() {
    top = kFloor;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  }

  // Keys of product k (32 keys k / (D / 16), dims k % (D / 16)) of a chunk;
  // first: key_place of the lane's row and half.
  static __device__ vec8<T> read_keys(const char* keys, int first, int k) {
    return *reinterpret_cast<const vec8<T>*>(keys + k / (D / 16) * 32 * D * 2 + (first ^ (k % (D / 16) << 5)));
  }
  // S^T of 32 N keys.  Reads run kAhead products ahead (the order is kept by the
  // barriers: left alone, each product waits for its own read).
  static constexpr int kAhead = 4;
  template <int N>
  __device__ void scores(const char* keys, int first, float16v (&s)[N]) const {
    vec8<T> k[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) k[j] = read_keys(keys, first, j);
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = float16v{};
#pragma unroll
    for (int j = 0; j < N * (D / 16); ++j) {
      s[j / (D / 16)] = mfma(k[j % kAhead], q[j % (D / 16)], s[j / (D / 16)]);
      if (j + kAhead < N * (D / 16)) k[j % kAhead] = read_keys(keys, first, j + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // float16 ends at 2^-24 below and at 65504 above, so `top` is kept 2^8 below the
  // maximum and weights go to 65504: the second product then loses at most 2^-33 of
  // the largest weight from any other one.  With the maximum itself it was 2^-25, and
  // keys lighter than that added to the sum but not to the output.  24 prompts of
  // heads of 64 over windows of 1024 take 247 us either way, 251 with 2^10.
  static constexpr bool kHalf = __is_same(T, _Float16);
  static constexpr float kLift = kHalf ? 8.f : 0.f, kMostSum = kHalf ? 65504.f : 1024.f;

  // Raises the running maximum.
  __device__ void raise(float most) {
    const float now = fmaxf(top, most - kLift), shrink = __builtin_amdgcn_exp2f(top - now);
    top = now;
    sum *= shrink;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] *= shrink;
  }

  // Weights of the scores s, rounded to 16 bits as the second product's matrix
  // instructions take them (with 32-bit weights it would run at an eighth of the
  // rate); their sum, of the 32-bit ones, is added to the row's.
  // They are first taken with the maximum as it stands: a sum of at most kMostSum
  // says that none is too large, and a maximum that is a few orders too low
  // loses nothing.  Else the maximum is raised and they are taken again.
  template <int N>
  __device__ void weigh(const float16v (&s)[N], float scale2, vec8<T> (&w)[2 * N]) {
    float add = weights<N>(s, scale2, w);
    if (__any(!(add <= kMostSum))) {
      float most = s[0][0];
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, s[j][r]);
      raise(pair_max(most) * scale2);
      add = weights<N>(s, scale2, w);
    }
    sum += add;
  }
  template <int N>
  __device__ float weights(const float16v (&s)[N], float scale2, vec8<T> (&w)[2 * N]) const {
    float add[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[j][r], scale2, -top));
        add[r % 2] += p;
        w[2 * j + r / 8][r % 8] = (T)p;
      }
    return add[0] + add[1];
  }

  // V^T of 16 keys and 32 dims, the first product's order of keys: chunk c of
  // the keys, i of the dims, k = c D / 32 + i; first: value_place of the lane's
  // row and column.
  static __device__ vec8<T> read_values(const char* values, int first, int k) {
    union {
      short4v part[2];
      vec8<T> all;
    } v;
    typedef __attribute__((address_space(3))) short4v* lds4;
    const char* at = values + k / (D / 32) * 16 * D * 2 + (first ^ (k % (D / 32) << 6));
    v.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
    v.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * D * 2));
    return v.all;
  }

  // O^T += V^T P^T over 32 N keys; v holds the values of the first products.
  template <int N>
  __device__ void add(const char* values, int first, const vec8<T> (&w)[2 * N], vec8<T> (&v)[kAhead]) {
#pragma unroll
    for (int k = 0; k < 2 * N * (D / 32); ++k) {
      const int i = k % (D / 32);
      o[i] = mfma(v[k % kAhead], w[k / (D / 32)], o[i]);
      if (k + kAhead < 2 * N * (D / 32)) v[k % kAhead] = read_values(values, first, k + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Where a lane's reads begin.
template <int D>
__device__ int first_key() {
  const int lane = threadIdx.x & 63;
  return key_place<D>(lane & 31, lane >> 5);
}
template <int D>
__device__ int first_value() {
  const int lane = threadIdx.x & 63, t = lane & 15;
  return value_place<D>(4 * (lane >> 5) + (t >> 2), 32 * ((lane >> 4) & 1) + 8 * (t & 3));
}

// The lowest n bits.
__device__ uint64_t bits_below(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }

// p - window, of a window of any length.
__device__ int left_by(int p, int window) { return __builtin_elementwise_sub_sat(p, window); }

// Scores of keys that a row does not see become -inf; seen: its keys from the
// lane's first one on.
__device__ void hide(float16v& s, uint32_t seen) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const uint32_t keep = __builtin_amdgcn_sbfe(seen, 8 * (r / 4) + r % 4, 1);  // all bits or none
    s[r] = __uint_as_float((__float_as_uint(s[r]) & keep) | (0xff800000u & ~keep));
  }
}

// Loads the queries of the rows of a lane, zeros past the last one.
template <typename T, int D>
__device__ void load_rows(const Args<T>& a, const Entry& x, int head, int row, vec8<T>* q) {
  const int lane = threadIdx.x & 63;
  const bool there = row < x.rows;
  const int at = x.row0 + (there ? row : 0), token = at / a.G;
  const Global<const T> p =
      global(a.q) + (x.q0 + token) * a.q_token + (head * a.G + at - token * a.G) * a.q_head + 8 * (lane >> 5);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    q[k] = *(Global<const vec8<T>>)(p + 16 * k);
    if (!there)
#pragma unroll
      for (int j = 0; j < 8; ++j) q[k][j] = (T)0.f;
  }
}

// Writes a unit's rows of a wave: the result, or a part of it.
template <typename T, int D>
__device__ void store_rows(const Args<T>& a, int phase, const Entry& x, int head, int row, int tile_rows, bool whole,
                           int64_t slot, Rows<T, D>& r) {
  const int h = (threadIdx.x & 63) >> 5;
  const float sum = pair_sum(r.sum);
  if (row >= x.rows) return;
  const int at = x.row0 + row, token = at / a.G;
  const int64_t dense = (int64_t)(x.q0 + token) * (a.kv_heads * a.G) + head * a.G + at - token * a.G;
  if (whole && !a.join) {
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const Global<T> to = global(a.out) + dense * D + 4 * h;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        T v[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d] = (T)(sum == 0.f ? 0.f : r.o[i][4 * j + d] * inv);
        *(Global<uint64_t>)(to + 32 * i + 8 * j) = *reinterpret_cast<const uint64_t*>(v);
      }
    if (h == 0)
      global(a.lse)[dense] = sum == 0.f ? -INFINITY : kLn2 * (r.top + __builtin_amdgcn_logf(sum));
    return;
  }
  const Parts& w = a.work.part[phase];
  const int64_t at_row = whole ? dense : slot * tile_rows + row;
  const Global<float> to = global(whole ? w.whole_o : w.o) + at_row * D + 4 * h;
  typedef __attribute__((ext_vector_type(4))) float f4;
  typedef __attribute__((ext_vector_type(2))) float f2;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(Global<f4>)(to + 32 * i + 8 * j) =
          f4{r.o[i][4 * j], r.o[i][4 * j + 1], r.o[i][4 * j + 2], r.o[i][4 * j + 3]};
  if (h == 0) *((Global<f2>)(whole ? w.whole_ml : w.ml) + at_row) = f2{r.top, sum};
}

// Keeps an address of the wave apart from the lane's places that are added to
// it, so that loads take both as they are.
__device__ Global<const char> apart(Global<const char> p) {
  asm volatile("" : "+s"(p));
  return p;
}
__device__ uint4 load_uint4(Global<const char> p) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  const u4 x = *(Global<const u4>)p;
  return make_uint4(x.x, x.y, x.z, x.w);
}

// The key tiles of a unit, TK places of a list each: the sinks, up to a multiple
// of 16, then the main run from a multiple of 16 on.  So tiles are full but for
// the last (with sinks in tiles of their own, 24 prompts over windows of 1024 took
// 260 us, so 247; over windows of 256, 167 and 146).
//
// Sixteens: pages have at least 16 tokens.  Tiles begin at multiples of 16, so
// each 16 keys lie in one page and are loaded from one address of the wave.
// The pages of kBatch tiles are looked up at once, one lane a page: those of
// the batch that the present tile is in and of the next one are held, even
// batches' in one register and odd ones' in the other.
// Otherwise every lane looks its key's page up before it loads.
template <typename T, int D, int TK, bool Sixteens>
struct Tiles {
  static constexpr int LPR = D / 8, KPI = 64 / LPR;  // lanes a key, keys a load
  static constexpr int kLoads = 16 / KPI;            // loads of 16 keys
  static constexpr int kGroups = TK / 16, kBatch = 64 / kGroups;
  Global<const int32_t> row;
  Global<const char> base;  // the key head's first key
  int hi, sink, skip, move, shift, pages;  // places below skip are keys, the others keys from `move` back
  int c0, c1;        // in tiles [c0, c1) every row sees every key
  int p_first, p_last;
  uint32_t page_bytes, page_bytes_hi, token_bytes;
  int64_t to_values;
  uint32_t step;  // a lane's place in a load, and how far on the next load of 16 keys is
  uint32_t stride;
  int batch, evens, odds;

  __device__ Tiles(const Args<T>& a, const Entry& x, int head) {
    const int lane = threadIdx.x & 63;
    const bool there_is = x.slot >= 0;
    row = global(a.table + (int64_t)(there_is ? x.slot : 0) * a.width);
    base = global(reinterpret_cast<const char*>(a.data + head * a.head_stride));
    hi = there_is ? x.end : 0, sink = there_is ? x.sink : 0;
    skip = (x.sink + 15) & ~15, move = x.lo - skip;
    shift = a.page_shift, pages = a.n_pages;
    p_first = x.pos0 + x.row0 / a.G, p_last = x.pos0 + (x.row0 + x.rows - 1) / a.G;
    const int below = p_first + 1 < hi ? p_first + 1 : hi;    // every row sees the keys before it,
    const int above = a.window > 0 ? left_by(p_last + 1 - move, a.window) : 0;  // and those from this place on
    c0 = ((above > skip ? above : skip) + TK - 1) / TK;
    c1 = below > move ? (below - move) / TK : 0;
    const uint64_t bytes = 2 * a.page_stride;
    page_bytes = (uint32_t)bytes, page_bytes_hi = (uint32_t)(bytes >> 32);
    token_bytes = 2 * (uint32_t)a.token_stride;
    to_values = 2 * a.kv_stride;
    step = lane / LPR * token_bytes + lane % LPR * 16;
    stride = KPI * token_bytes;
  }

  __device__ int key_at(int place) const { return place < skip ? place : place + move; }
  __device__ bool held(int page) const { return (unsigned)page < (unsigned)pages; }
  // The table's entry for a place (some entry, past the last key).
  __device__ int entry_of(int place) const {
    const int key = key_at(place);
    return row[(key < hi ? key : hi > 0 ? hi - 1 : 0) >> shift];
  }

  __device__ int find(int b) const { return entry_of(b * kBatch * TK + 16 * (threadIdx.x & 63)); }
  __device__ void begin(int t) {
    if (!Sixteens) return;
    batch = t / kBatch;
    evens = find(batch + batch % 2);
    odds = find(batch + 1 - batch % 2);
  }
  __device__ void advance(int t) {
    if (!Sixteens || t / kBatch == batch) return;
    ++batch;
    if (batch % 2) evens = find(batch + 1);
    else odds = find(batch + 1);
  }
  // The lookup that tile t is in.  Branches, so that nothing waits for the next
  // batch that does not need it: loads return in order, and the wait would be
  // for all loads before it.
  __device__ int lookup(int t) const {
    int r;
    if (t / kBatch % 2) {
      r = odds;
      asm volatile("" : "+v"(r));
    } else {
      r = evens;
      asm volatile("" : "+v"(r));
    }
    return r;
  }
  __device__ int page_at(int t, int group) const {
    return __builtin_amdgcn_readlane(lookup(t), t % kBatch * kGroups + group);
  }

  // Every key is there, and every row sees it.
  __device__ bool clean(int t) const {
    if (t < c0 || t >= c1) return false;
    if (Sixteens) {
      const uint64_t ok = __ballot(held(lookup(t)));
      const uint32_t mask = (1u << kGroups) - 1;
      return ((uint32_t)(ok >> (t % kBatch * kGroups)) & mask) == mask;
    }
    bool all = true;
#pragma unroll
    for (int c = 0; c < TK; c += 64) all = all && __all(held(entry_of(t * TK + c + (threadIdx.x & (TK < 64 ? 31 : 63)))));
    return all;
  }
  // Every row sees every key of the tile that is there (false for some tiles of which that is true).
  __device__ bool even(int t) const {
    if (t * TK < skip) return false;
    const int window = arguments<T>().window, sinks = arguments<T>().sinks;
    const int k0 = t * TK + move, k1 = k0 + TK < hi ? k0 + TK : hi;
    return k1 - 1 <= p_first && (window == 0 || k0 > left_by(p_last, window) || k1 <= sinks);
  }

  // Bits of the keys of chunk c (64 keys) that are there and that some row may
  // see.
  __device__ uint64_t there(int t, int c = 0) const {
    const int v0 = t * TK + 64 * c;
    uint64_t m = 0;
    if (Sixteens) {
#pragma unroll
      for (int j = 0; j < (TK < 64 ? TK : 64) / 16; ++j)
        if (held(page_at(t, 4 * c + j))) m |= 0xffffull << (16 * j);
    } else {
      m = __ballot(held(entry_of(v0 + (threadIdx.x & 63))));
      if (TK == 32) m = (uint32_t)m;
    }
    return m & merged(v0, bits_below(hi - v0 - move) & in_window(v0 + move, p_first));
  }
  // Bits of the 64 places from v0 on: the sinks, and of the main run those given.
  __device__ uint64_t merged(int v0, uint64_t main) const {
    return (main & ~bits_below(skip - v0)) | bits_below(sink - v0);
  }
  // Bits of the keys [here, here + 64) that a row at position p has not left behind.
  __device__ uint64_t in_window(int here, int p) const {
    const int window = arguments<T>().window, sinks = arguments<T>().sinks;
    return window > 0 ? ~bits_below(left_by(p - here + 1, window)) | bits_below(sinks - here) : ~0ull;
  }
  // Those of `there` (chunk c of tile t) that the row at position p sees.  Every row is past the sinks.
  __device__ uint64_t seen(uint64_t there, int t, int c, int p) const {
    const int v0 = t * TK + 64 * c, here = v0 + move;
    return there & merged(v0, bits_below(p - here + 1) & in_window(here, p));
  }
  // Some row at a position from `from` to `to` may see keys of the chunk.
  __device__ bool meets(int t, int c, int from, int to) const {
    const int v0 = t * TK + 64 * c, k0 = v0 + move, window = arguments<T>().window, sinks = arguments<T>().sinks;
    return v0 < skip || (k0 < hi && k0 <= to && (window == 0 || k0 + 63 > left_by(from, window) || k0 < sinks));
  }

  // Where 16 keys of a tile lie (page 0's where there is no page).
  struct At {
    Global<const char> k, v;
  };
  __device__ At address(int t, int key) const {
    const int at = page_at(t, key / 16);
    const uint32_t page = held(at) ? at : 0, in = key_at(t * TK + key) & ((1 << shift) - 1);
    const uint64_t off = (uint64_t)page * page_bytes + ((uint64_t)(page * page_bytes_hi) << 32) + in * token_bytes;
    At r;
    r.k = apart(base + off);
    r.v = apart(r.k + to_values);
    return r;
  }

  __device__ uint4 load16(Global<const char> p, int i) const {  // load i of 16 keys
    return load_uint4(apart(p + i * stride) + step);
  }

  // Loads keys [key0, key0 + NI KPI) of the tile, key0 a multiple of 16: 16
  // bytes a lane.
  template <int NI>
  __device__ void load(int t, int key0, uint4 (&k)[NI], uint4 (&v)[NI]) const {
    const int lane = threadIdx.x & 63, mask = (1 << shift) - 1;
    if (Sixteens) {
#pragma unroll
      for (int g = 0; g < NI / kLoads; ++g) {
        const At at = address(t, key0 + 16 * g);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          k[g * kLoads + i] = load16(at.k, i);
          v[g * kLoads + i] = load16(at.v, i);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int place = t * TK + key0 + i * KPI + lane / LPR, key = key_at(place), at = entry_of(place);
        const Global<const char> p = base + (held(at) ? at : 0) * (int64_t)((uint64_t)page_bytes_hi << 32 | page_bytes) +
                                     (key & mask) * token_bytes + lane % LPR * 16;
        k[i] = load_uint4(p);
        v[i] = load_uint4(p + to_values);
      }
    }
  }
};

// A tile's share of one wave, from registers to LDS.
template <typename T, int D, int NI>
__device__ void put_keys(char* keys, char* values, int key0, const uint4 (&k)[NI], const uint4 (&v)[NI]) {
  constexpr int LPR = D / 8, KPI = 64 / LPR;
  const int lane = threadIdx.x & 63, chunk = lane % LPR;
  const int kp = fresh(key_place<D>(key0 + lane / LPR, chunk));
  const int vp = fresh(value_place<D>(key0 + lane / LPR, chunk * 16));
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    // KPI keys on, a chunk's place in its row moves with the key
    const int step = i * KPI, move = D == 128 ? (step & 15) << 4 : ((step >> 1) & 7) << 4;
    *reinterpret_cast<uint4*>(keys + (kp ^ move) + step * D * 2) = k[i];
    *reinterpret_cast<uint4*>(values + vp + step * D * 2) = v[i];
  }
}

// Before that, zeros for the keys that are not there; true if a value is not
// finite.
template <typename T, int D, int NI>
__device__ bool clear_keys(int key0, uint64_t there, uint4 (&k)[NI], uint4 (&v)[NI]) {
  constexpr int LPR = D / 8, KPI = 64 / LPR;
  const int lane = threadIdx.x & 63;
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const uint32_t keep = there >> (key0 + i * KPI + lane / LPR) & 1 ? ~0u : 0u;
    k[i].x &= keep, k[i].y &= keep, k[i].z &= keep, k[i].w &= keep;
    v[i].x &= keep, v[i].y &= keep, v[i].z &= keep, v[i].w &= keep;
    bad |= not_finite(v[i].x, T()) | not_finite(v[i].y, T()) | not_finite(v[i].z, T()) | not_finite(v[i].w, T());
  }
  return bad != 0;
}

// ---------------------------------------------------------------------------
// The workgroup kernel: 32 rows a wave; the waves load a tile of keys and
// values for all, worked on in chunks of 64 keys.  While a tile is in use the
// next one goes from registers to the other half of LDS and the one after
// that is loaded; one barrier a tile.
//
// Bounds: a chunk's products of a wave take 32 cycles a matrix instruction and
// its softmax 8 an exponential, about as long in all with heads of 64 and half
// as long with heads of 128, of which a SIMD's two waves hide only a part from
// each other; and at full use of the matrix units the card lowers its clock (a
// loop of nothing but products on random registers: 1.7 PFLOP/s, with four
// vector instructions a product 1.5).  Heads of 128: 800 TFLOP/s on one prompt
// of 16,384 tokens, matrix instructions busy 40% of the cycles and vector
// instructions 39%, at 2.0 GHz.  Heads of 64: 720 TFLOP/s over windows of 4096;
// over windows of 1024 a unit has nine tiles, and its beginning, end and masks
// leave 500 (24 prompts, 20 query and 4 key heads, 253 us with the join).
//
// 256 rows (eight waves, tiles of 128 keys) read each key half as often as 128
// rows from L2 and put half as many barriers between products: 1.46 ms against
// 1.65 ms on that prompt.  Four waves serve up to 128 rows, where the others'
// would idle.
// ---------------------------------------------------------------------------
template <int D, int NW>
constexpr int kBlockRoom = 2 * 2 * block_keys(NW) * D * 2;  // LDS: two tiles' keys and values

template <typename T, int D, int NW, bool Sixteens>
__device__ __forceinline__ void block_units(char* room, int phase, int block, int blocks) {
  constexpr int TK = block_keys(NW);
  using Keys = Tiles<T, D, TK, Sixteens>;
  constexpr int NI = TK / NW / Keys::KPI, kChunk = 64 * D * 2, kTile = TK * D * 2;
  char* const keys = room;
  char* const values = room + 2 * kTile;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = wave * (TK / NW);  // the wave's first key of a tile
  const int id = block % 8 * (blocks / 8) + block / 8;
  int place, e, head, t0;
  int64_t left;
  {
    const Args<T>& a = arguments<T>();
    const Phase ph = constant(a.plan.phase + phase);
    if (id >= ph.workers) return;
    const int64_t all = ph.total * a.kv_heads, beg = id * ph.share;
    left = (beg + ph.share < all ? beg + ph.share : all) - beg;
    const Start st = constant(a.plan.start[phase] + id);
    place = st.place, e = st.entry, head = st.head, t0 = st.tile;
  }
  const float scale2 = arguments<T>().scale2;
  bool leading = true, odd = false;
  Rows<T, D> rows;

  while (left > 0) {
    const Args<T>& a = arguments<T>();
    const Entry x = constant(a.plan.entry[phase] + e);
    const int n = (int)(x.tiles - t0 < left ? x.tiles - t0 : left);
    const int row = wave * 32 + (lane & 31);
    Keys tiles(a, x, head);
    tiles.begin(t0);
    load_rows<T, D>(a, x, head, row, rows.q);
    rows.clear();
    const int p = x.pos0 + (x.row0 + (row < x.rows ? row : x.rows - 1)) / a.G;

    const bool busy = wave * 32 < x.rows;  // the wave's rows are at positions w_first .. w_end
    const int w_last = wave * 32 + 31 < x.rows ? wave * 32 + 31 : x.rows - 1;
    const int w_first = x.pos0 + (x.row0 + wave * 32) / a.G, w_end = x.pos0 + (x.row0 + w_last) / a.G;

    uint4 kreg[NI], vreg[NI];
    auto clear = [&](int t) {
      const bool bad = clear_keys<T, D, NI>(mine % 64, tiles.there(t, mine / 64), kreg, vreg);
      odd |= bad && !tiles.even(t);
    };
    auto chunk = [&](int buf, int c, bool clean, int t) {
      float16v s[2];
      const int kp = fresh(first_key<D>()), vp = fresh(first_value<D>());
      const char* kc = keys + buf * kTile + c * kChunk;
      const char* vc = values + buf * kTile + c * kChunk;
      vec8<T> v[Rows<T, D>::kAhead], w[4];
      rows.template scores<2>(kc, kp, s);
#pragma unroll
      for (int j = 0; j < Rows<T, D>::kAhead; ++j) v[j] = rows.read_values(vc, vp, j);
      if (!clean) {
        const uint64_t seen = tiles.seen(tiles.there(t, c), t, c, p) >> (4 * (lane >> 5));
        hide(s[0], (uint32_t)seen);
        hide(s[1], (uint32_t)(seen >> 32));
      }
      rows.template weigh<2>(s, scale2, w);
      rows.template add<2>(vc, vp, w, v);
    };

    bool clean = tiles.clean(t0), next = tiles.clean(t0 + 1);
    tiles.load(t0, mine, kreg, vreg);
    __syncthreads();  // the last unit's tiles are no longer read
    if (!clean) clear(t0);
    put_keys<T, D, NI>(keys, values, mine, kreg, vreg);
    tiles.load(t0 + 1, mine, kreg, vreg);
    for (int i = 0; i < n; ++i) {
      const int buf = i & 1, t = t0 + i, t2 = i + 2 < n ? t + 2 : t0 + n - 1;  // the last loads are of no use
      // The pages are looked up before the tile's loads: what waits for a lookup then does not wait for them.
      tiles.advance(t);
      const bool third = tiles.clean(t + 2);
      __syncthreads();
#pragma unroll
      for (int c = 0; c < TK / 64; ++c) {
        if (busy && (clean || tiles.meets(t, c, w_first, w_end))) chunk(buf, c, clean, t);
        if (c == 0) {
          // no load in a branch: where the ways meet, the registers would be copied, and the copies would wait
          if (!next) clear(t + 1);
          put_keys<T, D, NI>(keys + (buf ^ 1) * kTile, values + (buf ^ 1) * kTile, mine, kreg, vreg);
          tiles.load(t2, mine, kreg, vreg);
        }
      }
      clean = next, next = third;
    }
    const Args<T>& z = arguments<T>();
    const Entry y = constant(z.plan.entry[phase] + e);
    store_rows<T, D>(z, phase, y, head, row, NW * 32, t0 == 0 && n == y.tiles, (int64_t)id * 2 + (leading ? 0 : 1), rows);
    leading = false;
    left -= n;
    t0 = 0;
    const Phase ph = constant(z.plan.phase + phase);
    next_unit(z.plan, ph, ph.entries * z.kv_heads, place, e, head);
  }
  const Global<int32_t> flags = global(arguments<T>().work.odd[phase]);
  if (lane == 0) flags[id * NW + wave] = 0;
  if (odd) flags[id * NW + wave] = 1;
}

template <typename T, int D, int NW, bool Sixteens>
__global__ __launch_bounds__(NW * 64, 2) void attend_block(Args<T>, int phase) {
  __shared__ __align__(16) char room[kBlockRoom<D, NW>];
  block_units<T, D, NW, Sixteens>(room, phase, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------------------
// The wave kernel: up to 32 rows (a few query tokens), the keys streamed by
// waves that share nothing: each loads the next tile of 32 keys into registers
// while it works on the present one from LDS, so a CU's eight waves have 128
// KiB of loads in flight with heads of 128, and no wave waits for another.
// Bound by memory: 193 us for 0.97 GB of keys and values (256 sequences, windows
// of 4096, 8 key heads of 128), 5.0 TB/s, what a large copy reaches.  Short
// units lose to their beginnings (page lookup, first tile): 512 sequences' own
// 128 tokens, 0.28 GB, take 80 us, 3.4 TB/s.
//
// Split: a workgroup takes one unit, a quarter of its tiles a wave, and joins
// the four parts itself.
// ---------------------------------------------------------------------------
template <int D>
constexpr int kWaveRoom = 2 * kRowKeys * D * 2;  // LDS of a wave: a tile's keys and values

template <typename T, int D, bool Sixteens, bool Split>
__device__ __forceinline__ void wave_units(char* room, int phase, int block, int blocks) {
  using Keys = Tiles<T, D, kRowKeys, Sixteens>;
  constexpr int TK = kRowKeys, NI = TK / Keys::KPI;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* const keys = room + wave * kWaveRoom<D>;
  char* const values = keys + TK * D * 2;
  const int at_line = block % 8 * (blocks / 8) + block / 8, id = Split ? at_line : at_line * kWaves + wave;
  int place, e, head, t0;
  int64_t left;
  {
    const Args<T>& a = arguments<T>();
    const Phase ph = constant(a.plan.phase + phase);
    if (id >= ph.workers) return;
    const int64_t all = ph.total * a.kv_heads, beg = id * ph.share;
    left = (beg + ph.share < all ? beg + ph.share : all) - beg;
    const Start st = constant(a.plan.start[phase] + id);
    place = st.place, e = st.entry, head = st.head, t0 = st.tile;
    if (Split) {
      const int tiles = constant(a.plan.entry[phase] + e).tiles, part = (tiles + kWaves - 1) / kWaves;
      t0 = wave * part;
      left = tiles - t0 < part ? tiles - t0 : part;
      if (left < 0) left = 0;
    }
  }
  const float scale2 = arguments<T>().scale2;
  bool leading = true, odd = false;
  Rows<T, D> rows;

  if (Split) rows.clear();
  while (left > 0) {
    const Args<T>& a = arguments<T>();
    const Entry x = constant(a.plan.entry[phase] + e);
    const int n = (int)(x.tiles - t0 < left ? x.tiles - t0 : left);
    const int row = lane & 31;
    Keys tiles(a, x, head);
    tiles.begin(t0);
    load_rows<T, D>(a, x, head, row, rows.q);
    rows.clear();
    const int p = x.pos0 + (x.row0 + (row < x.rows ? row : x.rows - 1)) / a.G;
    uint4 kreg[NI], vreg[NI];
    tiles.load(t0, 0, kreg, vreg);
    for (int i = 0; i < n; ++i) {
      const int t = t0 + i;
      const bool clean = tiles.clean(t);
      uint32_t held = ~0u;
      if (!clean) {
        held = (uint32_t)tiles.there(t);
        const bool bad = clear_keys<T, D, NI>(0, held, kreg, vreg);
        // with one position, what is there is seen by all rows
        odd |= bad && tiles.p_first != tiles.p_last && !tiles.even(t);
      }
      put_keys<T, D, NI>(keys, values, 0, kreg, vreg);
      tiles.advance(t + 1);
      if (i + 1 < n) tiles.load(t + 1, 0, kreg, vreg);
      __builtin_amdgcn_wave_barrier();
      const int kp = fresh(first_key<D>()), vp = fresh(first_value<D>());
      float16v s[1];
      rows.template scores<1>(keys, kp, s);
      vec8<T> v[Rows<T, D>::kAhead];
#pragma unroll
      for (int j = 0; j < Rows<T, D>::kAhead; ++j) v[j] = rows.read_values(values, vp, j);
      if (!clean) hide(s[0], (uint32_t)tiles.seen(held, t, 0, p) >> (4 * (lane >> 5)));
      vec8<T> w[2];
      rows.template weigh<1>(s, scale2, w);
      rows.template add<1>(values, vp, w, v);
      __builtin_amdgcn_wave_barrier();
    }
    if (Split) break;
    const Args<T>& z = arguments<T>();
    const Entry y = constant(z.plan.entry[phase] + e);
    store_rows<T, D>(z, phase, y, head, row, kRowTile, t0 == 0 && n == y.tiles, (int64_t)id * 2 + (leading ? 0 : 1), rows);
    leading = false;
    left -= n;
    t0 = 0;
    const Phase ph = constant(z.plan.phase + phase);
    next_unit(z.plan, ph, ph.entries * z.kv_heads, place, e, head);
  }
  if (!Split) {
    const Global<int32_t> flags = global(arguments<T>().work.odd[phase]);
    if (lane == 0) flags[id] = 0;
    if (odd) flags[id] = 1;
    return;
  }
  __shared__ float2 ml[kWaves][kRowTile];
  const Args<T>& a = arguments<T>();
  const Entry x = constant(a.plan.entry[phase] + e);
  const int row = lane & 31, h = lane >> 5;
  const float sum = pair_sum(rows.sum);
  if (row < x.rows) {
    float* to = reinterpret_cast<float*>(keys) + row * D + 4 * h;  // the tiles have been read
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(to + 32 * i + 8 * j) = make_float4(
            rows.o[i][4 * j], rows.o[i][4 * j + 1], rows.o[i][4 * j + 2], rows.o[i][4 * j + 3]);
    if (h == 0) ml[wave][row] = make_float2(rows.top, sum);
  }
  __syncthreads();
  constexpr int W = D / 16;
  const int i16 = threadIdx.x & 15;
  for (int r = threadIdx.x / 16; r < x.rows; r += kWaves * 4) {
    float top = kFloor, all = 0.f, o[W] = {};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, ml[i][r].x);
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float w = __builtin_amdgcn_exp2f(ml[i][r].x - top);
      all = fmaf(ml[i][r].y, w, all);
      const float* from = reinterpret_cast<const float*>(room + i * kWaveRoom<D>) + r * D + i16 * W;
#pragma unroll
      for (int d = 0; d < W; ++d) o[d] = fmaf(from[d], w, o[d]);
    }
    const int at = x.row0 + r, token = at / a.G;
    const int64_t dense = (int64_t)(x.q0 + token) * (a.kv_heads * a.G) + head * a.G + at - token * a.G;
    const float inv = all == 0.f ? 0.f : 1.f / all;
    vec8<T> v = {};
#pragma unroll
    for (int d = 0; d < W; ++d) v[d] = (T)(all == 0.f ? 0.f : o[d] * inv);
    const Global<T> to = global(a.out) + dense * D + i16 * W;
    if (W == 8) *(Global<vec8<T>>)to = v;
    else *(Global<uint64_t>)to = *reinterpret_cast<const uint64_t*>(&v);
    if (i16 == 0) global(a.lse)[dense] = all == 0.f ? -INFINITY : kLn2 * (top + __builtin_amdgcn_logf(all));
  }
}

template <typename T, int D, bool Sixteens, bool Split>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_wave(Args<T>, int phase) {
  __shared__ __align__(16) char room[kWaves * kWaveRoom<D>];
  wave_units<T, D, Sixteens, Split>(room, phase, blockIdx.x, gridDim.x);
}

// Both phases of a batch behind shared prefixes at once: on each CU one
// workgroup has the shared keys, where the matrix unit is the limit, and one
// streams sequences' own keys, where memory is.  46 us for 64 sequences of 40
// key heads of 128 with up to 128 tokens each behind 2048 (0.24 GB, 5.3 TB/s),
// 17 us for 63 of 3 key heads of 64 behind up to 4001 tokens.
template <typename T, int D, bool Sixteens>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_both(Args<T>) {
  static_assert(kBlockRoom<D, 4> == kWaves * kWaveRoom<D>, "one room serves either");
  __shared__ __align__(16) char room[kBlockRoom<D, 4>];
  // Eight by eight, so that each XCD has both, and the other way round from the XCD's 33rd on, which join its first 32
  // on their CUs.
  const int block = blockIdx.x / 16 * 8 + blockIdx.x % 8;
  if ((blockIdx.x / 8 + blockIdx.x / 256) % 2 == 0) block_units<T, D, 4, Sixteens>(room, 0, block, gridDim.x / 2);
  else wave_units<T, D, Sixteens, false>(room, 1, block, gridDim.x / 2);
}

// ---------------------------------------------------------------------------
// The join
// ---------------------------------------------------------------------------

// The parts of unit (entry, head) of a phase: workers [w0, w1], whole if one.
struct Cut {
  int64_t w0, w1, c0, share;
};
__device__ Cut cut_of(const Phase& ph, const int64_t* cum, int entry, int head) {
  Cut u;
  u.share = ph.share;
  u.c0 = head * ph.total + cum[entry];
  u.w0 = u.c0 / ph.share;
  u.w1 = (head * ph.total + cum[entry + 1] - 1) / ph.share;
  return u;
}

// The parts of a row, joined by 16 lanes, four rows a wave.  Lane i of them
// first takes the maximum and sum of part i, so that all parts' weights are
// known at once and their outputs are loaded without waiting for one another.
template <int D>
struct Joined {
  static constexpr int W = D / 16;  // a lane's dims
  float top = kFloor, sum = 0.f, o[W] = {};

  // from(i, o, ml): where part i's row lies; 0 parts where there is no row.
  template <typename From>
  __device__ void take(int parts, From from) {
    const int i16 = threadIdx.x & 15;
    for (int i0 = 0; __any(i0 < parts); i0 += 16) {
      const int n = parts - i0 < 16 ? parts - i0 : 16;
      const float* at = nullptr;
      float2 ml = make_float2(kFloor, 0.f);
      if (i16 < n) {
        const float2* m;
        from(i0 + i16, at, m);
        ml = *m;
      }
      float now = fmaxf(top, ml.x);
#pragma unroll
      for (int d = 8; d; d >>= 1) now = fmaxf(now, __shfl_xor(now, d, 16));
      const float w = __builtin_amdgcn_exp2f(ml.x - now), shrink = __builtin_amdgcn_exp2f(top - now);
      float add = i16 < n ? ml.y * w : 0.f;
#pragma unroll
      for (int d = 8; d; d >>= 1) add += __shfl_xor(add, d, 16);
      sum = sum * shrink + add;
      top = now;
#pragma unroll
      for (int d = 0; d < W; ++d) o[d] *= shrink;
      const uint64_t addr = reinterpret_cast<uint64_t>(at);
      constexpr int kBatch = 4;
      for (int i = 0; __any(i < n); i += kBatch) {
        float4 v[kBatch][W / 4];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const float4* p = reinterpret_cast<const float4*>(__shfl(addr, i + j, 16)) + i16 * (W / 4);
#pragma unroll
          for (int d = 0; d < W / 4; ++d) v[j][d] = i + j < n ? p[d] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const float wi = __shfl(w, i + j, 16);
          if (i + j < n)
#pragma unroll
            for (int d = 0; d < W / 4; ++d) {
              o[4 * d] = fmaf(v[j][d].x, wi, o[4 * d]);
              o[4 * d + 1] = fmaf(v[j][d].y, wi, o[4 * d + 1]);
              o[4 * d + 2] = fmaf(v[j][d].z, wi, o[4 * d + 2]);
              o[4 * d + 3] = fmaf(v[j][d].w, wi, o[4 * d + 3]);
            }
        }
      }
    }
  }
};

// Part i of a cut unit's row.
__device__ void part_at(const Parts& p, const Cut& u, int i, int tile_rows, int row, int64_t dense, int D,
                        const float*& o, const float2*& ml) {
  if (u.w0 == u.w1) {
    o = p.whole_o + dense * D;
    ml = p.whole_ml + dense;
    return;
  }
  const int64_t w = u.w0 + i, at = (2 * w + (u.c0 <= w * u.share ? 0 : 1)) * tile_rows + row;
  o = p.o + at * D;
  ml = p.ml + at;
}

// A row's output again, key by key, without the keys that it does not see: the
// products of whole tiles take a weight of 0 times a value, which is not 0
// where the value is not finite.  Its weights keep 32 bits, so the row's last bits
// may differ from those of the tiles.  lse2: the row's lse in the exponent's units.
template <typename T, int D>
__device__ void redo_row(const Args<T>& a, const Entry& x, int head, int row, float lse2) {
  const int lane = threadIdx.x & 63;
  const int at = x.row0 + row, token = at / a.G, member = at - token * a.G;
  const int p = x.pos0 + token;
  const T* q = a.q + (x.q0 + token) * a.q_token + (head * a.G + member) * a.q_head;
  float o[D / 64] = {}, sum = 0.f;
  for (int k0 = 0; k0 <= p && x.slot >= 0; k0 += 64) {
    if (a.window > 0 && k0 >= a.sinks && k0 + 63 <= left_by(p, a.window)) continue;
    const int key = k0 + lane;
    int page = -1;
    if (key <= p && (a.window == 0 || key > left_by(p, a.window) || key < a.sinks))
      page = a.table[(int64_t)x.slot * a.width + (key >> a.page_shift)];
    if (page >= a.n_pages) page = -1;
    const int in = key & ((1 << a.page_shift) - 1);
    const T* k = a.data + (page < 0 ? 0 : page) * a.page_stride + head * a.head_stride + in * a.token_stride;
    float s = 0.f;
    for (int d = 0; d < D; ++d) s = fmaf((float)q[d], (float)k[d], s);
    const float w = __builtin_amdgcn_exp2f(fmaf(s, a.scale2, -lse2));
    const uint64_t v_at = reinterpret_cast<uint64_t>(k + a.kv_stride);
    for (uint64_t seen = __ballot(page >= 0); seen; seen &= seen - 1) {
      const int i = __builtin_ctzll(seen);
      const T* v = reinterpret_cast<const T*>(__shfl(v_at, i)) + lane * (D / 64);
      const float wi = __shfl(w, i);
      sum += wi;
      for (int d = 0; d < D / 64; ++d) o[d] = fmaf(wi, (float)v[d], o[d]);
    }
  }
  const int64_t dense = (int64_t)(x.q0 + token) * (a.kv_heads * a.G) + head * a.G + member;
  for (int d = 0; d < D / 64; ++d) a.out[dense * D + lane * (D / 64) + d] = (T)(sum == 0.f ? 0.f : o[d] / sum);
}

// Joins the rows of a unit of the sequences' own keys that this wave has: four
// from `row` on, then `step` on.
template <typename T, int D>
__device__ void join_rows(const Args<T>& a, const Entry& x, const Cut& u, int head, int row, int step, int rows0,
                          int rows1, bool odd) {
  const int lane = threadIdx.x & 63, i16 = lane & 15;
  constexpr int W = Joined<D>::W;
  for (; row < x.rows; row += step) {
    const int mine = row + lane / 16;
    const bool there = mine < x.rows;
    const int at = x.row0 + (there ? mine : row), token = at / a.G;
    const int64_t dense = (int64_t)(x.q0 + token) * (a.kv_heads * a.G) + head * a.G + at - token * a.G;
    Cut u0 = {};
    int before = 0, row0 = 0;
    if (x.prefix >= 0) {
      row0 = x.prefix_row + (there ? mine : row);
      u0 = cut_of(a.plan.phase[0], a.plan.cum[0], x.prefix + row0 / rows0, head);
      row0 %= rows0;
      before = (int)(u0.w1 - u0.w0) + 1;
    }
    Joined<D> r;
    r.take(there ? before + (int)(u.w1 - u.w0) + 1 : 0, [&](int i, const float*& o, const float2*& ml) {
      if (i < before) part_at(a.work.part[0], u0, i, rows0, row0, dense, D, o, ml);
      else part_at(a.work.part[1], u, i - before, rows1, mine, dense, D, o, ml);
    });
    const float inv = r.sum == 0.f ? 0.f : 1.f / r.sum;
    const float lse2 = r.sum == 0.f ? -INFINITY : r.top + __builtin_amdgcn_logf(r.sum);
    if (there) {
      vec8<T> v = {};
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = (T)(r.sum == 0.f ? 0.f : r.o[i] * inv);
      T* to = a.out + dense * D + i16 * W;
      if (W == 8) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(&v);
      else *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(&v);
      if (i16 == 0) a.lse[dense] = kLn2 * lse2;
    }
    for (int i = 0; odd && i < 4 && row + i < x.rows; ++i)
      redo_row<T, D>(a, x, head, row + i, __shfl(lse2, 16 * i));
  }
}

// Whether a worker of the cut met values that are not finite.
template <typename T>
__device__ bool any_odd(const Args<T>& a, const Cut& u, int flags) {
  int odd = 0;
  for (int64_t w = u.w0 * flags + (threadIdx.x & 63); w < (u.w1 + 1) * flags; w += 64) odd |= a.work.odd[1][w];
  return __any(odd);
}

// The join is bound by latency: a row's parts and its plan are found through
// three dependent loads.  9 us for 2560 rows of 128, 15 us for 16,384.
//
// With a shared prefix every row is joined: `fours` waves take a unit of key
// head blockIdx.y, four rows each.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_units(Args<T> a, int rows0, int rows1, int flags, int fours) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.y;
  const Phase own = a.plan.phase[1];
  for (int id = blockIdx.x * 4 + wave; id < own.entries * fours; id += gridDim.x * 4) {
    const int e = id / fours;
    const Entry x = a.plan.entry[1][e];
    const Cut u = cut_of(own, a.plan.cum[1], e, head);
    join_rows<T, D>(a, x, u, head, (id - e * fours) * 4, fours * 4, rows0, rows1, any_odd(a, u, flags));
  }
}

// Otherwise only the units that are cut: the worker whose share begins inside a
// unit, as the first one to, joins it.  A worker that met values that are not
// finite also does its whole units' rows again.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_cuts(Args<T> a, int rows1, int flags, int fours) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), id = blockIdx.x * 4 + wave, w = id / fours;
  const int row = (id - w * fours) * 4, step = fours * 4;
  const Phase own = a.plan.phase[1];
  if (w >= own.workers) return;
  const Start st = a.plan.start[1][w];
  if (st.tile > 0 && st.tile <= own.share) {
    const Entry x = a.plan.entry[1][st.entry];
    Cut u;
    u.share = own.share;
    u.c0 = w * own.share - st.tile;
    u.w0 = u.c0 / u.share;
    u.w1 = (u.c0 + x.tiles - 1) / u.share;
    join_rows<T, D>(a, x, u, st.head, row, step, rows1, rows1, any_odd(a, u, flags));
  }
  if (!any_odd(a, Cut{w, w, 0, 0}, flags)) return;
  const int64_t all = own.total * a.kv_heads, beg = w * own.share;
  int place = st.place, e = st.entry, head = st.head, t = st.tile;
  for (int64_t left = (beg + own.share < all ? beg + own.share : all) - beg; left > 0;) {
    const Entry x = a.plan.entry[1][e];
    const int n = (int)(x.tiles - t < left ? x.tiles - t : left);
    for (int r = row / 4; n == x.tiles && r < x.rows; r += step / 4) {
      const int at = x.row0 + r, token = at / a.G;
      const int64_t dense = (int64_t)(x.q0 + token) * (a.kv_heads * a.G) + head * a.G + at - token * a.G;
      redo_row<T, D>(a, x, head, r, a.lse[dense] * kLog2e);
    }
    left -= n;
    t = 0;
    next_unit(a.plan, own, own.entries * a.kv_heads, place, e, head);
  }
}

template <typename T, int D>
hipError_t launch_typed(const ewsjf_cache& c, const ewsjf_batch& b, int32_t layer, const void* q, int64_t q_token,
                        int64_t q_head, float scale, const void* plan, void* out, float* lse, void* ws,
                        hipStream_t stream) {
  const Shape s = shape_of(c, b);
  Args<T> a;
  a.data = static_cast<const T*>(c.data) + layer * c.layer_stride;
  a.q = static_cast<const T*>(q);
  a.q_token = q_token, a.q_head = q_head;
  a.table = c.table;
  a.out = static_cast<T*>(out);
  a.kv_stride = c.kv_stride, a.page_stride = c.page_stride, a.head_stride = c.head_stride;
  a.token_stride = c.token_stride;
  a.n_pages = c.n_pages, a.page_shift = __builtin_ctz(c.page_size), a.width = c.width, a.kv_heads = c.kv_heads;
  a.G = s.G, a.window = b.window, a.sinks = b.sinks;
  a.scale2 = scale * kLog2e;
  a.join = s.groups;
  a.plan = plan_of(s, const_cast<void*>(plan));
  a.work = work_of(c, b, s, ws);
  a.lse = lse != nullptr ? lse : a.work.lse;
  const bool sixteens = c.page_size >= 16;
  if (s.both) {
    auto kernel = sixteens ? attend_both<T, D, true> : attend_both<T, D, false>;
    kernel<<<s.blocks[0] + s.blocks[1], kWaves * 64, 0, stream>>>(a);
  }
  for (int p = s.groups ? 0 : 1; p < 2 && !s.both; ++p) {
    auto kernel = s.waves[p] == 8 ? (sixteens ? attend_block<T, D, 8, true> : attend_block<T, D, 8, false>)
                  : s.waves[p]    ? (sixteens ? attend_block<T, D, 4, true> : attend_block<T, D, 4, false>)
                  : s.whole && p  ? (sixteens ? attend_wave<T, D, true, true> : attend_wave<T, D, false, true>)
                                  : (sixteens ? attend_wave<T, D, true, false> : attend_wave<T, D, false, false>);
    kernel<<<s.blocks[p], 64 * (s.waves[p] ? s.waves[p] : kWaves), 0, stream>>>(a, p);
  }
  if (s.whole) return hipGetLastError();
  const int64_t most = (int64_t)b.max_q * s.G < s.rows[1] ? (int64_t)b.max_q * s.G : s.rows[1];
  const int fours = (int)((most + 3) / 4), flags = s.waves[1] ? s.waves[1] : 1;
  const int64_t waves = (a.join ? s.entries[1] : s.workers[1]) * fours;
  const unsigned grid = (unsigned)(waves < kMostJoins ? (waves + 3) / 4 : kMostJoins / 4);
  if (a.join) join_units<T, D><<<dim3(grid, c.kv_heads), 256, 0, stream>>>(a, s.rows[0], s.rows[1], flags, fours);
  else join_cuts<T, D><<<grid, 256, 0, stream>>>(a, s.rows[1], flags, fours);
  return hipGetLastError();
}

}  // namespace

size_t attention_plan_bytes(const ewsjf_cache& c, const ewsjf_batch& b) {
  return plan_of(shape_of(c, b), nullptr).bytes;
}
size_t attention_ws_bytes(const ewsjf_cache& c, const ewsjf_batch& b) {
  return work_of(c, b, shape_of(c, b), nullptr).bytes;
}

hipError_t launch_attention_plan(const ewsjf_cache& c, const ewsjf_batch& b, const int32_t* slot,
                                 const int32_t* q_start, const int32_t* group_start, const int32_t* shared,
                                 void* plan, hipStream_t stream) {
  const Shape s = shape_of(c, b);
  PlanArgs a{slot, q_start, group_start, shared, {s.rows[0], s.rows[1]}, {s.keys[0], s.keys[1]},
             {s.workers[0], s.workers[1]}, s.G, s.columns, s.whole};
  ewsjf_batch batch = b;
  if (!s.groups) batch.n_groups = 0;
  make_plan<<<1, kPlanThreads, 0, stream>>>(c, batch, a, plan_of(s, plan));
  return hipGetLastError();
}

hipError_t launch_attention(const ewsjf_cache& c, const ewsjf_batch& b, int32_t layer, const void* q, int64_t q_token,
                            int64_t q_head, float scale, const void* plan, void* out, float* lse, void* ws,
                            hipStream_t stream) {
  if (b.total_q == 0) return hipSuccess;
  auto go = [&](auto run) { return run(c, b, layer, q, q_token, q_head, scale, plan, out, lse, ws, stream); };
  if (c.dtype == EWSJF_BF16) return c.head_dim == 64 ? go(launch_typed<__bf16, 64>) : go(launch_typed<__bf16, 128>);
  return c.head_dim == 64 ? go(launch_typed<_Float16, 64>) : go(launch_typed<_Float16, 128>);
}

}  // namespace ewsjf
