// Pages of the key/value cache: taken, forked, released, copied, compacted,
// written.  Free pages are those with refs == 0; they are ranked by page
// number with prefix sums, so which page a request gets follows from the
// state alone and not from the order in which workgroups run.
//
// Books are a few KiB, so those kernels take as long as a launch and a few
// dependent loads do; only the pages' contents count against memory, 4.8 TB/s
// read and written in a large copy here.
#include <hip/hip_runtime.h>

#include "ewsjf_cache.h"

namespace ewsjf {
namespace {

constexpr int kThreads = 256;
// Pages ranked by one workgroup.  More take longer, fewer leave more sums to add:
// a compaction of 4096 pages 220 us, with 4096 a workgroup 232, with 256 218; an
// extend and a release in 2^20 pages 14.1 us against 13.8 and 27.0.
constexpr int kChunk = 1024;
constexpr int kMaxReq = EWSJF_MAX_CACHE_BATCH;
// Pools that one workgroup ranks, in one launch for two: an extend and a release
// of 8 slots take 10.2 us against 12.1 with 1024 pages, 14.5 against 12.0 with
// 8192; of 1024 slots, 15.2 against 18.7 with 4096.
constexpr int kSmallPool = 4096;
constexpr int kSmallThreads = 1024;
constexpr int kMostGrid = 65536;  // workgroups that copy pages of one plane: a launch has below 2^32 threads
// Requests whose rows it writes too, a wave each at once: 8 of them 10.2 us, in a
// launch of their own 11.5; 64 of them 13.9 against 11.6.
constexpr int kFewRequests = kSmallThreads / 64;

// Workspace: counts of the chunks, the requests' running needs, the pages
// picked for them; for a compaction the two ends of each move and, per moved
// page, the move's number.
struct CacheWs {
  int32_t* head;    // [4]: 0 free pages in all, 1 moves
  int32_t* counts;  // [chunks]
  int32_t* cum;     // [kMaxReq + 1]: pages needed by requests 0 .. i
  int32_t* fine;    // [kMaxReq]: 1 for a request that is valid by itself
  int32_t* picked;  // [n_pages]: picked free pages; a compaction's move targets
  int32_t* movers;  // [n_pages]: a compaction's move sources
  int32_t* number;  // [n_pages]: the move of a moved page
  size_t bytes;
};

CacheWs cache_ws(const ewsjf_cache& c, void* base) {
  CacheWs w;
  char* p = static_cast<char*>(base);
  size_t at = 0;
  auto take = [&](size_t ints) {
    int32_t* r = reinterpret_cast<int32_t*>(p + at);
    at += (ints * 4 + 255) & ~size_t(255);
    return r;
  };
  const size_t chunks = (c.n_pages + kChunk - 1) / kChunk;
  w.head = take(4);
  w.counts = take(chunks);
  w.cum = take(kMaxReq + 1);
  w.fine = take(kMaxReq);
  w.picked = take(c.n_pages);
  w.movers = take(c.n_pages);
  w.number = take(c.n_pages);
  w.bytes = at;
  return w;
}

__device__ int wave_scan(int v) {  // inclusive over the 64 lanes
  const int lane = threadIdx.x & 63;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// Exclusive prefix sum over the workgroup; total gets the sum.  A wave's sum
// has to fit 32 bits.
template <int kThreads = ewsjf::kThreads, typename N>
__device__ N block_scan(int v, N* sums, N& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int inc = wave_scan(v);
  __syncthreads();
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  N base = 0, all = 0;
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < wave) base += sums[i];
    all += sums[i];
  }
  total = all;
  return base + inc - v;
}

__device__ bool in_pool(const ewsjf_cache& c, int page) { return page >= 0 && page < c.n_pages; }
__device__ int pages_of(const ewsjf_cache& c, int64_t tokens) {
  return (int)((tokens + c.page_size - 1) / c.page_size);
}
__device__ int held(const ewsjf_cache& c, int slot) {
  const int n = c.length[slot];
  return n < 0 ? 0 : n;
}

// Checks the requests and sums what they need, in 64 bits: requests of up to
// 2^24 pages each pass 32 bits together.
template <int N>
__device__ void sum_needs(const ewsjf_cache& c, const CacheWs& w, int64_t* sums, const int32_t* parent,
                          const int32_t* slot, const int32_t* tokens, int n) {
  int64_t run = 0;
  for (int i0 = 0; i0 < n; i0 += N) {
    const int i = i0 + threadIdx.x;
    int need = 0, ok = 0;
    if (i < n) {
      const int s = slot[i];
      const int64_t t = tokens[i];
      if (s >= 0 && s < c.n_slots && t >= 0) {
        if (parent != nullptr) {
          const int p = parent[i];
          if (p >= 0 && p < c.n_slots && p != s && held(c, s) == 0 && t <= held(c, p) &&
              t <= (int64_t)c.width * c.page_size) {
            ok = 1;
            const int full = (int)(t / c.page_size);
            if (t % c.page_size) need = in_pool(c, c.table[(int64_t)p * c.width + full]);
          }
        } else {
          const int64_t have = held(c, s);
          if (have + t <= (int64_t)c.width * c.page_size) {
            ok = 1;
            need = pages_of(c, have + t) - pages_of(c, have);
          }
        }
      }
    }
    if (need > c.n_pages) need = c.n_pages + 1;
    int64_t total;
    const int64_t after = run + block_scan<N>(need, sums, total) + need;
    if (i < n) {
      w.cum[i] = after <= c.n_pages ? (int)after : c.n_pages + 1;  // more than are free
      w.fine[i] = ok;
    }
    run += total;
  }
}

// Workgroups 0 .. chunks - 1 count their chunk's free (or used) pages; the
// last one checks the requests and sums what they need.
__global__ __launch_bounds__(kThreads) void count_pages(ewsjf_cache c, CacheWs w, int chunks, bool used,
                                                        const int32_t* parent, const int32_t* slot,
                                                        const int32_t* tokens, int n) {
  __shared__ int64_t sums[kThreads / 64];
  if ((int)blockIdx.x < chunks) {
    int mine = 0;
    const int64_t base = (int64_t)blockIdx.x * kChunk;
    for (int i = threadIdx.x; i < kChunk; i += kThreads)
      if (base + i < c.n_pages) mine += (c.refs[base + i] != 0) == used;
    int64_t total;
    block_scan(mine, sums, total);
    if (threadIdx.x == 0) w.counts[blockIdx.x] = (int)total;
    return;
  }
  sum_needs<kThreads>(c, w, sums, parent, slot, tokens, n);
}

// Chunk sums before this workgroup's and in all.
__device__ void chunk_base(const int32_t* counts, int chunks, int* sums, int& base, int& all) {
  int before = 0, every = 0;
  for (int i = threadIdx.x; i < chunks; i += kThreads) {
    const int v = counts[i];
    every += v;
    if (i < (int)blockIdx.x) before += v;
  }
  block_scan(before, sums, base);
  block_scan(every, sums, all);
}

// Gives the lowest free pages to the granted needs.
__global__ __launch_bounds__(kThreads) void pick_pages(ewsjf_cache c, CacheWs w, int chunks, int n) {
  __shared__ int sums[kThreads / 64];
  __shared__ int top;
  int base, free;
  chunk_base(w.counts, chunks, sums, base, free);
  if (threadIdx.x == 0) top = 0;
  __syncthreads();
  int mine = 0;
  for (int i = threadIdx.x; i < n; i += kThreads)
    if (w.cum[i] <= free) mine = w.cum[i] > mine ? w.cum[i] : mine;
  atomicMax(&top, mine);
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) w.head[0] = free;
  const int64_t from = (int64_t)blockIdx.x * kChunk;
  for (int i0 = 0; i0 < kChunk && base < top; i0 += kThreads) {
    const int64_t p = from + i0 + threadIdx.x;
    const int is = p < c.n_pages && c.refs[p] == 0;
    int total;
    const int rank = base + block_scan(is, sums, total);
    if (is && rank < top) {
      w.picked[rank] = (int)p;
      c.refs[p] = 1;
    }
    base += total;
  }
}

// Writes request i's grant and row, and a fork's length, with threads `at`, `at`
// + step, ..; true if it is granted.  For new tokens the caller writes the
// length (grown), once all threads have read it.
__device__ bool write_row(const ewsjf_cache& c, const CacheWs& w, int free, const int32_t* parent, const int32_t* slot,
                          const int32_t* tokens, int32_t* granted, int i, int at, int step) {
  const int after = w.cum[i], first = i ? w.cum[i - 1] : 0;
  const bool ok = w.fine[i] && after <= free;
  if (at == 0) granted[i] = ok;
  if (!ok) return false;
  const int s = slot[i], t = tokens[i];
  int32_t* row = c.table + (int64_t)s * c.width;
  if (parent == nullptr) {
    const int64_t have = held(c, s);
    const int from = pages_of(c, have);
    for (int j = at; j < after - first && from + j < c.width; j += step) row[from + j] = w.picked[first + j];
    return true;
  }
  const int32_t* from = c.table + (int64_t)parent[i] * c.width;
  const int full = t / c.page_size;
  for (int j = at; j < full; j += step) {
    const int p = from[j];
    row[j] = p;
    if (in_pool(c, p)) atomicAdd(&c.refs[p], 1);
  }
  if (at == 0) {
    if (t % c.page_size) row[full] = after > first ? w.picked[first] : -1;
    c.length[s] = t;
  }
  return true;
}

__device__ void grown(const ewsjf_cache& c, int slot, int tokens) { c.length[slot] = held(c, slot) + tokens; }

// Request blockIdx.x: plane 0's workgroup writes its row, length and grant; for
// a fork each plane's (layer and keys or values) copies the partial page, 16
// bytes a thread at a time.  512 forks that each copy a page of 8 layers (512
// KiB): 78 to 94 us, 5.7 to 6.8 TB/s with parents' pages read from cache; one workgroup a
// page and plane is 8192 of them, enough to fill the chip without a division of
// the page.
__global__ __launch_bounds__(kThreads) void apply_growth(ewsjf_cache c, CacheWs w, const int32_t* parent,
                                                         const int32_t* slot, const int32_t* tokens,
                                                         int32_t* granted) {
  const int i = blockIdx.x, plane = blockIdx.y, free = w.head[0];
  if (plane == 0 && !write_row(c, w, free, parent, slot, tokens, granted, i, threadIdx.x, kThreads)) return;
  if (parent == nullptr) {
    __syncthreads();
    if (threadIdx.x == 0) grown(c, slot[i], tokens[i]);
    return;
  }
  const int after = w.cum[i], first = i ? w.cum[i - 1] : 0;
  if (!w.fine[i] || after > free || after == first) return;
  const int src = c.table[(int64_t)parent[i] * c.width + tokens[i] / c.page_size];
  if (!in_pool(c, src)) return;
  uint16_t* data = static_cast<uint16_t*>(c.data) + plane / 2 * c.layer_stride + plane % 2 * c.kv_stride;
  const uint4* a = reinterpret_cast<const uint4*>(data + src * c.page_stride);
  uint4* b = reinterpret_cast<uint4*>(data + w.picked[first] * c.page_stride);
  const int vecs = c.kv_heads * c.page_size * c.head_dim / 8;
  for (int j = threadIdx.x; j < vecs; j += kThreads) b[j] = a[j];
}

// count_pages and pick_pages of a small pool; for few requests of new tokens
// their rows too.
__global__ __launch_bounds__(kSmallThreads) void grow_small(ewsjf_cache c, CacheWs w, const int32_t* parent,
                                                            const int32_t* slot, const int32_t* tokens, int n,
                                                            int32_t* granted, bool rows) {
  __shared__ int64_t needs[kSmallThreads / 64];
  __shared__ int sums[kSmallThreads / 64];
  __shared__ int top;
  sum_needs<kSmallThreads>(c, w, needs, parent, slot, tokens, n);
  // a thread's pages lie together: one scan ranks them all
  const int each = (c.n_pages + kSmallThreads - 1) / kSmallThreads;
  const int64_t from = (int64_t)threadIdx.x * each, end = from + each < c.n_pages ? from + each : c.n_pages;
  int mine = 0;
  for (int64_t p = from; p < end; ++p) mine += c.refs[p] == 0;
  int free;
  int rank = block_scan<kSmallThreads>(mine, sums, free);
  if (threadIdx.x == 0) top = 0;
  __syncthreads();
  int most = 0;
  for (int i = threadIdx.x; i < n; i += kSmallThreads)
    if (w.cum[i] <= free) most = w.cum[i] > most ? w.cum[i] : most;
  atomicMax(&top, most);
  __syncthreads();
  for (int64_t p = from; p < end && rank < top; ++p)
    if (c.refs[p] == 0) {
      w.picked[rank++] = (int)p;
      c.refs[p] = 1;
    }
  if (threadIdx.x == 0) w.head[0] = free;
  if (!rows) return;
  __syncthreads();
  for (int i0 = 0; i0 < n; i0 += kSmallThreads / 64) {  // a wave a request
    const int i = i0 + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (i < n && write_row(c, w, free, parent, slot, tokens, granted, i, lane, 64)) {
      __builtin_amdgcn_wave_barrier();
      if (lane == 0) grown(c, slot[i], tokens[i]);
    }
  }
}

// A workgroup a slot.  Counts are integers, so the order of the atomics does
// not matter.
__global__ __launch_bounds__(kThreads) void release_rows(ewsjf_cache c, const int32_t* slot, const int32_t* begin,
                                                         const int32_t* end) {
  const int s = slot[blockIdx.x];
  if (s < 0 || s >= c.n_slots) return;
  int first = 0, last = c.width;
  if (begin != nullptr) {
    const int64_t b = begin[blockIdx.x] < 0 ? 0 : begin[blockIdx.x];
    int64_t e = end[blockIdx.x];
    const int64_t have = held(c, s);
    if (e > have) e = have;
    const int64_t lo = pages_of(c, b), hi = e < 0 ? 0 : e / c.page_size;
    first = (int)lo;
    last = hi > c.width ? c.width : (int)hi;
  }
  int32_t* row = c.table + (int64_t)s * c.width;
  for (int j = first + threadIdx.x; j < last; j += kThreads) {
    const int p = row[j];
    if (in_pool(c, p)) atomicSub(&c.refs[p], 1);
    row[j] = -1;
  }
  if (begin == nullptr && threadIdx.x == 0) c.length[s] = 0;
}

// A workgroup a page and plane.
__global__ __launch_bounds__(kThreads) void copy_pages(ewsjf_cache c, const int32_t* src, const int32_t* dst, int n) {
  const int plane = blockIdx.y;
  uint16_t* data = static_cast<uint16_t*>(c.data) + plane / 2 * c.layer_stride + plane % 2 * c.kv_stride;
  const int vecs = c.kv_heads * c.page_size * c.head_dim / 8;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int a = src[i], b = dst[i];
    if (!in_pool(c, a) || !in_pool(c, b)) continue;
    const uint4* from = reinterpret_cast<const uint4*>(data + a * c.page_stride);
    uint4* to = reinterpret_cast<uint4*>(data + b * c.page_stride);
    for (int j = threadIdx.x; j < vecs; j += kThreads) to[j] = from[j];
  }
}

// The moves of a compaction.  With U used pages and before(p) used pages below
// p: the hole p < U is the target of move p - before(p), the used page p >= U
// the source of move U - 1 - before(p).
__global__ __launch_bounds__(kThreads) void list_moves(ewsjf_cache c, CacheWs w, int chunks, int32_t* used) {
  __shared__ int sums[kThreads / 64];
  int base, U;
  chunk_base(w.counts, chunks, sums, base, U);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *used = U;
    if (U == 0) w.head[1] = 0;
  }
  const int64_t from = (int64_t)blockIdx.x * kChunk;
  for (int i0 = 0; i0 < kChunk; i0 += kThreads) {
    const int64_t p = from + i0 + threadIdx.x;
    const int is = p < c.n_pages && c.refs[p] != 0;
    int total;
    const int before = base + block_scan(is, sums, total);
    if (p < U && !is) w.picked[p - before] = (int)p;
    if (p >= U && p < c.n_pages) {
      if (is) w.movers[U - 1 - before] = (int)p;
      w.number[p] = is ? U - 1 - before : -1;
    }
    if (p == U - 1) w.head[1] = U - before - is;
    base += total;
  }
}

// The first `book` workgroups write rows and counts, the others take the moved
// pages' planes in turn.  A target lies below U and a source at or above it, so
// no page is both.  Bound by memory: 983 pages of 512 KiB, read and written, 210
// us, 4.9 TB/s, what a large copy reaches.
__global__ __launch_bounds__(kThreads) void move_pages(ewsjf_cache c, CacheWs w, int32_t* out_table,
                                                       int32_t* out_refs, const int32_t* used, int book) {
  const int moves = w.head[1], U = *used;
  if ((int)blockIdx.x < book) {  // rows and counts
    const int64_t step = (int64_t)book * kThreads, at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t entries = (int64_t)c.n_slots * c.width;
    for (int64_t i = at; i < entries; i += step) {
      int p = c.table[i];
      if (in_pool(c, p) && p >= U) p = w.number[p] >= 0 ? w.picked[w.number[p]] : -1;
      out_table[i] = p;
    }
    for (int64_t p = at; p < c.n_pages; p += step) {
      const int r = c.refs[p];
      if (p < U) {
        if (r != 0) out_refs[p] = r;  // a hole's count is written with its move
      } else {
        if (r != 0) out_refs[w.picked[w.number[p]]] = r;
        out_refs[p] = 0;
      }
    }
    return;
  }
  const int planes = 2 * c.layers, vecs = c.kv_heads * c.page_size * c.head_dim / 8;
  const int64_t tasks = (int64_t)moves * planes;
  for (int64_t i = blockIdx.x - book; i < tasks; i += gridDim.x - book) {
    const int j = (int)(i / planes), plane = (int)(i % planes);
    uint16_t* data = static_cast<uint16_t*>(c.data) + plane / 2 * c.layer_stride + plane % 2 * c.kv_stride;
    const uint4* a = reinterpret_cast<const uint4*>(data + w.movers[j] * c.page_stride);
    uint4* b = reinterpret_cast<uint4*>(data + w.picked[j] * c.page_stride);
    for (int v = threadIdx.x; v < vecs; v += kThreads) b[v] = a[v];
  }
}

// One workgroup a token: its heads' keys and values into the slot's page.  3 us
// for 8 tokens, a launch; the search for the sequence is its longest part.
// 16,384 tokens of 8 heads of 128: 22 us, 6.1 TB/s read and written; with
// divisions by the page size in place of shifts 24.4.
// Without grants a request may be one that found no room: its tokens would then
// land on tokens that it holds already.  A partial page is the slot's own, a
// whole one may be others' too, and two requests could write it at once; so a
// whole page is written only if this row alone has it.
__global__ __launch_bounds__(kThreads) void append_tokens(ewsjf_cache c, int layer, const uint16_t* k,
                                                          const uint16_t* v, int64_t k_token, int64_t k_head,
                                                          int64_t v_token, int64_t v_head, const int32_t* slot,
                                                          const int32_t* q_start, const int32_t* granted,
                                                          int n_seqs) {
  const int64_t t = blockIdx.x;
  int lo = 0, hi = n_seqs;  // the last s with q_start[s] <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (q_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int s = slot[lo];
  const int a = q_start[lo], e = q_start[lo + 1];
  if (s < 0 || s >= c.n_slots || t < a || t >= e || (granted != nullptr && granted[lo] == 0)) return;
  const int shift = __builtin_ctz(c.page_size);
  const int have = held(c, s), pos = have - (int)(e - t);
  if (pos < 0 || pos >> shift >= c.width) return;
  const int page = c.table[(int64_t)s * c.width + (pos >> shift)];
  if (!in_pool(c, page)) return;
  if (granted == nullptr && pos >> shift < have >> shift && c.refs[page] > 1) return;
  uint16_t* to = static_cast<uint16_t*>(c.data) + layer * c.layer_stride + page * c.page_stride +
                 (pos & (c.page_size - 1)) * c.token_stride;
  const int dv = c.head_dim / 8, vecs = c.kv_heads * dv;
  for (int i = threadIdx.x; i < 2 * vecs; i += kThreads) {
    const int x = i >= vecs, j = i - x * vecs, h = j / dv, d = j % dv * 8;
    const uint16_t* from = x ? v + t * v_token + h * v_head + d : k + t * k_token + h * k_head + d;
    *reinterpret_cast<uint4*>(to + x * c.kv_stride + h * c.head_stride + d) = *reinterpret_cast<const uint4*>(from);
  }
}

}  // namespace

size_t cache_ws_bytes(const ewsjf_cache& c) { return cache_ws(c, nullptr).bytes; }

hipError_t launch_cache_grow(const ewsjf_cache& c, const int32_t* parent, const int32_t* slot, const int32_t* tokens,
                             int32_t n, int32_t* granted, void* ws, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const CacheWs w = cache_ws(c, ws);
  const int chunks = (c.n_pages + kChunk - 1) / kChunk;
  if (c.n_pages <= kSmallPool) {
    const bool rows = parent == nullptr && n <= kFewRequests;
    grow_small<<<1, kSmallThreads, 0, stream>>>(c, w, parent, slot, tokens, n, granted, rows);
    if (rows) return hipGetLastError();
  } else {
    count_pages<<<chunks + 1, kThreads, 0, stream>>>(c, w, chunks, false, parent, slot, tokens, n);
    pick_pages<<<chunks, kThreads, 0, stream>>>(c, w, chunks, n);
  }
  apply_growth<<<dim3(n, parent ? 2 * c.layers : 1), kThreads, 0, stream>>>(c, w, parent, slot, tokens, granted);
  return hipGetLastError();
}

hipError_t launch_cache_release(const ewsjf_cache& c, const int32_t* slot, const int32_t* begin, const int32_t* end,
                                int32_t n, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  release_rows<<<n, kThreads, 0, stream>>>(c, slot, begin, end);
  return hipGetLastError();
}

hipError_t launch_cache_copy(const ewsjf_cache& c, const int32_t* src, const int32_t* dst, int32_t n,
                             hipStream_t stream) {
  if (n == 0) return hipSuccess;
  copy_pages<<<dim3(n < kMostGrid ? n : kMostGrid, 2 * c.layers), kThreads, 0, stream>>>(c, src, dst, n);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const ewsjf_cache& c, int32_t* out_table, int32_t* out_refs, int32_t* used, void* ws,
                                hipStream_t stream) {
  const CacheWs w = cache_ws(c, ws);
  const int chunks = (c.n_pages + kChunk - 1) / kChunk;
  count_pages<<<chunks, kThreads, 0, stream>>>(c, w, chunks, true, nullptr, nullptr, nullptr, 0);
  list_moves<<<chunks, kThreads, 0, stream>>>(c, w, chunks, used);
  const int book = 128;
  move_pages<<<book + 2048, kThreads, 0, stream>>>(c, w, out_table, out_refs, used, book);
  return hipGetLastError();
}

hipError_t launch_cache_append(const ewsjf_cache& c, int32_t layer, const void* k, const void* v, int64_t k_token,
                               int64_t k_head, int64_t v_token, int64_t v_head, const int32_t* slot,
                               const int32_t* q_start, const int32_t* granted, int32_t n_seqs, int64_t total,
                               hipStream_t stream) {
  if (n_seqs == 0 || total == 0) return hipSuccess;
  append_tokens<<<(unsigned)total, kThreads, 0, stream>>>(
      c, layer, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_token, k_head, v_token, v_head,
      slot, q_start, granted, n_seqs);
  return hipGetLastError();
}

}  // namespace ewsjf
