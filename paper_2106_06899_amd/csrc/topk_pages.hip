// A cache in pages: keys and values of requests lie in pages of page_rows rows of a common pool, and a
// table says which pages hold a request's rows, in order. refs[p] counts the table entries that hold page
// p; a page with 0 is free. That array and the tables are the whole state: a call that needs pages takes
// the free ones of the lowest numbers, in the order of requests and rows, so that results do not
// depend on scheduling, and nothing is kept between calls.
//
// The books (tables, counts) are a few kilobytes and bound by latency: one workgroup decides who gets
// which page, with prefix sums over requests and over the counts. Rows of keys and values move in a
// launch of their own, by many workgroups, in 16-byte pieces, and are bound by memory.
#include "topk_device.h"
#include "topk_pages.h"

#include <limits.h>

#include <algorithm>

namespace topk {
namespace {

constexpr int BOOK = 1024;       // threads of a workgroup on the books
constexpr int NT = 256;          // on rows
constexpr int PIECES = 8 * NT;   // 16-byte pieces that a workgroup copies at a time
constexpr int FREE_BLOCK = 4096; // pages of a block whose free ones are listed
constexpr int FREE_DIRECT = 4 * FREE_BLOCK;  // pages of a pool that a reservation looks through by itself

int64_t cdiv(int64_t x, int64_t y) { return (x + y - 1) / y; }
size_t up(size_t x) { return (x + 255) / 256 * 256; }

// (counts change by atomics, which pass the vector cache by; so do these reads)
__device__ __forceinline__ int count_of(const int32_t* refs, int p) { return __hip_atomic_load(refs + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void count_add(int32_t* refs, int p, int by) {
  __hip_atomic_fetch_add(refs + p, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Every access of the workgroup before this is done, and seen by all of it behind: they share one vector cache,
// which stores write through, and atomics are done where they are acknowledged. (A fence for the whole GPU would
// write its caches back: a reservation took 27 us with one at every step, 8.7 without.)
__device__ __forceinline__ void book_sync() {
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));  // no vector-memory operation outstanding
  __syncthreads();
}

// Inclusive prefix sum over the workgroup; *total: of all. `sums`: one entry a wave.
__device__ __forceinline__ uint32_t book_scan(uint32_t x, uint32_t* sums, uint32_t* total) {
  const int wave = threadIdx.x >> 6;
  x = wave_incl_scan_full(x);
  if ((threadIdx.x & 63) == 63) sums[wave] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < BOOK / 64; ++w) {
    const uint32_t s = sums[w];
    before += w < wave ? s : 0;
    all += s;
  }
  __syncthreads();
  *total = all;
  return before + x;
}

// What becomes of an entry: it stays; it takes a free page; it is one of several that hold its page and is
// to leave it for a copy.
enum { STAYS = 0, FRESH = 1, SHARED = 2, LEAVES = 3, KEEPS = 4 };

// The entries of the rows [lengths[b], lengths[b] + rows) of each request, in the order of requests: the workgroup
// takes BOOK requests at a time, each adding its entries to one list. Where that is one list of at most BOOK
// entries, each thread has one and keeps it, otherwise their kinds lie in memory.
struct Entries {
  const ReserveArgs& a;
  uint32_t *ends, *sums;
  int32_t* firsts;
  uint32_t total;
  bool one;
  int b, e, page, kind, left;  // one: request (-1: none), entry, its page, what becomes of it, rows in use behind its start

  __device__ void load(int base) {
    const int r = base + threadIdx.x;
    int64_t n = 0, first = 0;
    if (r < a.t.B) {
      const int64_t len = a.lengths[r], rows = a.rows_each ? a.rows_each[r] : a.rows;
      if (len >= 0 && rows > 0) {
        first = min(len / a.s.page_rows, (int64_t)a.t.M);
        n = min((len + rows + a.s.page_rows - 1) / a.s.page_rows, (int64_t)a.t.M) - first;
      }
    }
    __syncthreads();
    ends[threadIdx.x] = book_scan((uint32_t)n, sums, &total);
    firsts[threadIdx.x] = (int32_t)first;
    __syncthreads();
  }
  __device__ void find(uint32_t i, int base, int* to_b, int* to_e) const {
    int lo = 0, hi = BOOK - 1;  // the first request whose entries end behind i
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (ends[mid] > i) hi = mid;
      else lo = mid + 1;
    }
    *to_b = base + lo;
    *to_e = firsts[lo] + (int)(i - (lo ? ends[lo - 1] : 0));
  }
  __device__ void begin() {
    one = false;
    if (a.t.B > BOOK) return;
    load(0);
    one = total <= BOOK;
    b = -1;
    if (one && threadIdx.x < total) {
      find(threadIdx.x, 0, &b, &e);
      page = a.t.at[b * a.t.stride + e];
      left = a.lengths[b] - e * a.s.page_rows;
    }
  }
  // f(is there one, its number, its page, its kind to be read and changed, ...), by the whole workgroup
  template <typename F>
  __device__ void each(F f) {
    if (one) {
      f(b >= 0, (int)((int64_t)b * a.t.M + e), b, e, page, &kind, left);
      return;
    }
    for (int base = 0; base < a.t.B; base += BOOK) {
      if (a.t.B > BOOK) load(base);
      for (uint32_t i0 = 0; i0 < total; i0 += BOOK) {
        const bool ok = i0 + threadIdx.x < total;
        int fb = 0, fe = 0, k = STAYS, p = -1;
        int64_t number = 0;
        if (ok) {
          find(i0 + threadIdx.x, base, &fb, &fe);
          number = (int64_t)fb * a.t.M + fe;
          p = a.t.at[fb * a.t.stride + fe];
          k = a.kind[number];
        }
        const int was = k;
        f(ok, (int)number, fb, fe, p, &k, ok ? a.lengths[fb] - fe * a.s.page_rows : 0);
        if (ok && k != was) a.kind[number] = k;
      }
    }
  }
};

// The free pages of each block of a large pool. (A workgroup alone looks through 4096 pages in 1.6 us, a pool of a
// million in 390 us; listed by one workgroup a block it takes 17.)
__global__ __launch_bounds__(BOOK) void k_pages_free(ReserveArgs a) {
  __shared__ uint32_t sums[BOOK / 64];
  const int64_t base = (int64_t)blockIdx.x * FREE_BLOCK + 4 * threadIdx.x;
  bool free[4];
  uint32_t c = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) c += free[u] = base + u < a.s.n_pages && a.refs[base + u] == 0;
  uint32_t n, at = book_scan(c, sums, &n) - c;
  int32_t* list = a.listed + gridDim.x + (int64_t)blockIdx.x * FREE_BLOCK;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (free[u]) list[at++] = (int)(base + u);
  if (threadIdx.x == 0) a.listed[blockIdx.x] = (int)n;
}

// One workgroup: kinds of the entries, those who leave a shared page, free pages, the new books. Bound by the latency
// of these steps, one behind the other: 64 requests that write to pages shared by 8 beams 9.6 us,
// 32 with 16 new rows each 6.6.
__global__ __launch_bounds__(BOOK) void k_pages_reserve(ReserveArgs a) {
  __shared__ uint32_t ends[BOOK], sums[BOOK / 64], blocks[BOOK];
  __shared__ int32_t firsts[BOOK], found[BOOK];
  __shared__ int any_shared;
  const int tid = threadIdx.x, n_pages = (int)a.s.n_pages;
  Entries en = {a, ends, sums, firsts};
  if (tid == 0) any_shared = 0;
  en.begin();
  __syncthreads();
  uint32_t need = 0;
  en.each([&](bool ok, int, int, int, int p, int* k, int) {
    *k = -1;  // (whatever is in memory is written over)
    if (ok) {
      *k = (uint32_t)p >= (uint32_t)n_pages ? FRESH : count_of(a.refs, p) > 1 ? SHARED : STAYS;
      if (*k == SHARED) any_shared = 1;
    }
    uint32_t n;
    book_scan(*k == FRESH, sums, &n);
    need += n;
  });
  book_sync();
  const bool shared = any_shared;
  if (shared) {
    // Those that leave a page take themselves off its count. Where that leaves nobody, the first (in the order
    // of requests) stays: it is found as the smallest of their numbers, written into the count itself as a
    // negative one.
    en.each([&](bool ok, int, int, int, int p, int* k, int) {
      if (ok && *k == SHARED) count_add(a.refs, p, -1);
    });
    book_sync();
    en.each([&](bool ok, int number, int, int, int p, int* k, int) {
      if (ok && *k == SHARED && count_of(a.refs, p) <= 0)
        __hip_atomic_fetch_min(a.refs + p, INT_MIN + number, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    book_sync();
    en.each([&](bool ok, int number, int, int, int p, int* k, int) {
      if (ok && *k == SHARED) *k = count_of(a.refs, p) == INT_MIN + number ? KEEPS : LEAVES;
      uint32_t n;
      book_scan(ok && *k == LEAVES, sums, &n);
      need += n;
    });
    book_sync();
    en.each([&](bool ok, int, int, int, int p, int* k, int) {  // (a page that its first keeps: 1)
      if (ok && *k == KEEPS) a.refs[p] = 1;
    });
    book_sync();
  }
  // the free pages of the lowest numbers, as many as are needed
  const bool few = need <= BOOK;
  uint32_t have = 0;
  const int n_blocks = (int)(((int64_t)n_pages + FREE_BLOCK - 1) / FREE_BLOCK);
  for (int base = 0; a.listed && base < n_blocks && have < need; base += BOOK) {
    uint32_t n;
    blocks[tid] = book_scan(base + tid < n_blocks ? (uint32_t)a.listed[base + tid] : 0u, sums, &n);
    __syncthreads();
    for (uint32_t i = tid; i < n && have + i < need; i += BOOK) {
      int lo = 0, hi = BOOK - 1;  // the first block whose pages end behind i
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (blocks[mid] > i) hi = mid;
        else lo = mid + 1;
      }
      const int p = a.listed[n_blocks + (int64_t)(base + lo) * FREE_BLOCK + (i - (lo ? blocks[lo - 1] : 0))];
      if (few) found[have + i] = p;
      else a.free_list[have + i] = p;
    }
    have += n;
  }
  for (int64_t base = 0; !a.listed && base < n_pages && have < need; base += 4 * BOOK) {
    bool free[4];
    uint32_t c = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t p = base + 4 * tid + u;
      free[u] = p < n_pages && count_of(a.refs, (int)min(p, (int64_t)n_pages - 1)) == 0;
      c += free[u];
    }
    uint32_t n, at = have + book_scan(c, sums, &n) - c;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (free[u] && at < need) {
        if (few) found[at++] = (int)(base + 4 * tid + u);
        else a.free_list[at++] = (int)(base + 4 * tid + u);
      }
    have += n;
  }
  book_sync();
  if (have < need) {  // nothing is changed: those that left are counted again
    if (tid == 0) {
      *a.missing = (int)(need - have);
      a.copies[0].x = 0;
    }
    if (!shared) return;
    en.each([&](bool ok, int, int, int, int p, int* k, int) {
      if (ok && *k == KEEPS) a.refs[p] = 0;
    });
    book_sync();
    en.each([&](bool ok, int, int, int, int p, int* k, int) {
      if (ok && *k >= LEAVES) count_add(a.refs, p, 1);
    });
    return;
  }
  uint32_t taken = 0, copied = 0;
  en.each([&](bool ok, int, int b, int e, int p, int* k, int left) {
    const bool takes = ok && (*k == FRESH || *k == LEAVES);
    uint32_t n;
    const uint32_t at = taken + book_scan(takes, sums, &n) - 1;
    taken += n;
    const bool copies = takes && *k == LEAVES && left > 0;  // (`left` rows of the page are in use)
    uint32_t copy = 0;
    if (shared) {
      copy = copied + book_scan(copies, sums, &n);
      copied += n;
    }
    if (!takes) return;
    const int to = few ? found[at] : a.free_list[at];
    if (copies) a.copies[copy] = make_int4(p, to, left, 0);
    a.t.at[b * a.t.stride + e] = to;
    a.refs[to] = 1;
  });
  if (tid == 0) {
    *a.missing = 0;
    a.copies[0].x = (int)copied;
  }
}

__device__ __forceinline__ f32x4* piece_ptr(const PagePool& pool, int kv, int64_t layer, int64_t page, int64_t at, int es) {
  return (f32x4*)((char*)pool.p[kv] + (layer * pool.layer[kv] + page * pool.page[kv] + at) * es);
}

// Copies the first `rows` rows of every head of page `from` to page `to`, one part of PIECES pieces of them. Piece i is
// piece i % s.pieces of row i / s.pieces % rows of a head; FLAT: all of a page that lies in one piece in both pools.
template <bool FLAT>
__device__ __forceinline__ void copy_page(const PagePool& pa, const PagePool& pb, const PageShape& s, int kv, int layer, int part, int from,
                                          int to, int rows) {
  constexpr int U = PIECES / NT;
  const uint32_t total = (uint32_t)s.heads * rows * s.pieces, i0 = part * PIECES + threadIdx.x;
  if (part * PIECES >= total) return;
  const f32x4* src = piece_ptr(pa, kv, layer, from, 0, s.es);
  f32x4* dst = piece_ptr(pb, kv, layer, to, 0, s.es);
  const bool whole = (part + 1) * PIECES <= total;
  if (FLAT) {
    if (!whole) {
      for (uint32_t i = i0; i < total; i += NT) dst[i] = src[i];
      return;
    }
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = src[i0 + u * NT];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_nontemporal_store(x[u], dst + i0 + u * NT);
    return;
  }
  // the place of the first piece by division, of the others by steps of NT pieces
  const uint32_t step_c = NT % s.pieces, step_r = NT / s.pieces;
  uint32_t c = i0 % s.pieces, row = i0 / s.pieces % rows, head = i0 / s.pieces / rows;
  auto at = [&](const PagePool& p) { return (head * p.head[kv] + row * p.row[kv]) * s.es + c * 16; };
  auto step = [&]() {
    c += step_c;
    row += step_r;
    if (c >= (uint32_t)s.pieces) c -= s.pieces, ++row;
    if (row >= (uint32_t)rows) {
      head += row / rows;
      row %= rows;
    }
  };
  if (!whole) {
    for (uint32_t i = i0; i < total; i += NT, step()) *(f32x4*)((char*)dst + at(pb)) = *(const f32x4*)((const char*)src + at(pa));
    return;
  }
  f32x4 x[U];
  int64_t to_at[U];
#pragma unroll
  for (int u = 0; u < U; ++u, step()) {
    x[u] = *(const f32x4*)((const char*)src + at(pa));
    to_at[u] = at(pb);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) *(f32x4*)((char*)dst + to_at[u]) = x[u];
}

struct CopyPlace {
  int page, layer, part, kv;
};
// pieces of work of a page's copy in all layers
__device__ __forceinline__ uint32_t copy_parts(const PageShape& s) {
  return ((uint32_t)s.heads * s.page_rows * s.pieces + PIECES - 1) / PIECES * 2 * (uint32_t)s.layers;
}
// the page, layer, pool and part of piece i
__device__ __forceinline__ CopyPlace copy_place(const PageShape& s, uint32_t i) {
  const uint32_t parts = ((uint32_t)s.heads * s.page_rows * s.pieces + PIECES - 1) / PIECES, layers = (uint32_t)s.layers;
  CopyPlace c;
  c.part = (int)(i % parts);
  i /= parts;
  c.kv = (int)(i & 1);
  i >>= 1;
  c.layer = (int)(i % layers);
  c.page = (int)(i / layers);
  return c;
}

// The rows in use of the pages that were left, in all layers. (56 pages of two layers of 8 heads of 128: 4.8 us, a launch's
// latency and two rounds to memory.)
__global__ __launch_bounds__(NT) void k_pages_copy(ReserveArgs a) {
  const uint32_t all = (uint32_t)a.copies[0].x * copy_parts(a.s);
  for (uint64_t i = blockIdx.x; i < all; i += gridDim.x) {
    const CopyPlace c = copy_place(a.s, (uint32_t)i);
    const int4 x = a.copies[1 + c.page];
    copy_page<false>(a.pool, a.pool, a.s, c.kv, c.layer, c.part, x.x, x.y, x.z);
  }
}

// One token of one layer a workgroup: its keys and values to row lengths[b] + its place in the request. (64 tokens of
// two layers 3.4 us, 512 of four 6.9, of which the books' three look-ups one behind the other are most.)
__global__ __launch_bounds__(NT) void k_pages_append(AppendArgs a) {
  const uint32_t layers = (uint32_t)a.s.layers, layer = blockIdx.x % layers, i = blockIdx.x / layers;
  int64_t b, t, from;
  if (a.offsets) {  // the last request whose first token is not behind i
    int lo = 0, hi = a.t.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.offsets[mid] <= (int64_t)i) lo = mid;
      else hi = mid;
    }
    b = lo;
    t = (int64_t)i - a.offsets[b];
    if (t < 0 || (int64_t)i >= a.offsets[b + 1]) return;
    from = 0;
  } else {
    b = i / (uint32_t)a.T;
    t = i - b * a.T;
    from = b;
  }
  const int64_t len = a.lengths[b], r = len + t;
  if (len < 0 || r > INT_MAX) return;
  const int e = (int)r / a.s.page_rows;
  if (e >= a.t.M) return;
  const int p = a.t.at[b * a.t.stride + e];
  if ((uint32_t)p >= (uint32_t)a.s.n_pages) return;
  const int row = (int)r - e * a.s.page_rows, each = (int)a.s.heads * a.s.pieces;
  const int64_t token = a.offsets ? i : t;
  for (int x = threadIdx.x; x < 2 * each; x += NT) {
    const int kv = x >= each, y = x - kv * each, head = y / a.s.pieces, c = (y - head * a.s.pieces) * (16 / a.s.es);
    *piece_ptr(a.pool, kv, layer, p, head * a.pool.head[kv] + row * a.pool.row[kv] + c, a.s.es) =
        *piece_ptr(a.from, kv, layer, from, head * a.from.head[kv] + token * a.from.row[kv] + c, a.s.es);
  }
}

// Rows lengths[b] + kept[b][i] of one head, layer and pool go to rows lengths[b] + i: all of a slab of
// columns is read before any of it is written, so that the order of `kept` does not matter. (32 requests, four layers of 8
// heads of 128: 7.4 us, latency.)
__global__ __launch_bounds__(NT) void k_pages_keep(KeepArgs a) {
  __shared__ int2 from[KEEP_MAX], to[KEEP_MAX];  // page (-1: none), row
  __shared__ int count;
  uint32_t i = blockIdx.x;
  const uint32_t heads = (uint32_t)a.s.heads, layers = (uint32_t)a.s.layers;
  const int kv = (int)(i & 1);
  i >>= 1;
  const uint32_t head = i % heads, rest = i / heads, layer = rest % layers, b = rest / layers;
  const int64_t len = a.lengths[b];
  if (threadIdx.x < 64) {
    const int x = threadIdx.x < a.A ? a.kept[b * a.kept_stride + threadIdx.x] : -1;
    const uint64_t over = __builtin_amdgcn_ballot_w64(x < 0);
    const int n = len < 0 ? 0 : over ? __builtin_ctzll(over) : 64;
    if (threadIdx.x == 0) {
      count = n;
      if (!kv && !head && !layer) a.new_lengths[b] = (int32_t)(len + n);
    }
    auto place = [&](int64_t r) {
      const int e = r > INT_MAX ? INT_MAX : (int)r / a.s.page_rows;
      const int p = e < a.t.M ? a.t.at[b * a.t.stride + e] : -1;
      return make_int2((uint32_t)p < (uint32_t)a.s.n_pages ? p : -1, (int)r - e * a.s.page_rows);
    };
    if ((int)threadIdx.x < n) {
      int2 f = place(len + x);
      const int2 t = place(len + threadIdx.x);
      if (t.x < 0) f.x = -1;
      from[threadIdx.x] = f;
      to[threadIdx.x] = t;
    }
  }
  __syncthreads();
  constexpr int U = 4;
  const int n = count;
  if (!n) return;
  const int cols = min(a.s.pieces, U * NT / n);  // columns of a slab
  for (int c0 = 0; c0 < a.s.pieces; c0 += cols) {
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = threadIdx.x + u * NT, r = k / cols, c = c0 + k % cols;
      if (r < n && c < a.s.pieces && from[r].x >= 0)
        x[u] = *piece_ptr(a.pool, kv, layer, from[r].x, head * a.pool.head[kv] + from[r].y * a.pool.row[kv] + c * (16 / a.s.es), a.s.es);
    }
    __syncthreads();  // (waits for the loads, too)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = threadIdx.x + u * NT, r = k / cols, c = c0 + k % cols;
      if (r < n && c < a.s.pieces && from[r].x >= 0)
        *piece_ptr(a.pool, kv, layer, to[r].x, head * a.pool.head[kv] + to[r].y * a.pool.row[kv] + c * (16 / a.s.es), a.s.es) = x[u];
    }
  }
}

__device__ __forceinline__ int64_t pages_of(int64_t len, int rows) { return len <= 0 ? 0 : (len + rows - 1) / rows; }

// A request's new row of the table, and its old and new pages' counts. The tables change in a launch of
// their own, when nothing reads the old ones any more. (8 requests of 65536 entries 14 us for both.)
__global__ __launch_bounds__(NT) void k_pages_fork(ForkArgs a) {
  const int b = blockIdx.x;
  const int par = a.parents[b];
  if (par == b || par >= a.t.B) return;
  int32_t* tmp = a.tmp + (int64_t)b * (a.t.M + 1);
  const int len = par < 0 ? 0 : a.lengths[par];
  const int64_t n = pages_of(len, a.page_rows);
  for (int64_t e = blockIdx.y * NT + threadIdx.x; e < a.t.M; e += NT * gridDim.y) {
    const int old = a.t.at[b * a.t.stride + e];
    int p = par >= 0 && e < n ? a.t.at[par * a.t.stride + e] : -1;
    if ((uint32_t)p >= (uint32_t)a.n_pages) p = -1;
    if (old != p) {  // (beams share most of their pages)
      if ((uint32_t)old < (uint32_t)a.n_pages) count_add(a.refs, old, -1);
      if (p >= 0) count_add(a.refs, p, 1);
    }
    tmp[e] = p;
  }
  if (threadIdx.x == 0 && blockIdx.y == 0) tmp[a.t.M] = len;
}
__global__ __launch_bounds__(NT) void k_pages_forked(ForkArgs a) {
  const int b = blockIdx.x;
  const int par = a.parents[b];
  if (par == b || par >= a.t.B) return;
  const int32_t* tmp = a.tmp + (int64_t)b * (a.t.M + 1);
  for (int64_t e = blockIdx.y * NT + threadIdx.x; e < a.t.M; e += NT * gridDim.y) a.t.at[b * a.t.stride + e] = tmp[e];
  if (threadIdx.x == 0 && blockIdx.y == 0) a.lengths[b] = tmp[a.t.M];
}

// The same for tables of few entries, in one launch: one workgroup reads all of the old tables before it writes.
constexpr int FORK_FEW = 8192;
__global__ __launch_bounds__(BOOK) void k_pages_fork_few(ForkArgs a) {
  __shared__ int32_t old[FORK_FEW], lens[FORK_FEW];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, M = a.t.M;
  for (int b = wave; b < a.t.B; b += BOOK / 64)
    for (int e = lane; e < M; e += 64) old[b * M + e] = a.t.at[b * a.t.stride + e];
  for (int b = threadIdx.x; b < a.t.B; b += BOOK) lens[b] = a.lengths[b];
  __syncthreads();
  for (int b = wave; b < a.t.B; b += BOOK / 64) {
    const int par = a.parents[b];
    if (par == b || par >= a.t.B) continue;
    const int len = par < 0 ? 0 : lens[par];
    const int64_t n = pages_of(len, a.page_rows);
    for (int e = lane; e < M; e += 64) {
      const int was = old[b * M + e];
      int p = par >= 0 && e < n ? old[par * M + e] : -1;
      if ((uint32_t)p >= (uint32_t)a.n_pages) p = -1;
      if (was == p) continue;
      if ((uint32_t)was < (uint32_t)a.n_pages) count_add(a.refs, was, -1);
      if (p >= 0) count_add(a.refs, p, 1);
      a.t.at[b * a.t.stride + e] = p;
    }
    if (lane == 0) a.lengths[b] = len;
  }
}

__global__ __launch_bounds__(NT) void k_pages_release(PageTable t, int32_t* refs, const int32_t* lengths, int64_t n_pages, int page_rows) {
  const int b = blockIdx.x;
  for (int64_t e = pages_of(lengths[b], page_rows) + blockIdx.y * NT + threadIdx.x; e < t.M; e += NT * gridDim.y) {
    int32_t* at = t.at + b * t.stride + e;
    const int p = *at;
    if (p == -1) continue;
    if ((uint32_t)p < (uint32_t)n_pages) count_add(refs, p, -1);
    *at = -1;
  }
}

// The used pages' new numbers, in the order of their old ones, by one workgroup (5636 pages 6.8 us).
__global__ __launch_bounds__(BOOK) void k_pages_number(CompactArgs a) {
  __shared__ uint32_t sums[BOOK / 64];
  const int tid = threadIdx.x;
  const int64_t n_pages = a.s.n_pages;
  uint32_t have = 0;
  for (int64_t base = 0; base < n_pages; base += 4 * BOOK) {
    int r[4];
    uint32_t c = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t p = base + 4 * tid + u;
      r[u] = p < n_pages ? a.refs[p] : 0;
      c += r[u] > 0;
    }
    uint32_t n, at = have + book_scan(c, sums, &n) - c;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t p = base + 4 * tid + u;
      if (p < n_pages) a.number[p] = r[u] > 0 ? (int)at : -1;
      if (r[u] > 0) {
        if (at < a.n_to) {
          a.live[at] = (int)p;
          a.new_refs[at] = r[u];
        }
        ++at;
      }
    }
    have += n;
  }
  const bool fits = have <= a.n_to;
  if (tid == 0) {
    a.live[a.n_to] = fits ? (int)have : 0;
    *a.missing = fits ? 0 : (int)(have - a.n_to);
  }
  __syncthreads();
  for (int64_t p = (fits ? have : 0) + tid; p < a.n_to; p += BOOK) a.new_refs[p] = 0;
}
// The new table, and the pages: 32 KiB a workgroup at a time, loads before stores, stores past the cache. Bound by memory:
// 810 MB read and written in 144 us, 5.6 TB/s.
template <bool FLAT>
__global__ __launch_bounds__(NT) void k_pages_move(CompactArgs a, uint32_t table_wgs) {
  const int live = a.live[a.n_to];
  if (blockIdx.x < table_wgs) {
    const uint32_t i = blockIdx.x * NT + threadIdx.x;
    if (i >= (uint32_t)a.t.B * (uint32_t)a.t.M) return;
    const int p = a.t.at[i / a.t.M * a.t.stride + i % a.t.M];
    a.new_table[i] = live && (uint32_t)p < (uint32_t)a.s.n_pages ? a.number[p] : -1;
    return;
  }
  const uint64_t all = (uint64_t)live * copy_parts(a.s);  // (below 2^32)
  for (uint64_t i = blockIdx.x - table_wgs; i < all; i += gridDim.x - table_wgs) {
    const CopyPlace c = copy_place(a.s, (uint32_t)i);
    copy_page<FLAT>(a.pool, a.to, a.s, c.kv, c.layer, c.part, a.live[c.page], c.page, a.s.page_rows);
  }
}

}  // namespace

int64_t pages_parts(const PageShape& s, int64_t pages) {
  return pages * s.layers * 2 * cdiv(s.heads * s.page_rows * s.pieces, PIECES);
}

static size_t listed_bytes(const PageShape& s) { return s.n_pages <= FREE_DIRECT ? 0 : (cdiv(s.n_pages, FREE_BLOCK) + s.n_pages) * 4; }
size_t reserve_bytes(const PageShape& s, const PageTable& t) {
  const int64_t entries = (int64_t)t.B * t.M;
  return up((t.B + 1) * sizeof(int4)) + up(entries * 4) + up(std::min(entries, s.n_pages) * 4) + listed_bytes(s);
}
hipError_t launch_reserve(ReserveArgs a, void* ws, hipStream_t st) {
  const int64_t entries = (int64_t)a.t.B * a.t.M;
  a.copies = (int4*)ws;
  a.kind = (int32_t*)((char*)ws + up((a.t.B + 1) * sizeof(int4)));
  a.free_list = (int32_t*)((char*)a.kind + up(entries * 4));
  a.listed = listed_bytes(a.s) ? (int32_t*)((char*)a.free_list + up(std::min(entries, a.s.n_pages) * 4)) : nullptr;
  if (a.listed) k_pages_free<<<(unsigned)cdiv(a.s.n_pages, FREE_BLOCK), BOOK, 0, st>>>(a);
  k_pages_reserve<<<1, BOOK, 0, st>>>(a);
  k_pages_copy<<<(unsigned)std::min<int64_t>(pages_parts(a.s, a.t.B), 2048), NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  const int64_t tokens = a.offsets ? a.T : a.T * a.t.B;
  if (tokens) k_pages_append<<<(unsigned)(tokens * a.s.layers), NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_keep(const KeepArgs& a, hipStream_t st) {
  k_pages_keep<<<(unsigned)(a.t.B * a.s.layers * a.s.heads * 2), NT, 0, st>>>(a);
  return hipGetLastError();
}

// A workgroup a request and 1024 entries.
static dim3 table_grid(const PageTable& t) { return dim3(t.B, (unsigned)std::min<int64_t>(cdiv(t.M, 4 * NT), 1024)); }

// (64 requests with tables of 126 pages: 6.4 us in two launches or in one, which is 3.5 us less for the host)
size_t fork_bytes(const PageTable& t) { return (int64_t)t.B * t.M <= FORK_FEW ? 0 : (size_t)t.B * (t.M + 1) * 4; }
hipError_t launch_fork(ForkArgs a, void* ws, hipStream_t st) {
  if ((int64_t)a.t.B * a.t.M <= FORK_FEW) {
    k_pages_fork_few<<<1, BOOK, 0, st>>>(a);
    return hipGetLastError();
  }
  a.tmp = (int32_t*)ws;
  k_pages_fork<<<table_grid(a.t), NT, 0, st>>>(a);
  k_pages_forked<<<table_grid(a.t), NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_release(const PageTable& t, int32_t* refs, const int32_t* lengths, int64_t n_pages, int page_rows, hipStream_t st) {
  k_pages_release<<<table_grid(t), NT, 0, st>>>(t, refs, lengths, n_pages, page_rows);
  return hipGetLastError();
}

size_t compact_bytes(const PageShape& s, int64_t n_to) { return up(s.n_pages * 4) + (n_to + 1) * 4; }
hipError_t launch_compact(CompactArgs a, void* ws, hipStream_t st) {
  a.number = (int32_t*)ws;
  a.live = (int32_t*)((char*)ws + up(a.s.n_pages * 4));
  const int64_t table_wgs = cdiv((int64_t)a.t.B * a.t.M, NT);
  const unsigned grid = (unsigned)(table_wgs + std::min<int64_t>(pages_parts(a.s, std::min(a.n_to, a.s.n_pages)), 1 << 16));
  bool flat = true;  // (a stride along one entry is 0)
  for (const PagePool* p : {&a.pool, &a.to})
    for (int i = 0; i < 2; ++i) {
      const int64_t d = a.s.pieces * (16 / a.s.es);
      flat &= (a.s.page_rows == 1 || p->row[i] == d) && (a.s.heads == 1 || p->head[i] == d * a.s.page_rows);
    }
  k_pages_number<<<1, BOOK, 0, st>>>(a);
  if (flat) k_pages_move<true><<<grid, NT, 0, st>>>(a, (uint32_t)table_wgs);
  else k_pages_move<false><<<grid, NT, 0, st>>>(a, (uint32_t)table_wgs);
  return hipGetLastError();
}

}  // namespace topk
