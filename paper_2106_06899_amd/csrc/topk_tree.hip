// Attention of drafted tokens over a cache in pages. Request b holds lengths[b] rows, the last T of them its
// drafts, a tree: a draft sees the rows before the drafts, itself and the drafts that it follows. With one
// draft that is the step of a single token. out_i = sum_j softmax_j(scale q_i.k_j) v_j.
//
// The (H / Hkv) * T rows of a request and key head are one short list, so that its keys are read once for
// all of them (up to 128). A workgroup takes a tile of that list and a range of the request's keys, and where a
// request has several ranges leaves a partial result (maximum, sum and unnormalised output, in 32 bits),
// which a second kernel joins. Lengths lie on the device: ranges of equal length are laid out over all
// requests' keys together, and every workgroup finds its own from the lengths, so that the work is even
// whatever the lengths and the width of the table.
//
// Both forms find a key's row through the table: a lane of each wave looks up one key of the next tile but one,
// so that the table's latency is behind a tile's work, and passes the row's address on to the lanes that load
// it. Keys behind the range, and keys whose entry names no page, have a row of zeros in their place and a score
// of -inf.
//
// Few rows (up to 16, at d = 64 up to 32): four waves take key tiles of 32 in turn, K and V in registers, each with
// a running softmax of its own, joined through LDS; v_mfma_f32_16x16x32_bf16, S^T = K Q^T and O^T = V^T P^T, so that a lane
// holds one row's numbers. Weights enter the second product as the sum of two bf16 numbers (16 significant bits).
// Bound by reading the cache: the next token of 32 requests of 100 to 4096 keys, 32 heads of 128 on 8, 58 us (4.7 TB/s)
// and the join's 4.8.
// Many rows: 128, 32 a wave, every wave takes every key tile of 64 through LDS; v_mfma_f32_32x32x16_bf16, V^T by
// transposing LDS reads. With 64 rows a request and key head and more, weights are rounded to bf16
// (relative 2^-9 at most). Bound by reading too, beside the products: 24 drafts of 48 requests of 500 to 8192 keys
// 204 us (4.3 TB/s), 64 drafts of 2 requests of up to 100000 keys 190 (5.6), the joins 15 and 12.
#include "topk_packed_device.h"
#include "topk_tree.h"

#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

namespace topk {
namespace {

#define TOPK_INLINE __attribute__((always_inline))  // (a lambda that is called captures through memory)
int64_t cdiv(int64_t x, int64_t y) { return (x + y - 1) / y; }

constexpr int NT = 256, WAVES = 4;
constexpr int UNIT = 128;                             // keys; ranges are whole units
constexpr int64_t KEYS_MAX = (int64_t(1) << 31) - 4 * UNIT;  // of a request

// what a key without a page, or behind the range, has for a row
__device__ uint4 zero_row[16];

struct TreeArgs {
  TreeProblem p;
  TreePlan pl;
  float* po;   // [ranges][Hkv][rows][D]
  float2* ml;  // [ranges][Hkv][rows]: maximum of the scaled scores (to base 2), sum of weights
  int2* info;  // [B]: a request's first range, how many it has
  float c;     // scale * log2(e)
  uint32_t magic;  // floor(2^16 / page_rows) + 1
};

// a row's factor and its logarithm (to base e) from the sum of its weights, 0 where it saw no key, and the
// maximum that they were taken against (to base 2)
__device__ __forceinline__ float row_factor(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }
__device__ __forceinline__ float row_log(float top, float sum) {
  return sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
}

__device__ __forceinline__ int64_t keys_of(const TreeProblem& p, int b) {
  return max((int64_t)0, min((int64_t)p.lengths[b], min(p.M * p.page_rows, KEYS_MAX)));
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += (uint64_t)__shfl_xor((long long)x, o, 64);
  return x;
}
__device__ __forceinline__ uint32_t units_of(int64_t keys) { return (uint32_t)((keys + UNIT - 1) / UNIT); }

__device__ __forceinline__ uint32_t ranges_of(int64_t keys, uint32_t units) {
  return units == UINT32_MAX ? 1u : max(1u, (units_of(keys) + units - 1) / units);
}

// Units of a range. As many as leave the wanted number of ranges of all requests' keys (two and more workgroups a
// place on the chip, which even out: the next token of 32 requests of up to 4096 63 us, 69 in one round), or, where
// that would be short ranges, of SINGLE units at most, the fewest that leave one round of workgroups (20 requests of
// up to 1500: 22 us in one round of three units, 26 in two rounds of two; 30 with 8 drafts 37 and 44).
__device__ __forceinline__ uint32_t range_units(const TreeArgs& a) {
  constexpr uint32_t SINGLE = 8;
  if (!a.pl.ranges) return UINT32_MAX;
  const int lane = threadIdx.x & 63;
  uint64_t sum = 0;
  uint32_t mine = 0;
  if (a.p.B <= 64) {
    if (lane < a.p.B) mine = units_of(keys_of(a.p, lane));
    sum = wave_sum64(mine);
  } else {  // (by the whole workgroup)
    __shared__ uint64_t sums[WAVES];
#pragma unroll 4
    for (int b = threadIdx.x; b < a.p.B; b += NT) sum += units_of(keys_of(a.p, b));
    sum = wave_sum64(sum);
    if (lane == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = sums[0] + sums[1] + sums[2] + sums[3];
  }
  const uint32_t least = (uint32_t)max((sum + a.pl.ranges - 1) / a.pl.ranges, (uint64_t)1);
  if (a.pl.round > a.p.B / 2) {
    // (requests' last ranges are half full on average; where a wave holds all lengths the ranges are counted)
    const uint64_t full = a.p.B <= 64 ? a.pl.round : a.pl.round - a.p.B / 2;
    for (uint32_t u = (uint32_t)max((sum + full - 1) / full, (uint64_t)least); u <= SINGLE; ++u)
      if (a.p.B > 64 || wave_sum(lane < a.p.B ? max(1u, (mine + u - 1) / u) : 0) <= a.pl.round) return u;
  }
  return max(least, 2u);
}

struct TreeRange {
  int b;        // request; -1: there is none
  int of;       // ranges of the request
  int which;    // this one's place among them
  int first;    // this one's first key
  int n;        // its keys
  int len;      // the request's
};
// Range w of all requests', by every wave, or where there are more than 64 by the whole workgroup.
__device__ __forceinline__ TreeRange find_range(const TreeArgs& a, uint32_t w) {
  const int lane = threadIdx.x & 63;
  const uint32_t units = range_units(a);
  TreeRange r = {-1, 0, 0, 0, 0, 0};
  uint32_t mine = 0;
  if (!a.pl.ranges) {
    r.b = (int)w;
  } else if (a.p.B <= 64) {
    const uint32_t n = lane < a.p.B ? ranges_of(keys_of(a.p, lane), units) : 0, end = wave_incl_scan_full(n);
    const uint64_t those = __builtin_amdgcn_ballot_w64(end > w);
    if (!those) return r;
    r.b = __builtin_ctzll(those);
    mine = w - (uint32_t)(__builtin_amdgcn_readlane((int)end, r.b) - __builtin_amdgcn_readlane((int)n, r.b));
  } else {
    __shared__ uint32_t sums[4], found[2];
    if (threadIdx.x == 0) found[0] = UINT32_MAX;
    uint32_t before = 0, first;
    for (int64_t b0 = 0; b0 < a.p.B && before <= w; b0 += NT) {
      const int64_t b = b0 + threadIdx.x;
      if (block_find(b < a.p.B ? ranges_of(keys_of(a.p, (int)b), units) : 0, w, &before, &first, sums)) {
        found[0] = (uint32_t)b;
        found[1] = w - first;
      }
    }
    __syncthreads();
    if (found[0] == UINT32_MAX) return r;
    r.b = (int)found[0];
    mine = found[1];
  }
  const int64_t len = keys_of(a.p, r.b), first = (int64_t)mine * units * UNIT;
  r.which = __builtin_amdgcn_readfirstlane((int)mine);
  r.len = __builtin_amdgcn_readfirstlane((int)len);
  r.of = __builtin_amdgcn_readfirstlane((int)ranges_of(len, units));
  r.first = __builtin_amdgcn_readfirstlane((int)first);
  r.n = __builtin_amdgcn_readfirstlane(units == UINT32_MAX ? (int)len : (int)max((int64_t)0, min(len - first, (int64_t)units * UNIT)));
  return r;
}

// Which drafts draft i < T sees, as bits: itself and what it follows. The first 64 threads write them, the
// workgroup waits. (Parents that are not drafts before it stand for the text.)
__device__ __forceinline__ void tree_bits(const TreeProblem& p, int b, uint64_t* bits) {
  const int i = threadIdx.x;
  if (i < 64) {
    int up = p.parents ? (i < p.T ? p.parents[b * p.parents_stride + i] : -1) : i - 1;
    if ((uint32_t)up >= (uint32_t)i) up = i;
    uint64_t mine = 1ull << i;
#pragma unroll
    for (int s = 0; s < 6; ++s) {  // twice as far up each time
      mine |= (uint64_t)__shfl((long long)mine, up, 64);
      up = __shfl(up, up, 64);
    }
    bits[i] = mine;
  }
  __syncthreads();
}

// Where the rows of the keys lie.
struct Rows {
  const unsigned char* base[2];  // of the head, keys and values
  const int32_t* table;          // the request's
  int64_t page[2], row[2];       // strides in bytes
  int page_rows, M;
  uint32_t magic, n_pages;
  int one;                       // (no table) the request's only page

  __device__ __forceinline__ Rows(const TreeArgs& a, int b, int h) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      base[i] = (const unsigned char*)a.p.pool[i] + h * a.p.head[i] * 2;
      page[i] = a.p.page[i] * 2;
      row[i] = a.p.row[i] * 2;
    }
    table = a.p.table ? a.p.table + b * a.p.table_stride : nullptr;
    page_rows = (int)min(a.p.page_rows, (int64_t)INT_MAX);
    M = (int)a.p.M;
    magic = a.magic;
    n_pages = (uint32_t)a.p.n_pages;
    one = b;
  }
  // The entry of the table, and the row of its page, of the key o < 64 behind `first`; -1: there is none (o >= n).
  __device__ __forceinline__ int2 place(int first, int o, int n) const {
    const int e0 = first / page_rows, r0 = first - e0 * page_rows;  // (uniform)
    const int r = r0 + o, q = page_rows >= 64 ? (r >= page_rows) : (int)((uint32_t)r * magic >> 16);
    return make_int2(o < n ? e0 + q : -1, r - q * page_rows);
  }
  __device__ __forceinline__ int lookup(int e) const {
    const int p = table ? table[min(max(e, 0), M - 1)] : one;
    return (uint32_t)e < (uint32_t)M ? p : -1;
  }
  __device__ __forceinline__ bool valid(int p) const { return (uint32_t)p < n_pages; }
  __device__ __forceinline__ const unsigned char* at(int i, int p, int r) const {
    return valid(p) ? base[i] + p * page[i] + r * row[i] : (const unsigned char*)zero_row;
  }
};

// what lane `lane` < 64 holds
__device__ __forceinline__ const unsigned char* pass_on(const unsigned char* p, int lane) {
  const uint64_t x = (uint64_t)(uintptr_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(lane * 4, (int)(uint32_t)x), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(lane * 4, (int)(x >> 32));
  return (const unsigned char*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

// A look at the values of n keys from `first` on for sums that are NaN (see Infinities). sees(u): the drafts that row u sees.
template <int D, int U, typename F>
__device__ __forceinline__ void settle_range(Infinities<D, U>& is, const Rows& rows, int first, int n, int text, F sees) {
  typedef Infinities<D, U> Is;
  const int lane = is.own_lane();
  for (int k0 = 0; k0 < n && is.unsettled(); k0 += 64) {
    const int2 at = rows.place(first + k0, lane, n - k0);
    const int p = rows.lookup(at.x), d0 = first + k0 - text;  // (the draft that key 0 of these is)
    const unsigned char* v = rows.at(1, p, at.y);
    const uint64_t there = __builtin_amdgcn_ballot_w64(rows.valid(p));
#pragma unroll 4
    for (int j = 0; j < 64; j += Is::ROWS)
      is.look(lane, *(const u32x4*)(pass_on(v, j + lane / Is::PARTS) + lane % Is::PARTS * 16), [&](int k, int u) TOPK_INLINE {
        const int draft = d0 + j + k;
        return (there >> (j + k) & 1) && (draft < 0 || (draft < 64 && (sees(u) >> draft & 1)));
      });
  }
}

struct TreeLds {
  unsigned char *b0, *b1, *b2, *b3;
  float2 (*ml)[32], *sum;
  uint64_t *bits, *marks;
  uint32_t (*mask)[WAVES];
  __device__ TOPK_LDS unsigned char* of(int w) const {
    TOPK_LDS unsigned char *p0 = (TOPK_LDS unsigned char*)b0, *p1 = (TOPK_LDS unsigned char*)b1, *p2 = (TOPK_LDS unsigned char*)b2,
                           *p3 = (TOPK_LDS unsigned char*)b3;
    return w == 0 ? p0 : w == 1 ? p1 : w == 2 ? p2 : p3;
  }
};

struct TreeItem {
  TreeRange r;
  int h, r0, R;  // key head; first row of the tile; rows of the list
  int64_t slot;  // where the partial result goes: rows before its first
};

// 16 NR rows. FOUR: pages hold whole groups of four keys, which share a look-up.
template <int D, int NR, bool FOUR>
struct TreeFew {
  static constexpr int NS = D / 32, NC = D / 16, VB = NC * 2, KT = 32;

  static __device__ __forceinline__ bf16x8 column(const uint32_t (&x)[8][NC / 2], int c) {  // of eight keys' numbers, as an operand
    const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
    const int w = c / 2;
    return __builtin_bit_cast(bf16x8, make_uint4(__builtin_amdgcn_perm(x[1][w], x[0][w], sel), __builtin_amdgcn_perm(x[3][w], x[2][w], sel),
                                                 __builtin_amdgcn_perm(x[5][w], x[4][w], sel), __builtin_amdgcn_perm(x[7][w], x[6][w], sel)));
  }

  static __device__ __forceinline__ void run(const TreeArgs& a, const TreeItem& it, const TreeLds& sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int T = a.p.T, len = it.r.len, text = len - T;  // keys from `text` on are drafts
    const int end = it.r.first + it.r.n;
    const bool drafts = end > text;
    if (drafts) tree_bits(a.p, it.r.b, sh.bits);
    auto place = [&](int i) { return ((int64_t)it.r.b * a.p.H + it.h * (a.p.H / a.p.Hkv)) * T + i; };  // of row i in q and out
    auto lane_row = [&](int r) { return it.r0 + 16 * r + n < it.R ? it.r0 + 16 * r + n : it.r0; };
    bf16x8 bq[NR][NS];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const uint16_t* q = (const uint16_t*)a.p.q + place(lane_row(r)) * D + 8 * g;
#pragma unroll
      for (int s = 0; s < NS; ++s) bq[r][s] = *(const bf16x8*)(q + 32 * s);
    }
    f32x4 o[NR][NC];
    float m[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) o[r][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    uint32_t marks[NR] = {};  // bit v * NC + c: o[..][c][v], of feature 4 g NC + v NC + c, is NaN
    const Rows rows(a, it.r.b, it.h);
    const int tiles = (it.r.n + KT - 1) / KT;

    bf16x8 kr[2][NS];
    uint32_t vr[8][NC / 2];
    // lane l looks up key l % 32 of a tile, its page one tile of the wave before its rows are loaded
    auto look_up = [&](int t) TOPK_INLINE {
      const int2 x = rows.place(it.r.first + t * KT, lane & 31, it.r.n - t * KT);
      return make_int2(t < tiles ? rows.lookup(x.x) : -1, x.y);
    };
    auto load_k = [&](int2 x) TOPK_INLINE {
      const unsigned char* p = rows.at(0, x.x, x.y);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint16_t* k = (const uint16_t*)pass_on(p, 16 * kb + n) + 8 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) kr[kb][s] = *(const bf16x8*)(k + 32 * s);
      }
    };
    auto load_v = [&](int2 x) TOPK_INLINE {
      const unsigned char* p = rows.at(1, x.x, x.y);
      if (FOUR) {
        const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(rows.valid(x.x)) >> 4 * g;
#pragma unroll
        for (int e = 0; e < 8; e += 4) {  // (keys of the group behind the range: masked where they are used)
          const unsigned char* v = pass_on(p, 4 * e + 4 * g) + n * VB;
          const int64_t step = there >> 4 * e & 1 ? rows.row[1] : 0;
#pragma unroll
          for (int u = 0; u < 4; ++u) __builtin_memcpy(vr[e + u], __builtin_assume_aligned(v + u * step, VB), VB);
        }
        return;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned char* v = pass_on(p, 16 * (e >> 2) + 4 * g + (e & 3)) + n * VB;
        __builtin_memcpy(vr[e], __builtin_assume_aligned(v, VB), VB);
      }
    };
    int t = wave;
    int2 now = make_int2(-1, 0), next = now;
    if (t < tiles) {
      now = look_up(t);
      next = look_up(t + WAVES);
      load_k(now);
      load_v(now);
    }
    auto tile = [&](auto some_draft) TOPK_INLINE {  // some_draft: the tile holds drafts
      const int first = it.r.first + t * KT;
      // bit o: key o of the tile is one
      const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(rows.valid(now.x));
      const int2 here = now;
      now = next;
      f32x4 s[NR][2];
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int st = 0; st < NS; ++st) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[kb][st], bq[r][st], acc, 0, 0, 0);
          s[r][kb] = acc;
        }
      __builtin_amdgcn_sched_barrier(0);  // (one tile's keys and values at a time, for which the registers last)
      load_k(now);  // (behind the last tile: rows of zeros)
      if (there != 0xFFFFFFFFu || decltype(some_draft)::value) {
        // bit o: the lane's row sees key o of the tile
        uint32_t see[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          see[r] = there;
          if (decltype(some_draft)::value) {  // drafts first - text + o >= 0 by their bits, keys before them all
            const int d0 = first - text;
            const uint64_t sees = sh.bits[lane_row(r) % T], x = d0 >= 0 ? (d0 < 64 ? sees >> d0 : 0) : sees << -d0 | ((1u << -d0) - 1u);  // (d0 > -32)
            see[r] &= (uint32_t)x;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!(see[r] >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1)) s[r][e >> 2][e & 3] = -INFINITY;
        }
        // Drafts' values that are not finite go to the rows that see them, which become NaN there (and infinite,
        // where they are, at the end); the others would meet them as 0 times NaN.
        uint32_t bad = 0;
        if (decltype(some_draft)::value) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t is = there >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1 ? 0xFFFFFFFFu : 0u;
#pragma unroll
            for (int w = 0; w < NC / 2; ++w) {
              const uint32_t nf = not_finite(vr[e][w]) & is;
              bad |= nf;
              vr[e][w] &= is & ~(nf * 0xFFFFu);
            }
          }
        }
        if (decltype(some_draft)::value && __builtin_amdgcn_ballot_w64(bad)) {
          const unsigned char* p = rows.at(1, here.x, here.y);
#pragma unroll 1
          for (int k = 0; k < KT; ++k) {
            const uint32_t* v = (const uint32_t*)(pass_on(p, k) + 8 * g * NC);
            uint32_t x = 0;
#pragma unroll 1
            for (int w = 0; w < 2 * NC; ++w) {
              const uint32_t nf = not_finite(v[w]);
              x |= ((nf & 1) | nf >> 15) << 2 * w;
            }
#pragma unroll
            for (int r = 0; r < NR; ++r) marks[r] |= see[r] >> k & 1 ? x : 0;
          }
        }
      }
      next = look_up(t + 2 * WAVES);
      bf16x8 hi[NR], lo[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float mt = larger(larger(larger(s[r][0][0], s[r][0][1]), larger(s[r][0][2], s[r][0][3])),
                          larger(larger(s[r][1][0], s[r][1][1]), larger(s[r][1][2], s[r][1][3])));
        mt = larger(mt, __shfl_xor(mt, 16, 64));
        mt = larger(mt, __shfl_xor(mt, 32, 64));
        const float mn = larger(m[r], mt * a.c);
        const float off = mn == -INFINITY ? 0.f : mn;
        if (__builtin_amdgcn_ballot_w64(mn != m[r])) {
          const float alpha = exp2f(m[r] - off);  // (m = -inf: 0)
          l[r] *= alpha;
#pragma unroll
          for (int c = 0; c < NC; ++c) o[r][c] *= alpha;
          m[r] = mn;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w = exp2f(fmaf(s[r][e >> 2][e & 3], a.c, -off));
          l[r] += w;
          hi[r][e] = (__bf16)w;
          lo[r][e] = (__bf16)(w - (float)hi[r][e]);
        }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 av = column(vr, c);
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, hi[r], o[r][c], 0, 0, 0);
          o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, lo[r], o[r][c], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v(now);
    };
    for (; t < tiles && it.r.first + t * KT + KT <= text; t += WAVES) tile(std::false_type{});
    for (; t < tiles; t += WAVES) tile(std::true_type{});

#pragma unroll
    for (int r = 0; r < NR; ++r)
      if (__builtin_amdgcn_ballot_w64(marks[r] != 0))
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (marks[r] >> (v * NC + c) & 1) o[r][c][v] = NAN;
    // join the waves: every row's maximum and sum, then the scaled outputs through LDS, in parts of four
    // features whose order in a row is permuted by the row so that its lanes meet different banks
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      l[r] += __shfl_xor(l[r], 16, 64);
      l[r] += __shfl_xor(l[r], 32, 64);
      if (g == 0) sh.ml[wave][16 * r + n] = make_float2(m[r], l[r]);
    }
    __syncthreads();
    TOPK_LDS f32x4* mine = (TOPK_LDS f32x4*)sh.of(wave);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float2 x[WAVES];
      float top = -INFINITY, total = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        x[w] = sh.ml[w][16 * r + n];
        top = larger(top, x[w].x);
      }
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) total = fmaf(exp2f(x[w].x - base), x[w].y, total);
      const float f = exp2f(m[r] - base);  // (m = -inf: 0)
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int c = 0; c < NC; c += 4)
          mine[(16 * r + n) * (D / 4) + ((((4 * g + v) * NC + c) / 4) ^ n)] =
              (f32x4){o[r][c][v] * f, o[r][c + 1][v] * f, o[r][c + 2][v] * f, o[r][c + 3][v] * f};
      if (wave == 0 && g == 0) sh.sum[16 * r + n] = make_float2(top, total);
    }
    __syncthreads();
    constexpr int SU = 16 * NR * D / 4 / NT;  // stores
    const int part = tid % (D / 4);
    Infinities<D, SU> is;
    auto row_of = [&](int u) TOPK_INLINE { return (u * NT + tid) / (D / 4); };
    auto sums = [&](int u) TOPK_INLINE {
      const int row = row_of(u);
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += ((const TOPK_LDS f32x4*)sh.of(w))[row * (D / 4) + (part ^ (row & 15))];
      return sum;
    };
    auto store = [&](int u, const f32x4& sum) TOPK_INLINE {
      const int row = row_of(u);
      const float2 x = sh.sum[row];
      if (it.r0 + row >= it.R) return;
      if (it.r.of == 1) {
        const int64_t at = place(it.r0 + row);
        const float inv = row_factor(x.y);
        *(uint2*)((uint16_t*)a.p.out + at * D + 4 * part) = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
        if (a.p.lse && part == 0) a.p.lse[at] = row_log(x.x, x.y);
      } else {
        const int64_t at = it.slot + it.r0 + row;
        __builtin_nontemporal_store(sum, (f32x4*)(a.po + at * D + 4 * part));
        if (part == 0) a.ml[at] = x;
      }
    };
#pragma unroll
    for (int u = 0; u < SU; ++u) {
      const f32x4 x = sums(u);
      const float l = sh.sum[row_of(u)].y;
      is.nan(u, x, it.r0 + row_of(u) < it.R && l == l);
      store(u, x);
    }
    if (__builtin_amdgcn_ballot_w64(is.open != 0)) {
      settle_range(is, rows, it.r.first, it.r.n, text, [&](int u) TOPK_INLINE { return drafts ? sh.bits[(it.r0 + row_of(u)) % T] : 0; });
#pragma unroll 1
      for (int u = 0; u < SU; ++u) {
        f32x4 x = sums(u);
        is.settle(u, x);
        store(u, x);
      }
    }
  }
};

// 128 rows. TWO: weights enter the second product as two bf16 numbers.
template <int D, bool TWO>
struct TreeWide {
  typedef PackedTile<D> Tile;
  static constexpr float LEAD = 8.f;  // the maximum is moved only once a score leads it by 2^8 in weight
  static constexpr int KEYS = 64, NS = D / 16, CH = 2 * D / 16, TILEB = KEYS * 2 * D, LPW = TILEB / 1024 / WAVES, FB = D / 32;
  static constexpr int AHEAD_K = 6, AHEAD_V = 4;  // products by which LDS reads run ahead of their use

  static __device__ __forceinline__ void run(const TreeArgs& a, const TreeItem& it, const TreeLds& sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
    const int T = a.p.T, len = it.r.len, text = len - T;
    const int i = it.r0 + wave * 32 + n;
    const bool ok = i < it.R, work = it.r0 + wave * 32 < it.R;
    const int64_t list = ((int64_t)it.r.b * a.p.H + it.h * (a.p.H / a.p.Hkv)) * T;  // rows before the list's first
    const bool drafts = it.r.first + it.r.n > text;
    if (drafts) tree_bits(a.p, it.r.b, sh.bits);
    const uint64_t sees = drafts ? sh.bits[(ok ? i : it.r0) % T] : 0;
    bf16x8 bq[NS];
    {
      const uint16_t* q = (const uint16_t*)a.p.q + (list + (ok ? i : it.r0)) * D + (D / 2) * half;
#pragma unroll
      for (int s = 0; s < NS; ++s) bq[s] = *(const bf16x8*)(q + 8 * s);
    }
    f32x16 o[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f) o[f] = (f32x16){};
    float m = -INFINITY, l = 0.f;
    const uint32_t kbase = Tile::straight_base(), vbase = Tile::across_base();
    const Rows rows(a, it.r.b, it.h);
    const int tiles = (it.r.n + KEYS - 1) / KEYS;

    // A wave loads rows 16 wave .. of a tile; lane l looks up row 16 wave + l % 16, a tile ahead of its load.
    auto look_up = [&](int t) TOPK_INLINE {
      const int2 x = rows.place(it.r.first + t * KEYS, 16 * wave + (lane & 15), it.r.n - t * KEYS);
      return make_int2(t < tiles ? rows.lookup(x.x) : -1, x.y);
    };
    int2 next = look_up(0);
    constexpr int STEP = 64 / CH, FLIP = D == 128 ? 1 : 2;  // rows of a load; how its parts' places differ from the one before's
    const int lrow = lane / CH, lpart = lane % CH ^ Tile::swz(16 * wave + lrow);
    auto issue = [&](int t, unsigned char* kd, unsigned char* vd) TOPK_INLINE {
      const int2 x = next;
      const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(rows.valid(x.x)) & 0xFFFFu;
      if (lane == 0) sh.mask[t & 1][wave] = there;  // (read behind the barrier that publishes the tile)
      const unsigned char *kp = rows.at(0, x.x, x.y), *vp = rows.at(1, x.x, x.y);
      next = look_up(t + 1);
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        const uint32_t c = (lpart ^ (j * FLIP)) * 16;
        __builtin_amdgcn_global_load_lds((const void*)(pass_on(kp, j * STEP + lrow) + c), (TOPK_LDS void*)&kd[(wave * LPW + j) * 1024], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const void*)(pass_on(vp, j * STEP + lrow) + c), (TOPK_LDS void*)&vd[(wave * LPW + j) * 1024], 16, 0, 0);
      }
    };
    // bit k of the 64: the lane's row sees key k of tile t
    auto see = [&](int t) TOPK_INLINE {
      const uint32_t* x = sh.mask[t & 1];
      uint64_t there = (uint64_t)(x[2] | x[3] << 16) << 32 | (x[0] | x[1] << 16);
      const int d0 = it.r.first + t * KEYS - text;  // the draft that key 0 is
      if (d0 > -KEYS) there &= d0 >= 0 ? (d0 < 64 ? sees >> d0 : 0) : sees << -d0 | ((1ull << -d0) - 1);
      return there;
    };

    auto tile = [&](bool edge, uint64_t seen, const unsigned char* kb, const unsigned char* vb) TOPK_INLINE {
      f32x16 s[2] = {};
      {
        bf16x8 kf[AHEAD_K + 1];
        auto kp = [&](int i) TOPK_INLINE { return Tile::straight((const TOPK_LDS unsigned char*)kb, kbase, i & 1, i >> 1); };
#pragma unroll
        for (int i = 0; i < AHEAD_K; ++i) kf[i] = kp(i);
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i) {
          if (i + AHEAD_K < 2 * NS) kf[(i + AHEAD_K) % (AHEAD_K + 1)] = kp(i + AHEAD_K);
          s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % (AHEAD_K + 1)], bq[i >> 1], s[i & 1], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      float low = INFINITY;  // the tile's lowest score (masked keys' included, NaN too: they only choose the pass below)
#pragma unroll
      for (int v = 0; v < 32; v += 2)
        low = __builtin_elementwise_minimum(__builtin_elementwise_minimum(low, s[v >> 4][v & 15]), s[v >> 4][(v & 15) + 1]);
      if (edge) {
        const uint64_t x = seen >> 4 * half;
#pragma unroll
        for (int v = 0; v < 32; ++v)
          if (!(x >> ((v >> 4) * 32 + 8 * ((v & 15) >> 2) + (v & 3)) & 1)) s[v >> 4][v & 15] = -INFINITY;
      }
      float mt = -INFINITY;
#pragma unroll
      for (int v = 0; v < 32; v += 2)
        mt = larger(larger(mt, s[v >> 4][v & 15]), s[v >> 4][(v & 15) + 1]);
      mt = other_half_max(mt) * a.c;
      const bool leads = !(mt <= m + LEAD);  // (NaN too)
      if (__builtin_amdgcn_ballot_w64(leads)) {  // (the other rows multiply by 1: a row's result is its own)
        const float mn = leads ? larger(m, mt) : m;
        const float alpha = mn == -INFINITY ? 1.f : exp2f(m - mn);  // (below 2^-126 too: see the weights)
        m = mn;
        l *= alpha;
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[f][v] *= alpha;
      }
      constexpr int VM = 4 * FB;
      const float off = m == -INFINITY ? 0.f : m;
      auto vp = [&](int j) TOPK_INLINE { return Tile::across((const TOPK_LDS unsigned char*)vb, vbase, j % FB, j / FB); };
      // Weights below 2^-126, which the exponential instruction alone makes 0, are added by themselves
      // where the tile has any.
      if (__builtin_amdgcn_ballot_w64(!(fmaf(low, a.c, -off) >= -126.f))) {
        float bias = -off;
        asm volatile("" : "+v"(bias));  // (nothing of this pass is held for the other)
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          bf16x8 pt;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = fmaf(s[st >> 1][8 * (st & 1) + e], a.c, bias), w = x < -126.f ? exp2f(x) : 0.f;
            l += w;
            pt[e] = (__bf16)w;
          }
#pragma unroll
          for (int f = 0; f < FB; ++f) {
            o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp(st * FB + f), pt, o[f], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      bf16x8 pb[4], pl[4], vf[AHEAD_V + 1];
#pragma unroll
      for (int j = 0; j < AHEAD_V; ++j) vf[j] = vp(j);
      __builtin_amdgcn_s_setprio(1);  // the other wave's softmax yields to this one's products
      auto wt = [&](int v) TOPK_INLINE {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[v >> 4][v & 15], a.c, -off));
        l += w;
        pb[v >> 3][v & 7] = (__bf16)w;
        if (TWO) pl[v >> 3][v & 7] = (__bf16)(w - (float)pb[v >> 3][v & 7]);
      };
#pragma unroll
      for (int v = 0; v < 8; ++v) wt(v);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < VM; ++j) {
        if (j + AHEAD_V < VM) vf[(j + AHEAD_V) % (AHEAD_V + 1)] = vp(j + AHEAD_V);
        o[j % FB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j % (AHEAD_V + 1)], pb[j / FB], o[j % FB], 0, 0, 0);
        if (TWO) o[j % FB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j % (AHEAD_V + 1)], pl[j / FB], o[j % FB], 0, 0, 0);
        if (j + FB < VM)
#pragma unroll
          for (int v = 0; v < 8 / FB; ++v) wt(8 + j * (8 / FB) + v);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    };

    // One tile of lookahead: before tile t is read, this wave's loads of it are complete and the barrier
    // publishes every wave's part; it also proves that no wave still reads the buffers that the next loads
    // overwrite.
    auto own_part = [&](unsigned char* vb, int j) TOPK_INLINE { return (TOPK_LDS u32x4*)&vb[(wave * LPW + j) * 1024 + lane * 16]; };
    sh.marks[tid] = 0;
    auto step = [&](auto works, int t, unsigned char* kb, unsigned char* vb, unsigned char* kn, unsigned char* vn) TOPK_INLINE {
      __builtin_amdgcn_s_waitcnt(PACKED_WAIT_VM0);
      const bool some_draft = it.r.first + t * KEYS + KEYS > text;
      if (some_draft) {  // drafts' values that are not finite: each wave looks at its part of the tile
        uint32_t bad = 0;
#pragma unroll 1
        for (int j = 0; j < LPW; ++j) {
          const u32x4 x = *own_part(vb, j);
          bad |= not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3]);
        }
        const bool any = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
        if (lane == 0) sh.ml[wave][t & 1].x = any ? 1.f : 0.f;  // (read before the next barrier; the next tile's is another)
      }
      __syncthreads();
      if (t + 1 < tiles) issue(t + 1, kn, vn);
      const uint32_t* x = sh.mask[t & 1];
      const bool edge = some_draft || (x[0] & x[1] & x[2] & x[3]) != 0xFFFFu;
      const uint64_t seen = edge ? see(t) : ~0ull;
      if (some_draft && sh.ml[0][t & 1].x + sh.ml[1][t & 1].x + sh.ml[2][t & 1].x + sh.ml[3][t & 1].x > 0.f) {
        // They go only to the rows that see them, which become NaN there (at the end); the others would meet them
        // as 0 times NaN. (Bit 16 f + v: feature 32 f + 8 (v / 4) + 4 half + v % 4.)
        uint64_t marks = 0;
#pragma unroll 1
        for (int j = 0; j < KEYS; ++j)
#pragma unroll 1
          for (int u = 0; u < D / 8; ++u) {
            const TOPK_LDS uint32_t* y = (const TOPK_LDS uint32_t*)&vb[j * 2 * D + (u ^ Tile::swz(j)) * 16 + 8 * half];
            const uint32_t n0 = not_finite(y[0]), n1 = not_finite(y[1]);
            const uint64_t bit = (n0 & 1) | n0 >> 15 | (n1 & 1) << 2 | n1 >> 16 << 3;
            if (seen >> j & 1) marks |= bit << 4 * u;
          }
        sh.marks[tid] |= marks;
        __syncthreads();
#pragma unroll 1
        for (int j = 0; j < LPW; ++j) {
          u32x4 y = *own_part(vb, j);
#pragma unroll
          for (int w = 0; w < 4; ++w) y[w] &= ~(not_finite(y[w]) * 0xFFFFu);
          *own_part(vb, j) = y;
        }
        __syncthreads();
      }
      if (decltype(works)::value) tile(edge, seen, kb, vb);
    };
    if (tiles > 0) issue(0, sh.b0, sh.b2);
    auto all = [&](auto works) TOPK_INLINE {
      for (int t = 0; t < tiles; t += 2) {
        step(works, t, sh.b0, sh.b2, sh.b1, sh.b3);
        if (t + 1 < tiles) step(works, t + 1, sh.b1, sh.b3, sh.b0, sh.b2);
      }
    };
    if (work) all(std::true_type{});
    else all(std::false_type{});
    const uint64_t marks = sh.marks[tid];
    if (__builtin_amdgcn_ballot_w64(marks != 0)) {
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (marks >> (16 * f + v) & 1) o[f][v] = NAN;
    }
    l += __shfl_xor(l, 32, 64);
    float most = o[0][0];  // NaN where any of the sums is: rows that are written once more (see Infinities)
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int v = 0; v < 16; v += 2) most = larger(larger(most, o[f][v]), o[f][v + 1]);
    // through the wave's own part of LDS, in parts of four features permuted by the row, so that whole rows
    // are written; partial results past the cache
    __syncthreads();
    TOPK_LDS f32x4* mine = (TOPK_LDS f32x4*)sh.of(wave);
    constexpr int PARTS = D / 4, RPS = 64 / PARTS;
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        mine[n * PARTS + ((8 * f + v / 2 + half) ^ (n & 15))] = (f32x4){o[f][v], o[f][v + 1], o[f][v + 2], o[f][v + 3]};
    wave_sync_lds();
    const bool last = it.r.of == 1;
    const float inv = row_factor(l);
    const int part = lane % PARTS, row0 = it.r0 + wave * 32;
    constexpr int SU = 32 / RPS;  // stores
    auto sums = [&](int u) TOPK_INLINE {
      const int row = u * RPS + lane / PARTS;
      return mine[row * PARTS + (part ^ (row & 15))];
    };
    auto store = [&](int u, const f32x4& x) TOPK_INLINE {
      const int row = u * RPS + lane / PARTS;
      const float by = __shfl(inv, row, 64);
      if (row0 + row >= it.R) return;
      if (last) *(uint2*)((uint16_t*)a.p.out + (list + row0 + row) * D + 4 * part) = make_uint2(pack_bf16(x[0] * by, x[1] * by), pack_bf16(x[2] * by, x[3] * by));
      else __builtin_nontemporal_store(x, (f32x4*)(a.po + (it.slot + row0 + row) * D + 4 * part));
    };
#pragma unroll 4
    for (int u = 0; u < SU; ++u) store(u, sums(u));
    if (__builtin_amdgcn_ballot_w64(most != most)) {
      Infinities<D, SU> is;
      const int ln = is.own_lane();
#pragma unroll 1
      for (int u = 0; u < SU; ++u) {
        const int row = u * RPS + ln / PARTS;
        const float by = __shfl(inv, row, 64);
        is.nan(u, sums(u), row0 + row < it.R && by == by);
      }
      settle_range(is, rows, it.r.first, it.r.n, text,
                   [&](int u) TOPK_INLINE { return drafts ? sh.bits[(row0 + u * RPS + ln / PARTS) % T] : 0; });
#pragma unroll 1
      for (int u = 0; u < SU; ++u) {
        f32x4 x = sums(u);
        is.settle(u, x);
        store(u, x);
      }
    }
    if (!ok || half) return;
    if (!last) a.ml[it.slot + i] = make_float2(m, l);
    else if (a.p.lse) a.p.lse[list + i] = row_log(m, l);
  }
};

// A form by its number: 1 and 2 few rows (blocks of 16), 3 and 4 the same where pages hold whole groups of four
// keys, 8 and 9 many.
template <int D, int F>
struct TreeForm {
  static constexpr bool FOUR = F >= 3;
  static constexpr int NR = FOUR ? F - 2 : F, ROWS = 16 * NR;
  typedef TreeFew<D, NR, FOUR> type;
};
template <int D>
struct TreeForm<D, 8> {
  typedef TreeWide<D, true> type;
  static constexpr int ROWS = 128;
};
template <int D>
struct TreeForm<D, 9> {
  typedef TreeWide<D, false> type;
  static constexpr int ROWS = 128;
};

template <int D, int F>
__global__ __launch_bounds__(NT, 2) void k_tree(TreeArgs a) {
  constexpr int BUF = F >= 8 ? 64 * 2 * D : TreeForm<D, F>::ROWS * D * 4;
  __shared__ __attribute__((aligned(16))) unsigned char b0[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b1[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b2[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b3[BUF];
  __shared__ float2 ml[WAVES][32], sum[32];
  __shared__ uint64_t bits[64], marks[F >= 8 ? NT : 1];
  __shared__ uint32_t mask[2][WAVES];
  const TreeLds sh = {b0, b1, b2, b3, ml, sum, bits, marks, mask};
  int i = blockIdx.x;
  TreeItem it;
  it.R = a.p.H / a.p.Hkv * a.p.T;
  it.r0 = i % a.pl.tiles * TreeForm<D, F>::ROWS;
  i /= a.pl.tiles;
  it.h = i % a.p.Hkv;
  i /= a.p.Hkv;
  it.r = find_range(a, i);
  if (it.r.b < 0) return;
  it.slot = ((int64_t)i * a.p.Hkv + it.h) * it.R;
  if (a.pl.ranges && !it.r.which && !it.h && !it.r0 && threadIdx.x == 0) a.info[it.r.b] = make_int2(i, it.r.of);
  TreeForm<D, F>::type::run(a, it, sh);
}

// Joins a row's partial results, where there are several. ROWS rows a workgroup: TR threads a row, D / 4 of which take
// four features each, by as many groups as there are left, each taking every so manieth range. The ranges' factors
// come first, a thread a range.
template <int D, int ROWS>
__global__ __launch_bounds__(NT) void k_tree_join(TreeArgs a) {
  constexpr int TR = NT / ROWS, LR = D / 4, Q = TR / LR, WPR = TR / 64;  // WPR: waves of a row
  static_assert(Q >= 1, "a thread has at least one column group");
  __shared__ float fac[ROWS][TR], most[4], sums[4];
  __shared__ f32x4 part[ROWS][Q][LR];
  const int rl = threadIdx.x / TR, tr = threadIdx.x % TR, q = tr / LR, c = tr % LR;
  const int R = a.p.H / a.p.Hkv * a.p.T, per = (R + ROWS - 1) / ROWS;
  const int r = blockIdx.x % per * ROWS + rl, i = blockIdx.x / per, h = i % a.p.Hkv, b = i / a.p.Hkv;
  const int2 info = a.info[b];
  const int of = info.y;
  if (of == 1) return;
  const bool ok = r < R;
  const int64_t at = ((int64_t)info.x * a.p.Hkv + h) * R + (ok ? r : 0), step = (int64_t)a.p.Hkv * R;
  const float2 mine = tr < of ? a.ml[at + tr * step] : make_float2(-INFINITY, 0.f);
  float top = mine.x;
  for (int s = TR + tr; s < of; s += TR) top = larger(top, a.ml[at + s * step].x);
#pragma unroll
  for (int o = 1; o < (TR < 64 ? TR : 64); o <<= 1) top = larger(top, __shfl_xor(top, o, 64));
  if (WPR > 1) {
    if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WPR; ++w) top = larger(top, most[w]);
  }
  float total = 0.f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < of; s0 += TR) {
    const int s = s0 + tr;
    const float2 x = s0 == 0 ? mine : s < of ? a.ml[at + s * step] : make_float2(-INFINITY, 0.f);
    const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - top);
    total = fmaf(f, x.y, total);
    __syncthreads();
    fac[rl][tr] = f;
    __syncthreads();
    const float* p = a.po + (at + s0 * step) * D + 4 * c;
#pragma unroll 4
    for (int k = q; k < min(TR, of - s0); k += Q) sum += *(const f32x4*)(p + k * step * D) * fac[rl][k];  // (a range without keys leaves zeros)
  }
#pragma unroll
  for (int o = 1; o < (TR < 64 ? TR : 64); o <<= 1) total += __shfl_xor(total, o, 64);
  if (Q > 1) {
    part[rl][q][c] = sum;
    if (WPR > 1 && threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = total;
    __syncthreads();
    if (q > 0) return;
#pragma unroll
    for (int k = 1; k < Q; ++k) sum += part[rl][k][c];
    if (WPR > 1) {
      total = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) total += sums[w];
    }
  }
  if (!ok) return;
  if (total == total && (sum[0] != sum[0] || sum[1] != sum[1] || sum[2] != sum[2] || sum[3] != sum[3])) {
    // a range's infinity times a factor that 32 bits hold as 0: what the ranges have decides
    bool up[4] = {}, down[4] = {};
    for (int s = 0; s < of; ++s) {
      const f32x4 x = *(const f32x4*)(a.po + (at + s * step) * D + 4 * c);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        up[w] |= !(x[w] < INFINITY);
        down[w] |= !(x[w] > -INFINITY);
      }
    }
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (sum[w] != sum[w] && up[w] != down[w]) sum[w] = up[w] ? INFINITY : -INFINITY;
  }
  const int64_t to = ((int64_t)b * a.p.H + h * (a.p.H / a.p.Hkv)) * a.p.T + r;
  const float inv = row_factor(total);
  *(uint2*)((uint16_t*)a.p.out + to * D + 4 * c) = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
  if (a.p.lse && c == 0) a.p.lse[to] = row_log(top, total);
}

int tile_rows(int form) { return form >= 8 ? 128 : form == 1 || form == 3 ? 16 : 32; }
int64_t rows_of(const TreeProblem& p) { return (int64_t)p.H / p.Hkv * p.T; }

TreeArgs args_for(const TreeProblem& p, const TreePlan& pl, const void* ws) {
  TreeArgs a;
  a.p = p;
  a.pl = pl;
  a.po = (float*)ws;
  a.ml = (float2*)((char*)ws + (size_t)(pl.ranges + p.B) * p.Hkv * rows_of(p) * p.d * 4);
  a.info = (int2*)(a.ml + (size_t)(pl.ranges + p.B) * p.Hkv * rows_of(p));
  a.c = p.scale * 1.4426950408889634f;
  a.magic = (uint32_t)(65536 / std::min<int64_t>(p.page_rows, 65536) + 1);
  return a;
}

}  // namespace

TreePlan tree_plan(const TreeProblem& p) {
  TreePlan pl = {};
  const int64_t R = rows_of(p);
  // (With d = 128 the registers do not last for two blocks.)
  const bool four = p.page_rows % 4 == 0;
  pl.form = R <= 16 ? (four ? 3 : 1) : R <= 32 && p.d == 64 ? (four ? 4 : 2) : R < 64 ? 8 : 9;
  pl.tiles = (int)cdiv(R, tile_rows(pl.form));
  const int64_t S = std::min(p.M * p.page_rows, KEYS_MAX), units = p.Hkv * pl.tiles;
  // Few keys: one workgroup a request, key head and row tile takes all its keys, and nothing is left to join. (Of many
  // rows up to 512 keys, where that is more than a workgroup on every other CU: 188 of up to 388 keys 26 us -> 23, 480 of up to
  // 500 38 -> 33; 128 of up to 510 22 -> 23, 40 of them 19 -> 23.)
  const int64_t wgs = p.B * units;
  if (S <= 2 * UNIT || (wgs <= 512 && (pl.form < 8 ? S * p.d <= 1024 * 64 : wgs > 128 && S <= 512))) return pl;
  pl.ranges = std::max(cdiv(1024, units), p.B);
  pl.round = (int)(512 / units);
  return pl;
}

int64_t tree_workgroups(const TreeProblem& p, const TreePlan& pl) { return (pl.ranges + p.B) * p.Hkv * pl.tiles; }
size_t tree_bytes(const TreeProblem& p, const TreePlan& pl) {
  return pl.ranges ? (size_t)(pl.ranges + p.B) * p.Hkv * rows_of(p) * (p.d + 2) * 4 + p.B * sizeof(int2) : 0;
}

template <int D>
static void launch_d(const TreeArgs& a, unsigned grid, hipStream_t st) {
  if (a.pl.form == 1) k_tree<D, 1><<<grid, NT, 0, st>>>(a);
  else if (a.pl.form == 3) k_tree<D, 3><<<grid, NT, 0, st>>>(a);
  else if (D == 64 && a.pl.form == 2) k_tree<64, 2><<<grid, NT, 0, st>>>(a);
  else if (D == 64 && a.pl.form == 4) k_tree<64, 4><<<grid, NT, 0, st>>>(a);
  else if (a.pl.form == 8) k_tree<D, 8><<<grid, NT, 0, st>>>(a);
  else k_tree<D, 9><<<grid, NT, 0, st>>>(a);
}

hipError_t launch_tree(const TreeProblem& p, const TreePlan& pl, void* ws, hipStream_t st) {
  const TreeArgs a = args_for(p, pl, ws);
  const unsigned grid = (unsigned)tree_workgroups(p, pl);
  if (p.d == 64) launch_d<64>(a, grid, st);
  else launch_d<128>(a, grid, st);
  return hipGetLastError();
}

template <int D>
static void join_d(const TreeArgs& a, hipStream_t st) {
  // one row a workgroup while the rows leave CUs free
  constexpr int MANY = NT / (D / 4);
  const int64_t R = rows_of(a.p), lists = a.p.B * a.p.Hkv;
  if (lists * R <= 4096) k_tree_join<D, 1><<<(unsigned)(lists * R), NT, 0, st>>>(a);
  else k_tree_join<D, MANY><<<(unsigned)(lists * cdiv(R, MANY)), NT, 0, st>>>(a);
}

hipError_t launch_tree_join(const TreeProblem& p, const TreePlan& pl, const void* ws, hipStream_t st) {
  if (!pl.ranges) return hipSuccess;
  const TreeArgs a = args_for(p, pl, ws);
  if (p.d == 64) join_d<64>(a, st);
  else join_d<128>(a, st);
  return hipGetLastError();
}

}  // namespace topk
