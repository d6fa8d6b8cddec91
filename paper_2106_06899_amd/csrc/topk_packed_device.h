// Shared by the forward and the backward pass of packed attention: which rows a workgroup takes, and how
// tiles of rows come to LDS and are read there.
#pragma once

#include "topk_device.h"
#include "topk_packed.h"

#include <math.h>

namespace topk {

#define TOPK_LDS __attribute__((address_space(3)))
typedef float f32x16 __attribute__((__vector_size__(64)));
typedef short s16x4 __attribute__((__vector_size__(8)));
typedef uint32_t u32x4 __attribute__((__vector_size__(16)));
typedef TOPK_LDS s16x4 lds_s16x4;

// s_waitcnt immediate: no vector-memory operation outstanding, the other counters ignored
constexpr int PACKED_WAIT_VM0 = (7 << 4) | (15 << 8);

// the larger, and NaN where either is
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }
// the larger of x and what the lane 32 away holds
__device__ __forceinline__ float other_half_max(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
// Of two bf16 numbers, bit 0 and bit 16: is it infinite or NaN?
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return (((x & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u; }

// Sums that are NaN though their rows' weights are numbers. By the definition an infinite value whose weight is above 0
// makes a sum infinite, values of both signs, or one that is NaN, make it NaN; the products have it as NaN wherever a
// part of a weight is 0 (0 times infinity), so the values are looked at again, by the whole wave for its rows: as they
// lie in memory, 16 bytes a lane. (32768 causal tokens, 12 heads of 64, training: 2.69 ms, 3.58 where all see an infinite
// value.) A lane has features 4 (lane % (D / 4)) .. of U rows; bit 4 u + w of these is of the w-th of row u.
template <int D, int U>
struct Infinities {
  uint64_t open = 0, up = 0, down = 0;  // sums that are NaN; that meet +infinity or NaN; -infinity or NaN
  static_assert(U <= 16, "four bits a row");
  static constexpr int PARTS = D / 8, ROWS = 64 / PARTS;  // 16-byte parts of a row of values; rows of a look

  __device__ __forceinline__ void nan(int u, const f32x4& x, bool row) {
#pragma unroll
    for (int w = 0; w < 4; ++w) open |= (uint64_t)(row && x[w] != x[w]) << (4 * u + w);
  }
  // is there a sum that may yet turn out to be infinite?
  __device__ __forceinline__ bool unsettled() const { return __builtin_amdgcn_ballot_w64((open & ~(up & down)) != 0) != 0; }
  // lane: of the wave, formed anew, so that nothing that follows from it is held from above, where registers are few
  static __device__ __forceinline__ int own_lane() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
  }
  // x: the lane's part lane % PARTS of row lane / PARTS of ROWS; sees(k, u): does row u see the k-th of them?
  template <typename F>
  __device__ __forceinline__ void look(int lane, const u32x4& x, F sees) {
    const int part = lane % (D / 4);
    uint64_t hits = __builtin_amdgcn_ballot_w64((not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3])) != 0);
    while (hits) {
      const int b = __builtin_ctzll(hits);
      hits &= hits - 1;
      auto of = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)x[i], b); };
      const uint32_t y0 = of(0), y1 = of(1), y2 = of(2), y3 = of(3), lo = part & 1 ? y2 : y0, hi = part & 1 ? y3 : y1;
      uint64_t rises = 0, falls = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t h = (w < 2 ? lo : hi) >> 16 * (w & 1) & 0xFFFFu;
        const bool odd = part >> 1 == b % PARTS && (h & 0x7F80u) == 0x7F80u, is_nan = h & 0x7Fu;
        rises |= (uint64_t)(odd && (is_nan || !(h >> 15))) << w;
        falls |= (uint64_t)(odd && (is_nan || h >> 15)) << w;
      }
#pragma unroll 1
      for (int u = 0; u < U; ++u)
        if (sees(b / PARTS, u)) {
          up |= rises << 4 * u;
          down |= falls << 4 * u;
        }
    }
  }
  __device__ __forceinline__ void settle(int u, f32x4& x) const {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if ((open & (up ^ down)) >> (4 * u + w) & 1) x[w] = up >> (4 * u + w) & 1 ? INFINITY : -INFINITY;
  }
};

// A workgroup's tile: tile `tile` of the sequence of n tokens from token `first` on; n = 0: none.
struct PackedPlace {
  int64_t first;
  int n, tile;
};

__device__ __forceinline__ uint32_t wave_sum(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan_full(x), 63); }

// Where the interval of 256 threads' counts `mine`, laid one behind the other from `before` on, holds number t: true for
// the thread whose it is, with the numbers before its first. *before becomes the number behind the last. By the whole
// workgroup; `sums`: an entry a wave.
__device__ __forceinline__ bool block_find(uint32_t mine, uint32_t t, uint32_t* before, uint32_t* first, uint32_t* sums) {
  const int wave = threadIdx.x >> 6;
  const uint32_t end = wave_incl_scan_full(mine);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sums[wave] = end;
  __syncthreads();
  uint32_t at = *before;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) at += sums[w];
    *before += sums[w];
  }
  *first = at + end - mine;
  return t >= *first && t - *first < mine;
}

// Tile number t of all sequences' tiles of `rows` tokens. levels: up to 64 sequences' tiles are numbered by
// their place in their sequence, the last places (or, from_end, the first) first: under a causal mask these
// have the most to do. Every wave finds it by itself; more sequences are looked through by the whole workgroup, four a
// thread. *tiles, for a workgroup without a tile: how many there are.
__device__ __forceinline__ PackedPlace packed_place(const PackedProblem& p, int t, int rows, int heads, bool levels, bool from_end,
                                                    int* tiles = nullptr) {
  const int lane = threadIdx.x & 63;
  PackedPlace at = {0, 0, 0};
  auto bounds = [&](int s, int* a, int* len) {
    const int N = (int)p.N;
    *a = min(max(p.offsets[s], 0), N);
    *len = min(max(p.offsets[s + 1], 0), N) - *a;
    if (*len < 0) *len = 0;
  };
  int s = -1;
  if (p.n <= 64) {
    int a, len = 0;
    if (lane < p.n) bounds(lane, &a, &len);
    const int nt = (len + rows - 1) / rows;
    if (levels) {
      auto longer = [&](int c) { return (int)wave_sum((uint32_t)max(nt - c, 0)); };  // tiles in places from c on
      const int all = longer(0);
      if (tiles) *tiles = all;
      if (all <= t) return at;
      // Where every CU has one or two workgroups in all, those that come second are the shortest first: the longest
      // shares its CU with the shortest.
      if (all * heads <= 512 && t * heads >= 256) t = all - 1 - (t - (256 + heads - 1) / heads);
      int lo = 0, hi = (int)((p.N + rows - 1) / rows);  // longer(lo) > t >= longer(hi)
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (longer(mid) > t) lo = mid;
        else hi = mid;
      }
      const uint64_t those = __builtin_amdgcn_ballot_w64(nt > lo);
      const int r = t - longer(lo + 1);
      s = __builtin_ctzll(__builtin_amdgcn_ballot_w64(nt > lo && (int)lanes_below(those) == r));
      at.tile = lo;
    } else {
      const uint32_t end = wave_incl_scan_full((uint32_t)nt);
      const uint64_t those = __builtin_amdgcn_ballot_w64(end > (uint32_t)t);
      if (tiles) *tiles = __builtin_amdgcn_readlane((int)end, 63);
      if (!those) return at;
      s = __builtin_ctzll(those);
      at.tile = t - (__builtin_amdgcn_readlane((int)end, s) - __builtin_amdgcn_readlane(nt, s));
    }
  } else {
    __shared__ uint32_t sums[4];
    __shared__ int found[2];
    if (threadIdx.x == 0) found[0] = -1;
    uint32_t before = 0;
    for (int64_t s0 = 0; s0 < p.n && before <= (uint32_t)t; s0 += 1024) {
      int nt[4], a, len;
      uint32_t mine = 0, first;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t x = s0 + 4 * threadIdx.x + u;
        len = 0;
        if (x < p.n) bounds((int)x, &a, &len);
        mine += nt[u] = (len + rows - 1) / rows;
      }
      if (block_find(mine, (uint32_t)t, &before, &first, sums)) {
        uint32_t left = t - first;
        int u = 0;
#pragma unroll
        for (int w = 0; w < 3; ++w)
          if (u == w && left >= (uint32_t)nt[w]) {
            left -= nt[w];
            u = w + 1;
          }
        found[0] = (int)(s0 + 4 * threadIdx.x) + u;
        found[1] = (int)left;
      }
    }
    __syncthreads();
    s = found[0];
    if (tiles) *tiles = (int)min(before, (uint32_t)t);  // (t at most, whatever the offsets)
    if (s < 0) return at;
    at.tile = found[1];
  }
  int a, len;
  bounds(s, &a, &len);
  at.first = __builtin_amdgcn_readfirstlane(a);
  at.n = __builtin_amdgcn_readfirstlane(len);
  at.tile = __builtin_amdgcn_readfirstlane(at.tile);
  if (levels && p.n <= 64 && from_end) at.tile = (at.n + rows - 1) / rows - 1 - at.tile;
  return at;
}

// The head and tile number of a workgroup: all heads of a tile number before the next, so that the long
// tiles of every head start first; where 8 divides the heads, an XCD (every eighth workgroup) takes
// neighbouring ones, which share key heads.
__device__ __forceinline__ int2 packed_item(int heads) {
  const int t = blockIdx.x / heads, r = blockIdx.x % heads;
  return make_int2(heads % 8 == 0 ? (r % 8) * (heads / 8) + r / 8 : r, t);
}

// A tile of KEYS rows of D features in LDS, as it lies in memory but for its rows' 16-byte parts, part c of
// row r at place c ^ swz(r): sixteen rows' equal parts lie in different banks, for reads of whole parts, and four
// rows' equal halves of pairs of parts, for transposing reads.
template <int D>
struct PackedTile {
  static constexpr int CH = 2 * D / 16;  // parts of a row
  static __device__ __forceinline__ int swz(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
  // Where the lane's reads lie, in bytes from the tile's first: one number each, from which the others
  // follow by flipping bits, since swz is linear in the bits of a row's number.
  // Straight: features (D / 2) (lane / 32) + 8 i .. + 7 of row 32 rb + lane % 32, for i and rb that are known.
  static __device__ __forceinline__ uint32_t straight_base() {
    const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
    return n * 2 * D + ((half * (D / 16)) ^ swz(n)) * 16;
  }
  static __device__ __forceinline__ bf16x8 straight(const TOPK_LDS unsigned char* b, uint32_t base, int rb, int i) {
    return *(const TOPK_LDS bf16x8*)(b + (base ^ (i * 16)) + rb * 32 * 2 * D);
  }
  // Transposed: feature 32 f + lane % 32 of rows 16 j + 8 (e / 4) + 4 (lane / 32) + e % 4.
  static __device__ __forceinline__ uint32_t across_base() {
    const int lane = threadIdx.x & 63, va = lane & 15, r = 4 * (lane >> 5) + (va >> 2);
    return r * 2 * D + (((((lane >> 4) & 1) * 2 + ((va & 3) >> 1)) ^ swz(r)) * 16) + (va & 1) * 8;
  }
  static __device__ __forceinline__ bf16x8 across(const TOPK_LDS unsigned char* b, uint32_t base, int f, int j) {
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(b + (base ^ (f * 64) ^ (swz(16 * j) * 16)) + 16 * j * 2 * D));
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(b + (base ^ (f * 64) ^ (swz(16 * j + 8) * 16)) + (16 * j + 8) * 2 * D));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

}  // namespace topk
