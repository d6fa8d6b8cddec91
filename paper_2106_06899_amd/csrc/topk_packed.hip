// Attention over packed prompts: the tokens of n sequences lie one behind the other, a query sees the keys
// of its own sequence (causal: up to itself), out_i = sum_j softmax_j(scale q_i.k_j) v_j. G = H / Hkv query
// heads share a key head.
//
// A workgroup takes 128 tokens of one sequence and query head, 32 a wave; every wave takes every key tile of
// 64, K and V through LDS:
//   * S^T = K Q^T by v_mfma_f32_32x32x16_bf16: lane l holds 16 keys' scores of row l % 32 a 32-key
//     block, keys 8 (v / 4) + 4 (l / 32) + v % 4;
//   * a running softmax of each row in its two lanes;
//   * O^T += V^T P^T by the same instruction: the weights, rounded to bf16 (relative 2^-9 at most) and divided by
//     the sum of the rounded ones, in which what they have in common cancels, are its operand in the order
//     the lane holds them (TWO: as the sum of two bf16 numbers), V^T comes from the row-major tile by transposing LDS
//     reads.
// Tiles come by direct global-to-LDS loads, one ahead. Which sequence and tile a workgroup has it finds
// from the offsets itself, so that nothing is read back and no list is built by a launch of its own; there are at most
// N / 128 + n tiles a head, and those too many clear the tokens of no sequence.
// Bound by matrix and exponential instructions side by side: 16384 tokens, causal, 16 heads of 128 on 4: 1030 us,
// 1.07 PFLOP/s (a library's 8192^3 product: 1.12); 12 prompts of up to 3000 tokens 195.
#include "topk_packed_device.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace topk {
namespace {

constexpr int NT = 256, WAVES = 4;
#define TOPK_INLINE __attribute__((always_inline))  // (a lambda that is called captures through memory)

typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));
// c and eight bf16 numbers
__device__ __forceinline__ float sum_of(const bf16x8& x, float c) {
  typedef bf16x2 pairs[4];
  pairs p;
  __builtin_memcpy(p, &x, sizeof x);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_fdot2_f32_bf16(p[e], (bf16x2){(__bf16)1.f, (__bf16)1.f}, c, false);
  return c;
}

struct PackedArgs {
  PackedProblem p;
  float c;  // scale * log2(e)
};

// LSE: the logarithm of the sum is asked for, so that the weights are summed before rounding, too. KS = 2: half the
// rows a workgroup, and two waves share each 32, one taking the first and one the last 32 keys of every tile: twice
// the workgroups, each of half the length, where there are few.
template <int D, bool CAUSAL, bool LSE, int KS, bool TWO>
__global__ __launch_bounds__(NT, 2) void k_packed(PackedArgs a) {
  // The maximum that weights are taken against is moved, and the sums with it, only once a score leads it
  // by 2^8 in weight.
  constexpr float LEAD = 8.f;
  typedef PackedTile<D> Tile;
  constexpr int ROWS = PACKED_TILE / KS;  // of the workgroup
  constexpr int KEYS = 64;          // of a tile
  constexpr int NB = 2 / KS;        // blocks of 32 of a tile that a wave takes
  constexpr int NS = D / 16;        // steps over the features of the scores
  constexpr int CH = 2 * D / 16;    // 16-byte parts of a row
  constexpr int TILEB = KEYS * 2 * D;
  constexpr int LPW = TILEB / 1024 / WAVES;
  constexpr int FB = D / 32;        // 32-feature blocks of the output
  constexpr int AHEAD_K = 6, AHEAD_V = 4;  // products by which LDS reads run ahead of their use
  __shared__ __attribute__((aligned(16))) unsigned char k0[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char k1[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char v0[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char v1[TILEB];
  __shared__ float flag[WAVES][2];

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
  const int group = wave % (WAVES / KS), share = wave / (WAVES / KS);  // of rows; of a tile's keys
  const int2 item = packed_item(a.p.H);
  const int h = item.x;
  int all = 0;
  const PackedPlace at = packed_place(a.p, item.y, ROWS, a.p.H, CAUSAL, false, &all);
  if (!at.n) {  // the workgroups of a head that have no tile share the tokens of no sequence
    const int N = (int)a.p.N, z0 = min(max(a.p.offsets[0], 0), N), z1 = max(z0, min(max(a.p.offsets[a.p.n], 0), N));
    const int64_t parts = (int64_t)(z0 + N - z1) * CH, step = (int64_t)(gridDim.x / a.p.H - all) * NT;
    for (int64_t i = (int64_t)(item.y - all) * NT + tid; i < parts; i += step) {
      const int64_t r = i / CH, t = r < z0 ? r : r - z0 + z1;
      const int64_t e = h * a.p.out.head + t * a.p.out.token + i % CH * 8;
      *(uint4*)((uint16_t*)a.p.out.p + e) = make_uint4(0, 0, 0, 0);
      if (a.p.rest) *(uint4*)((uint16_t*)a.p.rest + e) = make_uint4(0, 0, 0, 0);
      if (a.p.lse && i % CH == 0) a.p.lse[h * a.p.N + t] = -INFINITY;
    }
    return;
  }
  const int hk = h / (a.p.H / a.p.Hkv);
  const int row = at.tile * ROWS + group * 32 + n;  // the lane's query in its sequence
  const bool ok = row < at.n;
  const bool work = at.tile * ROWS + group * 32 < at.n;  // the wave has rows
  bf16x8 bq[NS];
  {
    const uint16_t* q = (const uint16_t*)a.p.q.p + h * a.p.q.head + (at.first + (ok ? row : at.n - 1)) * a.p.q.token + (D / 2) * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) bq[s] = *(const bf16x8*)(q + 8 * s);
  }
  f32x16 o[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) o[f] = (f32x16){};
  float m = -INFINITY, l = 0.f, whole_l = 0.f;  // sums of the weights as they are multiplied; as they are
  const uint32_t kbase = Tile::straight_base(), vbase = Tile::across_base();

  // keys that some row of the workgroup sees; those that every row sees; those that the lane's does
  const int keys = CAUSAL ? min(at.n, at.tile * ROWS + ROWS) : at.n;
  const int all_see = CAUSAL ? at.tile * ROWS + 1 : at.n, seen = CAUSAL ? min(at.n, row + 1) : at.n;
  const int wave_keys = (CAUSAL ? at.tile * ROWS + group * 32 + 32 : at.n) - share * 32;  // its rows see none of a tile from here on
  const int tiles = (keys + KEYS - 1) / KEYS;
  const uint32_t ksl = (uint32_t)a.p.k.token * 2, vsl = (uint32_t)a.p.v.token * 2;  // bytes from one row to the next
  uint32_t koff[LPW], voff[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int cidx = (wave * LPW + j) * 64 + lane, r = cidx / CH, c = cidx % CH ^ Tile::swz(r);
    koff[j] = r * ksl + c * 16;
    voff[j] = r * vsl + c * 16;
  }
  const unsigned char* kt = (const unsigned char*)((const uint16_t*)a.p.k.p + hk * a.p.k.head + at.first * a.p.k.token);
  const unsigned char* vt = (const unsigned char*)((const uint16_t*)a.p.v.p + hk * a.p.v.head + at.first * a.p.v.token);
  auto issue = [&](int t, unsigned char* kd, unsigned char* vd) {
    const int left = min(KEYS, keys - t * KEYS) - 1;
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      uint32_t ko = koff[j], vo = voff[j];
      if (left < KEYS - 1) {  // rows past the last key load it
        const int r = ((wave * LPW + j) * 64 + lane) / CH, over = r - min(r, left);
        ko -= over * ksl;
        vo -= over * vsl;
      }
      __builtin_amdgcn_global_load_lds((const void*)(kt + ko), (TOPK_LDS void*)&kd[(wave * LPW + j) * 1024], 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const void*)(vt + vo), (TOPK_LDS void*)&vd[(wave * LPW + j) * 1024], 16, 0, 0);
    }
    kt += KEYS * (int64_t)ksl;
    vt += KEYS * (int64_t)vsl;
  };

  auto tile = [&](auto edge, int t, const unsigned char* kbuf, const unsigned char* vbuf) TOPK_INLINE {
    const TOPK_LDS unsigned char *kb = (const TOPK_LDS unsigned char*)kbuf + (KS > 1 ? share * 32 * 2 * D : 0),
                                 *vb = (const TOPK_LDS unsigned char*)vbuf + (KS > 1 ? share * 32 * 2 * D : 0);
    constexpr int SV = 16 * NB;  // scores of a lane
    f32x16 s[NB] = {};
    {
      bf16x8 kf[AHEAD_K + 1];
      auto kp = [&](int i) { return Tile::straight(kb, kbase, i % NB, i / NB); };
#pragma unroll
      for (int i = 0; i < AHEAD_K; ++i) kf[i] = kp(i);
#pragma unroll
      for (int i = 0; i < NB * NS; ++i) {
        if (i + AHEAD_K < NB * NS) kf[(i + AHEAD_K) % (AHEAD_K + 1)] = kp(i + AHEAD_K);
        s[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % (AHEAD_K + 1)], bq[i / NB], s[i % NB], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    float low = INFINITY;  // the tile's lowest score (masked keys' included, NaN too: they only choose the pass below)
#pragma unroll
    for (int v = 0; v < SV; v += 2)
      low = __builtin_elementwise_minimum(__builtin_elementwise_minimum(low, s[v >> 4][v & 15]), s[v >> 4][(v & 15) + 1]);
    if (decltype(edge)::value) {
      const int last = seen - t * KEYS - share * 32 - 4 * half;
#pragma unroll
      for (int v = 0; v < SV; ++v)
        if ((v >> 4) * 32 + 8 * ((v & 15) >> 2) + (v & 3) >= last) s[v >> 4][v & 15] = -INFINITY;
    }
    float mt = -INFINITY;
#pragma unroll
    for (int v = 0; v < SV; v += 2)
      mt = larger(larger(mt, s[v >> 4][v & 15]), s[v >> 4][(v & 15) + 1]);
    mt = other_half_max(mt) * a.c;
    const bool leads = !(mt <= m + LEAD);  // (NaN too)
    if (__builtin_amdgcn_ballot_w64(leads)) {  // (the other rows multiply by 1: a row's result is its own)
      const float mn = leads ? larger(m, mt) : m;
      const float alpha = mn == -INFINITY ? 1.f : exp2f(m - mn);  // (below 2^-126 too: see the weights)
      m = mn;
      l *= alpha;
      if (LSE) whole_l *= alpha;
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[f][v] *= alpha;
    }
    constexpr int VM = 2 * NB * FB;
    const float off = m == -INFINITY ? 0.f : m;
    auto vp = [&](int j) { return Tile::across(vb, vbase, j % FB, j / FB); };  // V^T of 16 keys j / FB, features 32 (j % FB) on
    // Weights below 2^-126, which the exponential instruction alone makes 0, are added by themselves where
    // the tile has any.
    if (__builtin_amdgcn_ballot_w64(!(fmaf(low, a.c, -off) >= -126.f))) {
      float bias = -off;
      asm volatile("" : "+v"(bias));  // (nothing of this pass is held for the other)
#pragma unroll
      for (int st = 0; st < 2 * NB; ++st) {
        bf16x8 pt;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = fmaf(s[st >> 1][8 * (st & 1) + e], a.c, bias), w = x < -126.f ? exp2f(x) : 0.f;
          if (LSE) whole_l += w;
          pt[e] = (__bf16)w;
        }
        if (!TWO) l = sum_of(pt, l);
#pragma unroll
        for (int f = 0; f < FB; ++f) {
          o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp(st * FB + f), pt, o[f], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    bf16x8 pb[2 * NB], pl[2 * NB], vf[AHEAD_V + 1];
#pragma unroll
    for (int j = 0; j < AHEAD_V; ++j) vf[j] = vp(j);
    __builtin_amdgcn_s_setprio(1);  // the other wave's softmax yields to this one's products
    auto wt = [&](int v) {
      const float w = __builtin_amdgcn_exp2f(fmaf(s[v >> 4][v & 15], a.c, -off));
      if (LSE) whole_l += w;
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
      if (!TWO && j % FB == 0) l = sum_of(pb[j / FB], l);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // One tile of lookahead: before tile t is read, this wave's loads of it are complete and the barrier
  // publishes every wave's part; it also proves that no wave still reads the buffers the next loads
  // overwrite. (The buffers are named at compile time, so that reads of one pair do not wait for loads
  // into the other.) Tiles that every row sees whole come first and need no mask.
  const int whole = min(keys, all_see) / KEYS;
  auto ready = [&](int t, unsigned char* kn, unsigned char* vn) {
    __builtin_amdgcn_s_waitcnt(PACKED_WAIT_VM0);
    __syncthreads();
    if (t + 1 < tiles) issue(t + 1, kn, vn);
  };
  issue(0, k0, v0);
  int t = 0;
  for (; t + 1 < whole; t += 2) {
    ready(t, k1, v1);
    if (work) tile(std::false_type{}, t, k0, v0);
    ready(t + 1, k0, v0);
    if (work) tile(std::false_type{}, t + 1, k1, v1);
  }
  // Where rows of the workgroup do not see all its keys, values that are not finite go only to the rows that
  // see theirs, which become NaN there (and infinite, where they are, at the end); the others would meet them as 0
  // times NaN. Each wave looks at its part of the tile.
  constexpr bool hides = CAUSAL;
  auto own_part = [&](unsigned char* vb, int j) { return (TOPK_LDS u32x4*)&vb[(wave * LPW + j) * 1024 + lane * 16]; };
  for (; t < tiles; ++t) {
    const bool odd = t & 1;
    unsigned char* vb = odd ? v1 : v0;
    if (hides) {
      __builtin_amdgcn_s_waitcnt(PACKED_WAIT_VM0);
      uint32_t bad = 0;
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        const u32x4 x = *own_part(vb, j);
        bad |= not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3]);
      }
      const bool any = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
      if (lane == 0) flag[wave][t & 1] = any ? 1.f : 0.f;  // (read before the next barrier; the next tile's is another)
    }
    ready(t, odd ? k0 : k1, odd ? v0 : v1);
    if (hides && flag[0][t & 1] + flag[1][t & 1] + flag[2][t & 1] + flag[3][t & 1] > 0.f) {
#pragma unroll 1
      for (int j = 0; j < KEYS; ++j) {
        const bool sees = j < seen - t * KEYS;
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const TOPK_LDS uint32_t* x = (const TOPK_LDS uint32_t*)&vb[j * 2 * D + ((4 * f + v / 4) ^ Tile::swz(j)) * 16 + 8 * half];
#pragma unroll
            for (int w = 0; w < 4; ++w)
              if (sees && (not_finite(x[w / 2]) >> 16 * (w & 1) & 1)) o[f][v + w] = NAN;
          }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        u32x4 x = *own_part(vb, j);
#pragma unroll
        for (int w = 0; w < 4; ++w) x[w] &= ~(not_finite(x[w]) * 0xFFFFu);
        *own_part(vb, j) = x;
      }
      __syncthreads();
    }
    if (work && t * KEYS < wave_keys) tile(std::true_type{}, t, odd ? k1 : k0, odd ? v1 : v0);
  }
  if (TWO) l = whole_l;
  l += __shfl_xor(l, 32, 64);
  if (LSE) whole_l += __shfl_xor(whole_l, 32, 64);
  __syncthreads();
  TOPK_LDS unsigned char *p0 = (TOPK_LDS unsigned char*)k0, *p1 = (TOPK_LDS unsigned char*)k1, *p2 = (TOPK_LDS unsigned char*)v0,
                         *p3 = (TOPK_LDS unsigned char*)v1;
  if (KS > 1) {  // the second half of the waves hand theirs over: four numbers a lane at a time, then maximum and sums
    TOPK_LDS f32x4* to = (TOPK_LDS f32x4*)(group ? p1 : p0) + lane;
    __shared__ float2 other[WAVES][64];
    __shared__ float other_l[WAVES][64];
    if (share) {
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int v = 0; v < 16; v += 4) to[(4 * f + v / 4) * 64] = (f32x4){o[f][v], o[f][v + 1], o[f][v + 2], o[f][v + 3]};
      other[group][lane] = make_float2(m, l);
      if (LSE) other_l[group][lane] = whole_l;
    }
    __syncthreads();
    if (share) return;
    const float2 x = other[group][lane];
    const float top = larger(m, x.x), base = top == -INFINITY ? 0.f : top, f0 = exp2f(m - base), f1 = exp2f(x.x - base);  // (-inf: 0)
    m = top;
    l = fmaf(f0, l, f1 * x.y);
    if (LSE) whole_l = fmaf(f0, whole_l, f1 * other_l[group][lane]);
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const f32x4 y = to[(4 * f + v / 4) * 64];
#pragma unroll
        for (int w = 0; w < 4; ++w) o[f][v + w] = fmaf(f0, o[f][v + w], f1 * y[w]);
      }
    wave_sync_lds();
  }
  float most = o[0][0];  // NaN where any of the sums is: rows that are written once more (see Infinities)
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int v = 0; v < 16; v += 2) most = larger(larger(most, o[f][v]), o[f][v + 1]);
  // through the wave's own part of LDS, in parts of four features permuted by the row, so that whole rows
  // are written, two (D = 128) or four a store
  TOPK_LDS f32x4* mine = (TOPK_LDS f32x4*)(KS > 1 ? group ? p1 : p0 : wave == 0 ? p0 : wave == 1 ? p1 : wave == 2 ? p2 : p3);
  constexpr int PARTS = D / 4, RPS = 64 / PARTS;
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      mine[n * PARTS + ((8 * f + v / 2 + half) ^ (n & 15))] = (f32x4){o[f][v], o[f][v + 1], o[f][v + 2], o[f][v + 3]};
  wave_sync_lds();
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int part = lane % PARTS;
  uint16_t* to = (uint16_t*)a.p.out.p + h * a.p.out.head + at.first * a.p.out.token + 4 * part;
  constexpr int SU = 32 / RPS;  // stores
  auto sums = [&](int u) TOPK_INLINE {
    const int r = u * RPS + lane / PARTS;
    return mine[r * PARTS + (part ^ (r & 15))];
  };
  auto store = [&](int u, const f32x4& x) TOPK_INLINE {
    const int r = u * RPS + lane / PARTS, i = at.tile * ROWS + group * 32 + r;
    const float by = __shfl(inv, r, 64);
    if (i >= at.n) return;
    const uint2 y = make_uint2(pack_bf16(x[0] * by, x[1] * by), pack_bf16(x[2] * by, x[3] * by));
    *(uint2*)(to + i * a.p.out.token) = y;
    if (a.p.rest)  // (nothing was taken from what is not finite)
      *(uint2*)((uint16_t*)a.p.rest + (to - (uint16_t*)a.p.out.p) + i * a.p.out.token) =
          make_uint2(pack_bf16(x[0] * by - __uint_as_float(y.x << 16), x[1] * by - __uint_as_float(y.x & 0xFFFF0000u)) & ~(not_finite(y.x) * 0xFFFFu),
                     pack_bf16(x[2] * by - __uint_as_float(y.y << 16), x[3] * by - __uint_as_float(y.y & 0xFFFF0000u)) & ~(not_finite(y.y) * 0xFFFFu));
  };
#pragma unroll 4
  for (int u = 0; u < SU; ++u) store(u, sums(u));
  if (__builtin_amdgcn_ballot_w64(most != most)) {
    Infinities<D, SU> is;
    const int ln = is.own_lane(), row0 = at.tile * ROWS + group * 32 + ln / PARTS;  // the lane's row of the first store
#pragma unroll 1
    for (int u = 0; u < SU; ++u) {
      const float by = __shfl(inv, u * RPS + ln / PARTS, 64);
      is.nan(u, sums(u), row0 + u * RPS < at.n && by == by);
    }
    constexpr int LOOKS = 4, LR = Infinities<D, SU>::ROWS;
    const uint16_t* v = (const uint16_t*)a.p.v.p + hk * a.p.v.head + at.first * a.p.v.token + ln % CH * 8;
    for (int j0 = 0; j0 < keys && is.unsettled(); j0 += LOOKS * LR) {
      u32x4 x[LOOKS];
#pragma unroll
      for (int e = 0; e < LOOKS; ++e) x[e] = *(const u32x4*)(v + min(j0 + e * LR + ln / CH, keys - 1) * a.p.v.token);
#pragma unroll
      for (int e = 0; e < LOOKS; ++e)
        is.look(ln, x[e], [&](int k, int u) TOPK_INLINE {
          const int j = j0 + e * LR + k;
          return j < keys && (!CAUSAL || j <= row0 + u * RPS);
        });
    }
#pragma unroll 1
    for (int u = 0; u < SU; ++u) {
      f32x4 x = sums(u);
      is.settle(u, x);
      store(u, x);
    }
  }
  if (LSE && ok && !half) a.p.lse[h * a.p.N + at.first + row] = whole_l == 0.f ? -INFINITY : (m + log2f(whole_l)) * 0.69314718055994531f;
}

// In a training pass (rest is asked for) over heads of 64, or a short one, weights are two numbers: the D of the
// backward pass is as exact as they are. (Heads of 64: dQ is off by 1.46 times its own rounding, from rounded weights
// by 1.50; heads of 128: 1.44 and 1.47, for 7 % of a pass.)
bool packed_two(const PackedProblem& p) { return p.rest && p.lse && (p.d == 64 || packed_short(p)); }

template <bool LSE, int KS, bool TWO>
void launch_for(const PackedArgs& a, unsigned grid, hipStream_t st) {
  if (a.p.d == 64 && a.p.causal) k_packed<64, true, LSE, KS, TWO><<<grid, NT, 0, st>>>(a);
  else if (a.p.d == 64) k_packed<64, false, LSE, KS, TWO><<<grid, NT, 0, st>>>(a);
  else if (a.p.causal) k_packed<128, true, LSE, KS, TWO><<<grid, NT, 0, st>>>(a);
  else k_packed<128, false, LSE, KS, TWO><<<grid, NT, 0, st>>>(a);
}
template <int KS>
void launch_ks(const PackedArgs& a, unsigned grid, hipStream_t st) {
  if (packed_two(a.p)) launch_for<true, KS, true>(a, grid, st);
  else if (a.p.lse) launch_for<true, KS, false>(a, grid, st);
  else launch_for<false, KS, false>(a, grid, st);
}

}  // namespace

int64_t packed_tiles(const PackedProblem& p, int rows) { return p.N / rows + std::min<int64_t>(p.n, p.N) + 1; }

// (One text of 8192 tokens, heads of 128, causal: 2 heads 141 -> 98 us, 4 142 -> 105, 8 170 either way, 16 268 -> 315; all
// keys, 8 heads 259 -> 302.)
bool packed_few(const PackedProblem& p, int heads) { return p.N / PACKED_TILE * heads <= 256; }

bool packed_short(const PackedProblem& p) { return p.N <= 1024 || p.N <= 64 * (int64_t)p.n; }

hipError_t launch_packed(const PackedProblem& p, hipStream_t st) {
  PackedArgs a = {p, p.scale * 1.4426950408889634f};
  const bool few = packed_few(p, p.H);
  const unsigned grid = (unsigned)(packed_tiles(p, few ? PACKED_TILE / 2 : PACKED_TILE) * p.H);
  if (few) launch_ks<2>(a, grid, st);
  else launch_ks<1>(a, grid, st);
  return hipGetLastError();
}

}  // namespace topk
