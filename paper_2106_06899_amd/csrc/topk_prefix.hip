// Attention of a batch whose requests share a long prefix: every row attends to the prefix
// (P keys and values of each key head, one copy for all requests) and to its own request's
// cache, out_i = sum_j softmax_j(scale q_i.k_j) v_j over both. G = H / Hkv query heads share a
// key head.
//
// The prefix is read once for a tile of rows of all requests, not once a request: the rows
// (request, query head of the group, token) of one key head are one long list for the prefix,
// and one short list a request for the caches. A workgroup takes one row tile and one key
// range, of the prefix or of one cache, and leaves a partial result (the maximum, the sum and
// the unnormalised output, all in 32 bits) which a second kernel joins; where there is one
// range in all, it writes the output itself. Both kinds of workgroup run in one launch, so that
// the prefix's products and the caches' reads overlap. Requests with many rows of their own take
// prefix and cache as one list of keys instead, which leaves fewer partial results.
//
// Row tiles come in two forms. Few (up to 32 rows) keeps K and V in registers and is bound by
// reading them: 8 requests behind 65536 keys, 16 heads of 128, read 571 MB in 98 us (5.8 TB/s; a
// device copy: 4.94). Wide (128 rows) goes through LDS and is bound by matrix and vector
// instructions, which run side by side: 4 requests of 512 tokens, 16
// heads of 128 on 4 key heads behind 16384 keys, 277 us with the join, 1.0 PFLOP/s (a large
// library matrix product: 1.38). Short calls are bound by launches and latency, and by the partial
// results, whose join is a launch of its own: 64 requests behind 8192 keys, 32 heads of 128 on 8, 28 +
// 6 us, where the bytes would take 23. Calls with few keys in all take one range instead.
//
// Few rows. Four waves take key tiles of 32 in turn, each with a running softmax of its own, joined
// through LDS at the end. Scores are S^T = K Q^T and the output O^T = V^T P^T by
// v_mfma_f32_16x16x32_bf16, so that a lane holds scores, weights and outputs of one row
// (lane % 16): the weights of 32 keys are the second product's operand as they stand. K and V go
// from memory to registers: a lane's part of K is the first product's operand as it lies in
// memory, V is read in whole rows (8 keys x D / 16 columns a lane) and paired up by byte
// permutes. Keys of the next tile are loaded while the softmax runs, values while the next
// scores are formed. Weights enter the second product as the sum of two bf16 numbers (16
// significant bits), which costs little where the keys' memory is the bound.
#include "topk_device.h"
#include "topk_prefix.h"

#include <math.h>

#include <algorithm>

namespace topk {
namespace {

int64_t cdiv(int64_t x, int64_t y) { return (x + y - 1) / y; }

constexpr int NT = 256, WAVES = 4, KT = 32;
constexpr int JOIN_MAX = 1024;  // key ranges of a row at most,
constexpr int JOIN_FEW = 16;    // where a workgroup joins several rows
constexpr int64_t RANGE_MAX = int64_t(1) << 30;  // keys of a range (their numbers, and rows on top, are 32 bits)
// s_waitcnt immediate: no vector-memory operation outstanding, the other counters ignored
constexpr int WAIT_VM0 = (7 << 4) | (15 << 8);

struct PrefixArgs {
  PrefixProblem p;
  PrefixPlan pl;
  float* po;   // [splits][rows][D]
  float2* ml;  // [splits][rows]: maximum of the scaled scores (to base 2), sum of weights
  float c;     // scale * log2(e)
};

// the larger, and NaN where either is (a row whose scores hold one is NaN, no other)
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }
// a row's factor and its logarithm (to base e) from the sum of its weights, 0 where it saw no key, and the
// maximum that they were taken against (to base 2)
__device__ __forceinline__ float row_factor(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }
__device__ __forceinline__ float row_log(float top, float sum) {
  return sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
}

// Of two bf16 numbers, bit 0 and bit 16: is it infinite or NaN?
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return (((x & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u; }

// A range of keys, of the prefix or of a request's own.
struct Span {
  const uint16_t *k, *v;  // its first
  uint32_t k_sl, v_sl;    // elements from one to the next
  int n;                  // keys
  int before;             // (own:) keys of the request before the first one that the row of token 0 does
                          // not see, from the range's first on; may be negative or beyond n
};

// One work item: rows from r0 of a list of `count` against keys of the prefix, of a request, or both.
struct Item {
  Span prefix, own;
  int r0, count;
  int h;      // key head
  int b;      // request (-1: rows of all requests, against the prefix)
  int split;  // where its partial result goes
};

// A workgroup's LDS: four tile buffers (the few-row form keeps a wave's outputs in each), and the
// waves' maxima and sums.
// (The few-row form picks its buffer by an LDS address: a generic one would make flat accesses.)
#define TOPK_LDS __attribute__((address_space(3)))
struct Lds {
  unsigned char *b0, *b1, *b2, *b3;
  float2 (*ml)[32], *sum;
  int64_t* row;
  __device__ TOPK_LDS unsigned char* of(int w) const {
    TOPK_LDS unsigned char *p0 = (TOPK_LDS unsigned char*)b0, *p1 = (TOPK_LDS unsigned char*)b1, *p2 = (TOPK_LDS unsigned char*)b2,
                           *p3 = (TOPK_LDS unsigned char*)b3;
    return w == 0 ? p0 : w == 1 ? p1 : w == 2 ? p2 : p3;
  }
};

// 16 NR rows: the waves take key tiles in turn, K and V in registers. BOTH: of the prefix and of the request's
// own keys, as one list.
template <int D, int NR, bool BOTH>
struct Few {
  static constexpr int NS = D / 32;  // steps over the features of the scores
  static constexpr int NC = D / 16;  // blocks of 16 output features; columns of V a lane reads
  static constexpr int VB = NC * 2;  // their bytes
  static constexpr int TILE = 16 * NR;

  // column c of eight keys' numbers, as an operand
  static __device__ __forceinline__ bf16x8 column(const uint32_t (&x)[8][NC / 2], int c) {
    const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
    const int w = c / 2;
    return __builtin_bit_cast(bf16x8, make_uint4(__builtin_amdgcn_perm(x[1][w], x[0][w], sel), __builtin_amdgcn_perm(x[3][w], x[2][w], sel),
                                                 __builtin_amdgcn_perm(x[5][w], x[4][w], sel), __builtin_amdgcn_perm(x[7][w], x[6][w], sel)));
  }

  static __device__ __forceinline__ void run(const PrefixArgs& a, const Item& it, const Lds& sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int R = (int)a.pl.req_rows, Lq = (int)a.p.Lq;
    auto place = [&](int i) {  // of row i in q and out
      const int b = it.b >= 0 ? it.b : i / R;
      return b * a.p.H * Lq + it.h * R + (it.b >= 0 ? i : i - b * R);
    };
    auto lane_row = [&](int r) { return it.r0 + 16 * r + n < it.count ? it.r0 + 16 * r + n : it.r0; };
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

    int turn = wave;  // the wave's next tile
    // (code of its own for each part is faster, 5.1 us for 5.6 with 100 + 60 keys, where registers last)
    constexpr int COPIES = D * NR > 128 ? 1 : 2;
#pragma unroll COPIES
    for (int part = 0; part < (BOTH ? 2 : 1); ++part) {
    const Span sp = (BOTH ? part == 1 : it.b >= 0) ? it.own : it.prefix;
    const bool causal = (BOTH ? part == 1 : it.b >= 0) && a.p.causal;
    // how many keys the lane's rows see; keys before all_see are seen by every row
    int seen[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) seen[r] = causal ? min(sp.n, sp.before + lane_row(r) % Lq) : sp.n;
    const int all_see = causal ? min(sp.n, sp.before) : sp.n;

    bf16x8 kr[2][NS];
    uint32_t vr[8][NC / 2];
    const int tiles = (sp.n + KT - 1) / KT;
    // keys past the range load its last one: their scores are masked, their values put to 0
    auto load_k = [&](int t) {
      const int left = min(KT, sp.n - t * KT) - 1;
      const uint16_t* p = sp.k + (int64_t)(t * KT) * sp.k_sl;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t off = (uint32_t)min(16 * kb + n, left) * sp.k_sl + 8 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) kr[kb][s] = *(const bf16x8*)(p + off + 32 * s);
      }
    };
    auto load_v = [&](int t) {
      const int left = min(KT, sp.n - t * KT) - 1;
      const uint16_t* p = sp.v + (int64_t)(t * KT) * sp.v_sl;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t off = (uint32_t)min(16 * (e >> 2) + 4 * g + (e & 3), left) * sp.v_sl + n * NC;
        __builtin_memcpy(vr[e], __builtin_assume_aligned(p + off, VB), VB);
      }
    };
    int t = turn;
    if (t < tiles) {
      load_k(t);
      load_v(t);
    }
    for (; t < tiles; t += WAVES) {
      const int first = t * KT;
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
      if (t + WAVES < tiles) load_k(t + WAVES);
      if (first + KT > all_see) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (first + 16 * (e >> 2) + 4 * g + (e & 3) >= seen[r]) s[r][e >> 2][e & 3] = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (first + 16 * (e >> 2) + 4 * g + (e & 3) >= sp.n)
#pragma unroll
            for (int w = 0; w < NC / 2; ++w) vr[e][w] = 0;
        // Values that are not finite go to the rows that see their keys, which become NaN there; the others
        // would meet them as 0 times NaN.
        uint32_t bad = 0;
        if (causal && all_see < sp.n) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int w = 0; w < NC / 2; ++w) bad |= not_finite(vr[e][w]);
        }
        if (__builtin_amdgcn_ballot_w64(bad)) {
          int key0 = first + 4 * g;
          asm volatile("" : "+v"(key0));  // (nothing of this is held from above)
          bf16x8 sees[NR];
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[r][e] = (__bf16)(key0 + 16 * (e >> 2) + (e & 3) < seen[r] ? 1.f : 0.f);
#pragma unroll
          for (int w = 0; w < NC / 2; ++w) {
            uint32_t mark[8][NC / 2];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint32_t x = vr[e][w];
              asm volatile("" : "+v"(x));
              const uint32_t nf = not_finite(x);
              mark[e][w] = nf * 0x3F80u;  // 1 of bf16
              vr[e][w] = x & ~(nf * 0xFFFFu);
            }
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
              for (int c = 2 * w; c < 2 * w + 2; ++c) {
                const f32x4 met = __builtin_amdgcn_mfma_f32_16x16x32_bf16(column(mark, c), sees[r], (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                  if (met[v] > 0.f) o[r][c][v] = NAN;
              }
          }
        }
      }
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
      if (t + WAVES < tiles) load_v(t + WAVES);
    }
    turn = t - tiles;
    }

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
      if (wave == 0 && g == 0) {
        const int i = min(it.r0 + 16 * r + n, it.count - 1);
        sh.row[16 * r + n] = place(i);
        sh.sum[16 * r + n] = make_float2(top, total);
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 16 * NR * D / 4 / NT; ++u) {
      const int i = u * NT + tid, row = i / (D / 4), part = i % (D / 4);
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += ((const TOPK_LDS f32x4*)sh.of(w))[row * (D / 4) + (part ^ (row & 15))];
      const int64_t at = sh.row[row];
      const float2 x = sh.sum[row];
      if (it.r0 + row >= it.count) continue;
      if (a.pl.splits == 1) {
        const float inv = row_factor(x.y);
        *(uint2*)((uint16_t*)a.p.out + at * D + 4 * part) = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
        if (a.p.lse && part == 0) a.p.lse[at] = row_log(x.x, x.y);
      } else {
        __builtin_nontemporal_store(sum, (f32x4*)(a.po + (it.split * a.pl.rows + at) * D + 4 * part));
        if (part == 0) a.ml[it.split * a.pl.rows + at] = x;
      }
    }
  }
};

// 128 rows, 32 a wave: every wave takes every key tile of 64, K and V through LDS.
//   * S^T = K Q^T by v_mfma_f32_32x32x16_bf16: lane l holds 16 keys' scores of row l % 32 a 32-key
//     block, keys 8 (v / 4) + 4 (l / 32) + v % 4;
//   * O^T += V^T P^T by the same instruction: the weights are its operand in the order the lane holds
//     them, V^T comes from the row-major tile by transposing LDS reads (four keys of a feature each).
// Tiles come by direct global-to-LDS loads, one ahead; the 16-byte parts of their rows are permuted so
// that the lanes of one LDS cycle meet different banks. TWO: weights enter the second product as two
// bf16 numbers, as in the few-row form, which costs 3 to 17 % (5 tokens of 16 requests: 28.7 us, 25.0
// without); with 64 rows a request and more they are rounded to bf16 (relative 2^-8 at most), which
// saves a quarter of the products.
//
// Measured and left: the scores of the next tile formed between this tile's weights (no faster at
// sustained clocks, slower on short ranges: 31 us for 25), 64 rows a wave (accumulators spill), eight
// waves and 256 rows a workgroup (274 us for 276), three tiles ahead (the same).
typedef float f32x16 __attribute__((__vector_size__(64)));
typedef short s16x4 __attribute__((__vector_size__(8)));
typedef uint32_t u32x4 __attribute__((__vector_size__(16)));
typedef TOPK_LDS s16x4 lds_s16x4;

// the larger of x and what the lane 32 away holds
__device__ __forceinline__ float other_half_max(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

template <int D, bool TWO>
struct Wide {
  // The maximum that weights are taken against is moved, and the sums with it, only once a score
  // leads it by 2^8 in weight (291 -> 277 us at 4 x 512 tokens; s_setprio below: 277 -> 270).
  static constexpr float LEAD = 8.f;
  static constexpr int TILE = 32 * WAVES; // rows of a workgroup
  static constexpr int KEYS = 64;         // of a tile
  static constexpr int NS = D / 16;       // steps over the features of the scores
  static constexpr int CH = 2 * D / 16;   // 16-byte parts of a row
  static constexpr int TILEB = KEYS * 2 * D;
  static constexpr int LPW = TILEB / 1024 / WAVES;
  static constexpr int FB = D / 32;       // 32-feature blocks of the output
  static constexpr int AHEAD_K = 6, AHEAD_V = 4;  // products by which LDS reads run ahead of their use

  static __device__ __forceinline__ int swz_k(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int swz_v(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }

  static __device__ __forceinline__ void run(const PrefixArgs& a, const Item& it, const Lds& sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
    const int R = (int)a.pl.req_rows, Lq = (int)a.p.Lq;
    const int i = it.r0 + wave * 32 + n;
    const bool ok = i < it.count;
    const bool work = it.r0 + wave * 32 < it.count;  // the wave has rows
    const int ii = ok ? i : it.r0;
    const int b = it.b >= 0 ? it.b : ii / R, rr = it.b >= 0 ? ii : ii - b * R;
    const int64_t at = b * a.p.H * Lq + it.h * R + rr;
    bf16x8 bq[NS];
    {
      const uint16_t* q = (const uint16_t*)a.p.q + at * D + (D / 2) * half;
#pragma unroll
      for (int s = 0; s < NS; ++s) bq[s] = *(const bf16x8*)(q + 8 * s);
    }
    f32x16 o[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f) o[f] = (f32x16){};
    float m = -INFINITY, l = 0.f;
    // the lane's place in a V tile: row 4 half + (lane & 15) / 4, 8 bytes of it
    const int va = lane & 15, vrow = 4 * half + (va >> 2);
    int vat[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f)
      vat[f] = vrow * 2 * D + (((f * 4 + ((lane >> 4) & 1) * 2 + ((va & 3) >> 1)) ^ swz_v(vrow)) * 16) + (va & 1) * 8;

    for (int part = 0; part < 2; ++part) {
    const Span sp = part ? it.own : it.prefix;
    // keys before all_see are seen by every row of the workgroup, keys from keys on by none; the lane's sees `seen`
    int all_see = sp.n, keys = sp.n, seen = sp.n;
    if (part && a.p.causal) {
      const int r1 = min(it.r0 + TILE, it.count) - 1;
      const bool wraps = r1 / Lq != it.r0 / Lq;
      all_see = sp.before + (wraps ? 0 : it.r0 % Lq);
      keys = min(keys, sp.before + (wraps ? Lq - 1 : r1 % Lq));
      seen = min(keys, sp.before + rr % Lq);
    }
    if (keys <= 0) continue;
    const int tiles = (keys + KEYS - 1) / KEYS;
    // where the lane's parts of a tile lie, in bytes from its first key
    uint32_t koff[LPW], voff[LPW];
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int cidx = (wave * LPW + j) * 64 + lane, r = cidx / CH, c = cidx % CH;
      koff[j] = r * sp.k_sl * 2 + (c ^ swz_k(r)) * 16;
      voff[j] = r * sp.v_sl * 2 + (c ^ swz_v(r)) * 16;
    }
    const unsigned char *kt = (const unsigned char*)sp.k, *vt = (const unsigned char*)sp.v;  // of the next tile to load
    auto issue = [&](int t, unsigned char* kd, unsigned char* vd) {
      const int left = min(KEYS, keys - t * KEYS) - 1;
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        uint32_t ko = koff[j], vo = voff[j];
        if (left < KEYS - 1) {  // rows past the range load its last one
          const int r = ((wave * LPW + j) * 64 + lane) / CH, over = r - min(r, left);
          ko -= over * sp.k_sl * 2;
          vo -= over * sp.v_sl * 2;
        }
        __builtin_amdgcn_global_load_lds((const void*)(kt + ko), (TOPK_LDS void*)&kd[(wave * LPW + j) * 1024], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const void*)(vt + vo), (TOPK_LDS void*)&vd[(wave * LPW + j) * 1024], 16, 0, 0);
      }
      kt += KEYS * 2 * (int64_t)sp.k_sl;
      vt += KEYS * 2 * (int64_t)sp.v_sl;
    };

    auto tile = [&](auto edge, int t, const unsigned char* kb, const unsigned char* vb) {
      f32x16 s[2] = {};
      {
        bf16x8 kf[AHEAD_K + 1];
        auto kp = [&](int i) { return *(const bf16x8*)(kb + ((i & 1) * 32 + n) * 2 * D + ((half * NS + (i >> 1)) ^ swz_k(n)) * 16); };
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
      if (decltype(edge)::value) {
        const int last = seen - t * KEYS - 4 * half;
#pragma unroll
        for (int v = 0; v < 32; ++v)
          if ((v >> 4) * 32 + 8 * ((v & 15) >> 2) + (v & 3) >= last) s[v >> 4][v & 15] = -INFINITY;
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
      auto vp = [&](int j) {  // V^T of 16 keys j / FB, features 32 (j % FB) on
        const unsigned char* p = vb + vat[j % FB] + j / FB * 16 * 2 * D;
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * 2 * D));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      };
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
      auto wt = [&](int v) {
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
    // publishes every wave's part; it also proves that no wave still reads the buffers the next loads
    // overwrite. (The buffers are named at compile time, so that reads of one pair do not wait for loads
    // into the other.) Tiles that every row sees whole come first and need no mask.
    const int whole = max(0, min(keys, all_see)) / KEYS;
    auto ready = [&](int t, unsigned char* kn, unsigned char* vn) {
      __builtin_amdgcn_s_waitcnt(WAIT_VM0);
      __syncthreads();
      if (t + 1 < tiles) issue(t + 1, kn, vn);
    };
    __syncthreads();  // (the other part's last tile is read)
    issue(0, sh.b0, sh.b2);
    int t = 0;
    for (; t + 1 < whole; t += 2) {
      ready(t, sh.b1, sh.b3);
      if (work) tile(std::false_type{}, t, sh.b0, sh.b2);
      ready(t + 1, sh.b0, sh.b2);
      if (work) tile(std::false_type{}, t + 1, sh.b1, sh.b3);
    }
    // Where rows of the workgroup do not see all its keys, values that are not finite go only to the rows that
    // see theirs, which become NaN there; the others would meet them as 0 times NaN. Each wave looks at its part
    // of the tile.
    const bool hides = part && a.p.causal && all_see < keys;
    auto own_part = [&](unsigned char* vb, int j) { return (TOPK_LDS u32x4*)&vb[(wave * LPW + j) * 1024 + lane * 16]; };
    for (; t < tiles; ++t) {
      const bool odd = t & 1;
      unsigned char* vb = odd ? sh.b3 : sh.b2;
      if (hides) {
        __builtin_amdgcn_s_waitcnt(WAIT_VM0);
        uint32_t bad = 0;
#pragma unroll
        for (int j = 0; j < LPW; ++j) {
          const u32x4 x = *own_part(vb, j);
          bad |= not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3]);
        }
        const bool any = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
        if (lane == 0) sh.ml[wave][t & 1].x = any ? 1.f : 0.f;  // (read before the next barrier; the next tile's is another)
      }
      ready(t, odd ? sh.b0 : sh.b1, odd ? sh.b2 : sh.b3);
      if (hides && sh.ml[0][t & 1].x + sh.ml[1][t & 1].x + sh.ml[2][t & 1].x + sh.ml[3][t & 1].x > 0.f) {
#pragma unroll 1
        for (int j = 0; j < KEYS; ++j) {
          const bool sees = j < seen - t * KEYS;
#pragma unroll
          for (int f = 0; f < FB; ++f)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
              const TOPK_LDS uint32_t* x = (const TOPK_LDS uint32_t*)&vb[j * 2 * D + ((4 * f + v / 4) ^ swz_v(j)) * 16 + 8 * half];
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
      if (work) tile(std::true_type{}, t, odd ? sh.b1 : sh.b0, odd ? sh.b3 : sh.b2);
    }
    }
    l += __shfl_xor(l, 32, 64);
    // through the wave's own part of LDS, in parts of four features permuted by the row, so that whole rows
    // are written, two (D = 128) or four a store; partial results past the cache, which would otherwise
    // be emptied of them at the kernel's end (16 requests of 5 tokens behind 20001 keys: 27.8 -> 26.1 us)
    __syncthreads();
    TOPK_LDS f32x4* mine = (TOPK_LDS f32x4*)sh.of(wave);
    constexpr int PARTS = D / 4, RPS = 64 / PARTS;
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        mine[n * PARTS + ((8 * f + v / 2 + half) ^ (n & 15))] = (f32x4){o[f][v], o[f][v + 1], o[f][v + 2], o[f][v + 3]};
    wave_sync_lds();
    const bool last = a.pl.splits == 1;
    const float inv = row_factor(l);
    const int part = lane % PARTS;
#pragma unroll 4
    for (int u = 0; u < 32 / RPS; ++u) {
      const int row = u * RPS + lane / PARTS;
      const f32x4 x = mine[row * PARTS + (part ^ (row & 15))];
      const int64_t to = (int64_t)(uint32_t)__shfl((int)at, row, 64);
      const float by = __shfl(inv, row, 64);
      if (it.r0 + wave * 32 + row >= it.count) continue;
      if (last) *(uint2*)((uint16_t*)a.p.out + to * D + 4 * part) = make_uint2(pack_bf16(x[0] * by, x[1] * by), pack_bf16(x[2] * by, x[3] * by));
      else __builtin_nontemporal_store(x, (f32x4*)(a.po + (it.split * a.pl.rows + to) * D + 4 * part));
    }
    if (!ok || half) return;
    if (!last) a.ml[it.split * a.pl.rows + at] = make_float2(m, l);
    else if (a.p.lse) a.p.lse[at] = row_log(m, l);
  }
};

// A form by its number: 1 and 2 few rows (blocks of 16), 8 and 9 the wide one (with weights as two
// numbers, as one).
template <int D, int NB, bool BOTH = false>
struct Form {
  typedef Few<D, NB, BOTH> type;
};
template <int D, bool BOTH>
struct Form<D, 8, BOTH> {
  typedef Wide<D, true> type;
};
template <int D, bool BOTH>
struct Form<D, 9, BOTH> {
  typedef Wide<D, false> type;
};

// keys [k0, k1) of the prefix of key head h, as far as there are
__device__ __forceinline__ Span prefix_span(const PrefixArgs& a, int h, int64_t k0, int64_t k1) {
  Span s;
  k0 = min(k0, a.p.P);
  s.k = (const uint16_t*)a.p.pk + h * a.p.pk_sh + k0 * a.p.pk_sl;
  s.v = (const uint16_t*)a.p.pv + h * a.p.pv_sh + k0 * a.p.pv_sl;
  s.k_sl = (uint32_t)a.p.pk_sl;
  s.v_sl = (uint32_t)a.p.pv_sl;
  s.n = (int)(min(k1, a.p.P) - k0);
  s.before = s.n;
  return s;
}
// keys [k0, k1) of request b's own, as far as it holds them
__device__ __forceinline__ Span own_span(const PrefixArgs& a, int b, int h, int64_t k0, int64_t k1) {
  Span s;
  int64_t len = a.p.lengths ? a.p.lengths[b] : a.p.S;
  len = max((int64_t)0, min(len, a.p.S));
  k0 = max((int64_t)0, min(k0, len));
  s.k = (const uint16_t*)a.p.k + b * a.p.k_sb + h * a.p.k_sh + k0 * a.p.k_sl;
  s.v = (const uint16_t*)a.p.v + b * a.p.v_sb + h * a.p.v_sh + k0 * a.p.v_sl;
  s.k_sl = (uint32_t)a.p.k_sl;
  s.v_sl = (uint32_t)a.p.v_sl;
  s.n = (int)max((int64_t)0, min(k1, len) - k0);
  s.before = (int)max((int64_t)-(1 << 30), min(len - a.p.Lq + 1 - k0, (int64_t)(1 << 30)));
  return s;
}

// NBP, NBS: the forms of the items on the prefix (row tiles over all requests) and on own keys. BOTH:
// an item's rows are one request's and take the prefix and its own keys as one list, in form NBS.
template <int D, int NBP, int NBS, bool BOTH>
__global__ __launch_bounds__(NT, 2) void k_prefix(PrefixArgs a) {
  constexpr int BUF = 64 * 2 * D;
  __shared__ __attribute__((aligned(16))) unsigned char b0[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b1[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b2[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b3[BUF];
  __shared__ float2 ml[WAVES][32], sum[32];
  __shared__ int64_t row[32];
  const Lds sh = {b0, b1, b2, b3, ml, sum, row};
  const PrefixPlan& pl = a.pl;
  const int B = (int)a.p.B, Hkv = (int)a.p.Hkv, ptiles = (int)pl.ptiles, stiles = (int)pl.stiles, psplits = (int)pl.psplits,
            ssplits = (int)pl.ssplits;
  int i = blockIdx.x;
  Item it;
  if (BOTH) {
    const int n = gridDim.x, splits = (int)pl.splits;
    if (n % 8 == 0) i = (i % 8) * (n / 8) + i / 8;  // an XCD's workgroups share key ranges
    const int tile = i % stiles, rest = i / stiles, rest2 = rest / B;
    it.b = rest % B;
    it.split = rest2 % splits;
    it.h = rest2 / splits;
    it.count = (int)pl.req_rows;
    typedef typename Form<D, NBS, true>::type F;
    it.r0 = tile * F::TILE;
    const int64_t k0 = it.split * pl.pkeys;
    it.prefix = prefix_span(a, it.h, k0, k0 + pl.pkeys);
    it.own = own_span(a, it.b, it.h, k0 - a.p.P, k0 + pl.pkeys - a.p.P);
    F::run(a, it, sh);
    return;
  }
  const int np = Hkv * psplits * ptiles;
  if (i < np) {
    if (np % 8 == 0) i = (i % 8) * (np / 8) + i / 8;
    const int tile = i % ptiles, rest = i / ptiles;
    it.split = rest % psplits;
    it.h = rest / psplits;
    it.b = -1;
    it.prefix = prefix_span(a, it.h, it.split * pl.pkeys, it.split * pl.pkeys + pl.pkeys);
    it.own = it.prefix;
    it.own.n = 0;
    it.own.before = 0;
    it.count = (int)(a.p.B * pl.req_rows);
    it.r0 = tile * Form<D, NBP>::type::TILE;
    Form<D, NBP>::type::run(a, it, sh);
    return;
  }
  i -= np;
  const int tile = i % stiles, rest = i / stiles, split = rest % ssplits, bh = rest / ssplits;
  it.b = bh / Hkv;
  it.h = bh - it.b * Hkv;
  it.split = psplits + split;
  it.own = own_span(a, it.b, it.h, split * pl.skeys, split * pl.skeys + pl.skeys);
  it.prefix = it.own;
  it.prefix.n = 0;
  it.count = (int)pl.req_rows;
  it.r0 = tile * Form<D, NBS>::type::TILE;
  Form<D, NBS>::type::run(a, it, sh);
}

// Joins a row's partial results. ROWS rows a workgroup: NT / ROWS threads a row, D / 4 columns by
// as many groups as there are left, each taking every so manieth range; the ranges' factors come
// first, one thread a range.
template <int D, int ROWS>
__global__ __launch_bounds__(NT) void k_prefix_join(PrefixArgs a) {
  constexpr int TR = NT / ROWS, LR = D / 4, Q = TR / LR;
  static_assert(Q >= 1, "a thread has at least one column group");
  __shared__ float fac[ROWS][ROWS == 1 ? JOIN_MAX : JOIN_FEW];
  __shared__ f32x4 part[ROWS][Q][LR];
  const int rl = threadIdx.x / TR, tr = threadIdx.x % TR, q = tr / LR, c = tr % LR;
  const int64_t row = (int64_t)blockIdx.x * ROWS + rl;
  const bool ok = row < a.pl.rows;
  const int splits = (int)a.pl.splits;
  float top = -INFINITY, total = 0.f;
  if (ok) {
    if (splits <= 4) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s < splits) top = larger(top, a.ml[s * a.pl.rows + row].x);
    } else {
      for (int s = tr; s < splits; s += TR) top = larger(top, a.ml[s * a.pl.rows + row].x);
    }
  }
  if (splits > 4) {  // (TR lanes of a row: 16 or 32 of one wave, or whole waves)
    for (int o = 1; o < (TR < 64 ? TR : 64); o <<= 1) top = larger(top, __shfl_xor(top, o, 64));
    if (TR > 64) {
      if (threadIdx.x % 64 == 0) fac[rl][threadIdx.x % TR / 64] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < TR / 64; ++w) top = larger(top, fac[rl][w]);
      __syncthreads();
    }
  }
  if (ok)
    for (int s = tr; s < splits; s += TR) {
      const float2 x = a.ml[s * a.pl.rows + row];
      const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - top);
      fac[rl][s] = f;
      total += f * x.y;
    }
  for (int o = 1; o < (TR < 64 ? TR : 64); o <<= 1) total += __shfl_xor(total, o, 64);
  __syncthreads();
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (ok) {
    const float* p = a.po + row * D + 4 * c;
#pragma unroll 4
    for (int s = q; s < splits; s += Q) {
      const float f = fac[rl][s];
      sum += *(const f32x4*)(p + (int64_t)s * a.pl.rows * D) * f;  // (a range without keys leaves zeros)
    }
  }
  if (Q > 1) {
    part[rl][q][c] = sum;
    __shared__ float tot[ROWS][4];
    if (TR > 64 && threadIdx.x % 64 == 0) tot[rl][threadIdx.x % TR / 64] = total;
    __syncthreads();
    if (q > 0) return;
#pragma unroll
    for (int k = 1; k < Q; ++k) sum += part[rl][k][c];
    if (TR > 64) {
      total = 0.f;
#pragma unroll
      for (int w = 0; w < TR / 64; ++w) total += tot[rl][w];
    }
  }
  if (!ok) return;
  const float inv = row_factor(total);
  const uint2 w = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
  *(uint2*)((uint16_t*)a.p.out + row * D + 4 * c) = w;
  if (a.p.lse && c == 0) a.p.lse[row] = row_log(top, total);
}

PrefixArgs args_for(const PrefixProblem& pp, const PrefixPlan& pl, const void* ws) {
  PrefixArgs a;
  a.p = pp;
  a.pl = pl;
  a.po = (float*)ws;
  a.ml = (float2*)((char*)ws + (size_t)pl.splits * pl.rows * pp.d * 4);
  a.c = pp.scale * 1.4426950408889634f;
  return a;
}

// The form for so many rows. Measured, 8 key heads of 128: 16 rows behind 30000 keys, 28.4 us as one block
// of 16 rows, 30.6 as two; 20 rows a request against 16 caches of 1000 to 3000 keys, 37 us as two blocks,
// 42 as a wide tile; 64 rows behind 30000 keys, 34.4 us as a wide tile, 38.5 as two tiles of 32, and 40 rows
// against such caches 45 and 57.
int form_for(int64_t rows, int wide) { return rows <= 16 ? 1 : rows <= 32 ? 2 : wide; }
int tile_rows(int form) { return form >= 8 ? 128 : 16 * form; }
// Microseconds of `items` wide tiles of 128 rows against `keys` keys each: as many layers on 256 CUs as it
// takes, a step of 64 keys in 1.05 us (d = 128) times the workgroups that share a CU; 1.25 alone, 1.45 where
// hundreds of caches' workgroups (crowded) find no CU free of them, and 1.65 for two whose registers or weights as
// two numbers leave the units idle.
double wide_us(int d, bool two, bool crowded, int64_t items, int64_t keys) {
  const int64_t layers = cdiv(items, 256);
  const double step = (d == 64 ? 0.7 : 1.05) * (two ? 1.3 : 1.0);
  const double share = layers == 1 ? (crowded && items > 208 ? 1.45 : 1.25) : layers == 2 && (two || d == 64) ? 1.65 : (double)layers;
  return share * step * (keys / 64.0 + 3);
}
constexpr int64_t ONE_ITEMS = 512, ONE_KEYS = 1024;  // requests and key heads, keys of 64 features, of calls in one range
constexpr double JOIN_US = 2e-6;  // of a partial result's number, written and read

}  // namespace

PrefixPlan prefix_plan(const PrefixProblem& pp) {
  PrefixPlan pl = {};
  pl.rows = pp.B * pp.H * pp.Lq;
  pl.req_rows = pp.H / pp.Hkv * pp.Lq;
  const int wide = pl.req_rows < 64 ? 8 : 9;
  pl.sform = form_for(pl.req_rows, wide);
  pl.pform = pp.P ? form_for(pp.B * pl.req_rows, wide) : pl.sform;
  pl.ptiles = cdiv(pp.B * pl.req_rows, tile_rows(pl.pform));
  pl.stiles = cdiv(pl.req_rows, tile_rows(pl.sform));
  // (many rows are joined several a workgroup, from few ranges)
  const int64_t longest = std::max(pp.P, pp.S), least = cdiv(longest, (pl.rows > 1 << 20 ? JOIN_FEW : JOIN_MAX) / 2 * 128) * 128;
  // Few rows and few keys: one workgroup a request and key head takes all its keys, and nothing is left to join.
  // (12 heads of 64, 4 requests, 500 + 130 keys: 7.8 us either way, 700 + 300: 9.3 and 8.1, but a launch less for
  // the host, 5 us; 32 heads on 8, 16 requests, 500 + 130: 8.0 and 13.0, at d = 128 with 1000 + 500 22 and 17; 64
  // requests of d = 64 with 700 + 300 16.4 and 15.7, 128 with 400 + 100 16.7 and 14.3.)
  if (pl.sform < 8 && pp.B * pp.Hkv <= ONE_ITEMS && pp.P + pp.S > 0 && (pp.P + pp.S) * pp.d <= ONE_KEYS * 64) {
    pl.both = true;
    pl.pkeys = pp.P + pp.S;
    pl.splits = 1;
    return pl;
  }
  // one list of prefix and own keys, unless more than an eighth of a tile's rows would be idle on the prefix
  // (4 x 512 tokens: 277 us, 286 in two lists; 8 requests of 80 rows, of 128: 24.6 us, 21.0 in two lists)
  pl.both = pl.sform == 9 && pl.stiles * 128 * 8 <= pl.req_rows * 9;
  if (pl.both) {
    const int64_t items = pp.Hkv * pp.B * pl.stiles, keys = pp.P + pp.S;
    // as many ranges as finish soonest, the join's traffic included (a request of 64 tokens, 16 heads of 128 on 4,
    // behind 60000 keys: 55 us in 32 ranges, 78 in 16)
    double best = 0;
    const int64_t most = pl.rows > 1 << 20 ? JOIN_FEW : JOIN_MAX / 2;
    for (int64_t s = 1; s <= most && (s == 1 || cdiv(keys, s) >= 128); s += std::max<int64_t>(1, s / 8)) {
      const int64_t range = std::max<int64_t>({64, least, cdiv(cdiv(keys, s), 64) * 64}), n = std::max<int64_t>(1, cdiv(keys, range));
      const double us = wide_us(pp.d, false, false, items * n, range) + (n > 1 ? 4 + n * pl.rows * pp.d * JOIN_US : 0);
      if (s == 1 || us < best) {
        best = us;
        pl.pkeys = range;
      }
    }
    pl.pkeys = std::min(pl.pkeys, RANGE_MAX);
    pl.splits = std::max<int64_t>(1, cdiv(keys, pl.pkeys));
    return pl;
  }
  // ranges of equal length, as many as give two workgroups a CU, of 128 keys at least (4 requests behind 500
  // keys: 8.6 us, 9.5 with 256 at least)
  const int64_t keys = pp.Hkv * pl.ptiles * pp.P + pp.B * pp.Hkv * pl.stiles * pp.S;
  const int64_t range = std::min(std::max(std::max<int64_t>(128, cdiv(cdiv(keys, 512), 128) * 128), least), RANGE_MAX);
  pl.psplits = cdiv(pp.P, range);
  pl.ssplits = cdiv(pp.S, range);
  if (pl.pform >= 8 && pl.sform < 8) {
    // Wide tiles on the prefix beside few rows on the caches: as many ranges as finish soonest beside the
    // caches' reads (of which the lengths may leave about 0.6), the join's traffic included: 64 requests
    // behind 8192 keys without caches 28 us, 32 with equal ranges; 128 behind 4096 with caches of 2048, 8 key
    // heads of 128: 125 and 143; 256 behind 1000 with caches of 1000, 8 of 64: 66 and 64.
    const double own = (double)pp.S * pp.B * pp.Hkv * pp.d * 4 * 0.6 / 5e6;
    double best = 0;
    for (int64_t s = 1; s <= JOIN_MAX / 2 && (s == 1 || cdiv(pp.P, s) >= 128); s += std::max<int64_t>(1, s / 8)) {
      const int64_t part = std::max(cdiv(cdiv(pp.P, s), 128) * 128, least), n = cdiv(pp.P, part);
      const double wide_t = wide_us(pp.d, wide == 8, pp.B * pp.Hkv >= 256, pp.Hkv * pl.ptiles * n, part);
      const double us = std::max(wide_t, own) + 0.25 * std::min(wide_t, own) + n * pl.rows * pp.d * JOIN_US;
      if (best == 0 || us < best) {
        best = us;
        pl.psplits = n;
      }
    }
    pl.psplits = std::max(pl.psplits, cdiv(pp.P, RANGE_MAX));
  }
  pl.pkeys = pl.psplits ? cdiv(cdiv(pp.P, pl.psplits), 128) * 128 : 128;
  pl.skeys = pl.ssplits ? cdiv(cdiv(pp.S, pl.ssplits), 128) * 128 : 128;
  pl.psplits = cdiv(pp.P, pl.pkeys);
  pl.ssplits = cdiv(pp.S, pl.skeys);
  pl.splits = pl.psplits + pl.ssplits;
  return pl;
}

size_t prefix_bytes(const PrefixProblem& pp, const PrefixPlan& pl) {
  return pl.splits == 1 ? 0 : (size_t)pl.splits * pl.rows * (pp.d + 2) * 4;
}

template <int D>
static void launch_d(const PrefixArgs& a, unsigned grid, hipStream_t st) {
  const int np = a.pl.pform, ns = a.pl.sform;
  if (a.pl.both && ns == 1) k_prefix<D, 1, 1, true><<<grid, NT, 0, st>>>(a);
  else if (a.pl.both && ns == 2) k_prefix<D, 2, 2, true><<<grid, NT, 0, st>>>(a);
  else if (a.pl.both) k_prefix<D, 9, 9, true><<<grid, NT, 0, st>>>(a);
  else if (np == 1) k_prefix<D, 1, 1, false><<<grid, NT, 0, st>>>(a);
  else if (np == 2 && ns == 1) k_prefix<D, 2, 1, false><<<grid, NT, 0, st>>>(a);
  else if (np == 2) k_prefix<D, 2, 2, false><<<grid, NT, 0, st>>>(a);
  else if (ns == 1) k_prefix<D, 8, 1, false><<<grid, NT, 0, st>>>(a);
  else if (ns == 2) k_prefix<D, 8, 2, false><<<grid, NT, 0, st>>>(a);
  else if (ns == 8) k_prefix<D, 8, 8, false><<<grid, NT, 0, st>>>(a);
  else k_prefix<D, 9, 9, false><<<grid, NT, 0, st>>>(a);
}

int64_t prefix_items(const PrefixProblem& pp, const PrefixPlan& pl) {
  return pl.both ? pp.Hkv * pp.B * pl.stiles * pl.splits : pp.Hkv * pl.psplits * pl.ptiles + pp.B * pp.Hkv * pl.ssplits * pl.stiles;
}

hipError_t launch_prefix(const PrefixProblem& pp, const PrefixPlan& pl, void* ws, hipStream_t st) {
  const int64_t items = prefix_items(pp, pl);
  if (!items) return hipSuccess;
  const PrefixArgs a = args_for(pp, pl, ws);
  if (pp.d == 64) launch_d<64>(a, (unsigned)items, st);
  else launch_d<128>(a, (unsigned)items, st);
  return hipGetLastError();
}

template <int D>
static void join_d(const PrefixArgs& a, hipStream_t st) {
  // one row a workgroup while the rows leave CUs free, or have many ranges
  constexpr int MANY = NT / (D / 4);
  if (a.pl.rows <= 2048 || a.pl.splits > JOIN_FEW) k_prefix_join<D, 1><<<(unsigned)a.pl.rows, NT, 0, st>>>(a);
  else k_prefix_join<D, MANY><<<(unsigned)cdiv(a.pl.rows, MANY), NT, 0, st>>>(a);
}

hipError_t launch_prefix_join(const PrefixProblem& pp, const PrefixPlan& pl, const void* ws, hipStream_t st) {
  if (pl.splits == 1) return hipSuccess;
  const PrefixArgs a = args_for(pp, pl, ws);
  if (pp.d == 64) join_d<64>(a, st);
  else join_d<128>(a, st);
  return hipGetLastError();
}

}  // namespace topk
