// Attention of a batch whose requests share a long prefix: every row attends to the prefix
// (P keys and values of each key head, one copy for all requests) and to its own request's
// cache, out_i = sum_j softmax_j(scale q_i.k_j) v_j over both. G = H / Hkv query heads share a
// key head.
//
// The prefix is read once for a tile of rows of all requests, not once a request: the rows
// (request, query head of the group, token) of one key head are one long list for the prefix,
// and one short list a request for the caches. A workgroup takes one row tile and one key
// range, of the prefix or of one cache, and leaves a partial result (the running maximum, the
// sum and the unnormalised output, all in 32 bits) which a second kernel joins; where there is
// one range in all, it writes the output itself. Both kinds of workgroup run in one launch.
//
// Within a workgroup four waves take key tiles of 32 in turn, each with a running softmax of
// its own, joined through LDS at the end. Scores are S^T = K Q^T and the output O^T = V^T P^T by
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

constexpr int NT = 256, WAVES = 4, KT = 32;
constexpr int JOIN_MAX = 1024;  // key ranges of a row at most,
constexpr int JOIN_FEW = 16;    // where a workgroup joins several rows
// s_waitcnt immediate: no vector-memory operation outstanding, the other counters ignored
constexpr int WAIT_VM0 = (7 << 4) | (15 << 8);

struct PrefixArgs {
  PrefixProblem p;
  PrefixPlan pl;
  float* po;   // [splits][rows][D]
  float2* ml;  // [splits][rows]: maximum of the scaled scores (to base 2), sum of weights
  float c;     // scale * log2(e)
};

// One work item: rows [r0, r0 + 16 NR) of a list of `count` rows against keys [k0, k1).
struct Item {
  const uint16_t *k, *v;
  int64_t k_sl, v_sl;
  int64_t r0, count, k0, k1;
  int64_t h;      // key head
  int64_t b;      // request (-1: rows of all requests)
  int64_t len;    // keys in all
  int64_t split;  // where its partial result goes
};

// A workgroup's LDS: four tile buffers (the few-row form keeps a wave's outputs in each), and the
// waves' maxima and sums.
struct Lds {
  unsigned char *b0, *b1, *b2, *b3;
  float2 (*ml)[32];
  __device__ unsigned char* of(int w) const { return w == 0 ? b0 : w == 1 ? b1 : w == 2 ? b2 : b3; }
};

// 16 NR rows: the waves take key tiles in turn, K and V in registers.
template <int D, int NR>
struct Few {
  static constexpr int NS = D / 32;  // steps over the features of the scores
  static constexpr int NC = D / 16;  // blocks of 16 output features; columns of V a lane reads
  static constexpr int VB = NC * 2;  // their bytes
  static constexpr int LD = D + 4;
  typedef float Rows[LD];            // 16 of them a wave

  static __device__ __forceinline__ void run(const PrefixArgs& a, const Item& it, const Lds& sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int64_t R = a.pl.req_rows, Lq = a.p.Lq, HL = a.p.H * Lq;
    // the lane's rows: where they lie in q and out, and how many keys they see
    int64_t at[NR], seen[NR];
    bf16x8 bq[NR][NS];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int64_t i = it.r0 + 16 * r + n;
      const bool ok = i < it.count;
      const int64_t ii = ok ? i : it.r0;
      const int64_t b = it.b >= 0 ? it.b : ii / R, rr = it.b >= 0 ? ii : ii - b * R;
      at[r] = b * HL + it.h * R + rr;
      seen[r] = it.len;
      if (it.b >= 0 && a.p.causal) {
        const int64_t t = it.len - Lq + rr % Lq + 1;
        seen[r] = t < 0 ? 0 : t;
      }
      const uint16_t* q = (const uint16_t*)a.p.q + at[r] * D + 8 * g;
#pragma unroll
      for (int s = 0; s < NS; ++s) bq[r][s] = *(const bf16x8*)(q + 32 * s);
      if (!ok) at[r] = -1;
    }
    const int64_t all_see = it.b >= 0 && a.p.causal ? it.len - Lq + 1 : it.len;  // keys before this are seen by every row

    f32x4 o[NR][NC];
    float m[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) o[r][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    bf16x8 kr[2][NS];
    uint32_t vr[8][NC / 2];
    const int64_t tiles = (it.k1 - it.k0 + KT - 1) / KT;
    // keys past the range load its last one: their scores are masked, their values put to 0
    auto load_k = [&](int64_t t) {
      const int64_t first = it.k0 + t * KT;
      const int left = (int)min((int64_t)KT, it.k1 - first) - 1;
      const uint16_t* p = it.k + first * it.k_sl;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t off = (uint32_t)min(16 * kb + n, left) * (uint32_t)it.k_sl + 8 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) kr[kb][s] = *(const bf16x8*)(p + off + 32 * s);
      }
    };
    auto load_v = [&](int64_t t) {
      const int64_t first = it.k0 + t * KT;
      const int left = (int)min((int64_t)KT, it.k1 - first) - 1;
      const uint16_t* p = it.v + first * it.v_sl;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t off = (uint32_t)min(16 * (e >> 2) + 4 * g + (e & 3), left) * (uint32_t)it.v_sl + n * NC;
        __builtin_memcpy(vr[e], __builtin_assume_aligned(p + off, VB), VB);
      }
    };
    int64_t t = wave;
    if (t < tiles) {
      load_k(t);
      load_v(t);
    }
    for (; t < tiles; t += WAVES) {
      const int64_t first = it.k0 + t * KT;
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
      if (first + KT > min(it.k1, all_see)) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int64_t j = first + 16 * (e >> 2) + 4 * g + (e & 3);
            if (j >= it.k1 || j >= seen[r]) s[r][e >> 2][e & 3] = -INFINITY;
          }
        const int64_t left = it.k1 - first;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (16 * (e >> 2) + 4 * g + (e & 3) >= left)
#pragma unroll
            for (int w = 0; w < NC / 2; ++w) vr[e][w] = 0;
      }
      bf16x8 hi[NR], lo[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float mt = fmaxf(fmaxf(fmaxf(s[r][0][0], s[r][0][1]), fmaxf(s[r][0][2], s[r][0][3])),
                         fmaxf(fmaxf(s[r][1][0], s[r][1][1]), fmaxf(s[r][1][2], s[r][1][3])));
        mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
        mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
        const float mn = fmaxf(m[r], mt * a.c);
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
        const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
        const int w = c / 2;
        const uint4 u = make_uint4(__builtin_amdgcn_perm(vr[1][w], vr[0][w], sel), __builtin_amdgcn_perm(vr[3][w], vr[2][w], sel),
                                   __builtin_amdgcn_perm(vr[5][w], vr[4][w], sel), __builtin_amdgcn_perm(vr[7][w], vr[6][w], sel));
        const bf16x8 av = __builtin_bit_cast(bf16x8, u);
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, hi[r], o[r][c], 0, 0, 0);
          o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, lo[r], o[r][c], 0, 0, 0);
        }
      }
      if (t + WAVES < tiles) load_v(t + WAVES);
    }

    // join the waves: row by row maxima, then the scaled outputs through LDS
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      l[r] += __shfl_xor(l[r], 16, 64);
      l[r] += __shfl_xor(l[r], 32, 64);
      if (g == 0) sh.ml[wave][16 * r + n] = make_float2(m[r], l[r]);
    }
    __syncthreads();
    const bool last = a.pl.psplits + a.pl.ssplits == 1;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sh.ml[w][16 * r + n].x);
      const float f = m[r] == -INFINITY ? 0.f : exp2f(m[r] - top);
      if (r) __syncthreads();
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int c = 0; c < NC; ++c) ((Rows*)sh.of(wave))[n][(4 * g + v) * NC + c] = o[r][c][v] * f;
      __syncthreads();
      for (int i = tid; i < 16 * D / 4; i += NT) {
        const int row = i / (D / 4), col = (i % (D / 4)) * 4;
        const int64_t ri = it.r0 + 16 * r + row;
        if (ri >= it.count) continue;
        const int64_t b = it.b >= 0 ? it.b : ri / R, rr = it.b >= 0 ? ri : ri - b * R;
        const int64_t gr = b * HL + it.h * R + rr;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float tm = -INFINITY, tl = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          sum += *(const f32x4*)&((const Rows*)sh.of(w))[row][col];
          tm = fmaxf(tm, sh.ml[w][16 * r + row].x);
        }
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const float2 x = sh.ml[w][16 * r + row];
          if (x.x != -INFINITY) tl += x.y * exp2f(x.x - tm);
        }
        if (last) {
          const float inv = tl > 0.f ? 1.f / tl : 0.f;
          const uint2 w = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
          *(uint2*)((uint16_t*)a.p.out + gr * D + col) = w;
          if (a.p.lse && col == 0) a.p.lse[gr] = tl > 0.f ? (tm + log2f(tl)) * 0.69314718055994531f : -INFINITY;
        } else {
          *(f32x4*)(a.po + (it.split * a.pl.rows + gr) * D + col) = sum;
          if (col == 0) a.ml[it.split * a.pl.rows + gr] = make_float2(tm, tl);
        }
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
// that the lanes of one LDS cycle meet different banks. Weights enter the second product rounded to
// bf16 (relative 2^-8 at most): products bound this form, and a second term would add half as many.
typedef float f32x16 __attribute__((__vector_size__(64)));
typedef short s16x4 __attribute__((__vector_size__(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <int D, bool TWO>
struct Wide {
  // Weights are formed as 2^24 times themselves, so that the exponential instruction, which knows no
  // numbers below 2^-126, keeps every weight that 32 bits can hold.
  static constexpr float LIFT = 24.f;
  static constexpr int KEYS = 64;         // of a tile
  static constexpr int NS = D / 16;       // steps over the features of the scores
  static constexpr int CH = 2 * D / 16;   // 16-byte parts of a row
  static constexpr int TILEB = KEYS * 2 * D;
  static constexpr int LPW = TILEB / 1024 / WAVES;
  static constexpr int FB = D / 32;       // 32-feature blocks of the output

  static __device__ __forceinline__ int swz_k(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int swz_v(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }

  static __device__ __forceinline__ void run(const PrefixArgs& a, const Item& it, const Lds& sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
    const int64_t R = a.pl.req_rows, Lq = a.p.Lq, HL = a.p.H * Lq;
    const bool causal = it.b >= 0 && a.p.causal;
    const int64_t i = it.r0 + wave * 32 + n;
    const bool ok = i < it.count;
    const bool work = it.r0 + wave * 32 < it.count;  // the wave has rows
    const int64_t ii = ok ? i : it.r0;
    const int64_t b = it.b >= 0 ? it.b : ii / R, rr = it.b >= 0 ? ii : ii - b * R;
    const int64_t at = b * HL + it.h * R + rr;
    int64_t seen = it.len;
    if (causal) {
      const int64_t t = it.len - Lq + rr % Lq + 1;
      seen = t < 0 ? 0 : t;
    }
    bf16x8 bq[NS];
    {
      const uint16_t* q = (const uint16_t*)a.p.q + at * D + (D / 2) * half;
#pragma unroll
      for (int s = 0; s < NS; ++s) bq[s] = *(const bf16x8*)(q + 8 * s);
    }
    // keys before all_see are seen by every row, keys from k1 by none of the tile
    int64_t all_see = it.len, k1 = it.k1;
    if (causal) {
      const int64_t r1 = min(it.r0 + 128, it.count) - 1;
      const bool wraps = r1 / Lq != it.r0 / Lq;
      all_see = it.len - Lq + (wraps ? 0 : it.r0 % Lq) + 1;
      k1 = min(k1, it.len - Lq + (wraps ? Lq - 1 : r1 % Lq) + 1);
    }
    const int64_t tiles = k1 > it.k0 ? (k1 - it.k0 + KEYS - 1) / KEYS : 0;

    // where the lane's parts of a tile lie, in bytes from its first key
    uint32_t koff[LPW], voff[LPW];
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int cidx = (wave * LPW + j) * 64 + lane, r = cidx / CH, c = cidx % CH;
      koff[j] = r * (uint32_t)it.k_sl * 2 + (c ^ swz_k(r)) * 16;
      voff[j] = r * (uint32_t)it.v_sl * 2 + (c ^ swz_v(r)) * 16;
    }
    auto issue = [&](int64_t t, unsigned char* kd, unsigned char* vd) {
      const int64_t first = it.k0 + t * KEYS;
      const unsigned char* kt = (const unsigned char*)(it.k + first * it.k_sl);
      const unsigned char* vt = (const unsigned char*)(it.v + first * it.v_sl);
      const int left = (int)min((int64_t)KEYS, k1 - first) - 1;
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        uint32_t ko = koff[j], vo = voff[j];
        if (left < KEYS - 1) {  // rows past the range load its last one
          const int r = ((wave * LPW + j) * 64 + lane) / CH, over = r - min(r, left);
          ko -= over * (uint32_t)it.k_sl * 2;
          vo -= over * (uint32_t)it.v_sl * 2;
        }
        __builtin_amdgcn_global_load_lds((const void*)(kt + ko), (__attribute__((address_space(3))) void*)&kd[(wave * LPW + j) * 1024], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const void*)(vt + vo), (__attribute__((address_space(3))) void*)&vd[(wave * LPW + j) * 1024], 16, 0, 0);
      }
    };

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

    auto tile = [&](auto edge, int64_t t, const unsigned char* kb, const unsigned char* vb) {
      f32x16 s[2];
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const int r = rb * 32 + n;
        f32x16 acc = {};
#pragma unroll
        for (int st = 0; st < NS; ++st) {
          const bf16x8 av = *(const bf16x8*)(kb + (r * CH + ((half * NS + st) ^ swz_k(r))) * 16);
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, bq[st], acc, 0, 0, 0);
        }
        s[rb] = acc;
      }
      if (decltype(edge)::value) {
        const int last = (int)max((int64_t)-1, min(min(k1, seen) - it.k0 - t * KEYS, (int64_t)KEYS)) - 4 * half;
#pragma unroll
        for (int v = 0; v < 32; ++v)
          if ((v >> 4) * 32 + 8 * ((v & 15) >> 2) + (v & 3) >= last) s[v >> 4][v & 15] = -INFINITY;
      }
      float mt = -INFINITY;
#pragma unroll
      for (int v = 0; v < 32; v += 2)
        mt = __builtin_elementwise_maximum(__builtin_elementwise_maximum(mt, s[v >> 4][v & 15]), s[v >> 4][(v & 15) + 1]);
      mt = __builtin_elementwise_maximum(mt, __shfl_xor(mt, 32, 64));
      mt *= a.c;
      if (__builtin_amdgcn_ballot_w64(!(mt <= m))) {  // (for NaN too; rows whose maximum stays multiply by 1)
        const float mn = fmaxf(m, mt);
        const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[f][v] *= alpha;
      }
      const float bias = LIFT - (m == -INFINITY ? 0.f : m);
#pragma unroll
      for (int st = 0; st < 4; ++st) {  // 16 keys each
        bf16x8 pb, pl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w = __builtin_amdgcn_exp2f(fmaf(s[st >> 1][8 * (st & 1) + e], a.c, bias));
          l += w;
          pb[e] = (__bf16)w;
          if (TWO) pl[e] = (__bf16)(w - (float)pb[e]);
        }
#pragma unroll
        for (int f = 0; f < FB; ++f) {
          const unsigned char* p = vb + vat[f] + st * 16 * 2 * D;
          const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
          const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * 2 * D));
          const bf16x8 av = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
          o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, pb, o[f], 0, 0, 0);
          if (TWO) o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, pl, o[f], 0, 0, 0);
        }
      }
    };

    // One tile of lookahead: before tile t is read, this wave's loads of it are complete and the barrier
    // publishes every wave's part; it also proves that no wave still reads the buffers the next loads
    // overwrite. (The buffers are named at compile time, so that reads of one pair do not wait for loads
    // into the other.) Tiles that every row sees whole come first and need no mask.
    const int64_t whole = min(tiles, max((int64_t)0, min(k1, all_see) - it.k0) / KEYS);
    auto ready = [&](int64_t t, unsigned char* kn, unsigned char* vn) {
      __builtin_amdgcn_s_waitcnt(WAIT_VM0);
      __syncthreads();
      if (t + 1 < tiles) issue(t + 1, kn, vn);
    };
    if (tiles > 0) issue(0, sh.b0, sh.b2);
    int64_t t = 0;
    for (; t + 1 < whole; t += 2) {
      ready(t, sh.b1, sh.b3);
      if (work) tile(std::false_type{}, t, sh.b0, sh.b2);
      ready(t + 1, sh.b0, sh.b2);
      if (work) tile(std::false_type{}, t + 1, sh.b1, sh.b3);
    }
    for (; t < tiles; ++t) {
      const bool odd = t & 1;
      ready(t, odd ? sh.b0 : sh.b1, odd ? sh.b2 : sh.b3);
      if (work) tile(std::true_type{}, t, odd ? sh.b1 : sh.b0, odd ? sh.b3 : sh.b2);
    }
    m -= LIFT;
    l += __shfl_xor(l, 32, 64);
    if (!ok) return;
    if (a.pl.psplits + a.pl.ssplits == 1) {
      const float inv = l > 0.f ? 1.f / l : 0.f;
      uint16_t* dst = (uint16_t*)a.p.out + at * D + 4 * half;
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *(uint2*)(dst + 32 * f + 2 * v) = make_uint2(pack_bf16(o[f][v] * inv, o[f][v + 1] * inv), pack_bf16(o[f][v + 2] * inv, o[f][v + 3] * inv));
      if (a.p.lse && half == 0) a.p.lse[at] = l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
      return;
    }
    float* dst = a.po + (it.split * a.pl.rows + at) * D + 4 * half;
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int v = 0; v < 16; v += 4) *(f32x4*)(dst + 32 * f + 2 * v) = (f32x4){o[f][v], o[f][v + 1], o[f][v + 2], o[f][v + 3]};
    if (half == 0) a.ml[it.split * a.pl.rows + at] = make_float2(m, l);
  }
};

// NB: blocks of 16 rows of an item; 8 is the wide form
template <int D, int NB>
struct Form {
  typedef Few<D, NB> type;
};
template <int D>
struct Form<D, 8> {
  typedef Wide<D, false> type;
};
template <int D>
struct Form<D, 9> {
  typedef Wide<D, true> type;
};

template <int D, int NBP, int NBS>
__global__ __launch_bounds__(NT, 2) void k_prefix(PrefixArgs a) {
  constexpr int BUF = 64 * 2 * D;
  __shared__ __attribute__((aligned(16))) unsigned char b0[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b1[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b2[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char b3[BUF];
  __shared__ float2 ml[WAVES][32];
  const Lds sh = {b0, b1, b2, b3, ml};
  const PrefixPlan& pl = a.pl;
  const int64_t np = a.p.Hkv * pl.psplits * pl.ptiles;
  int64_t i = blockIdx.x;
  Item it;
  if (i < np) {
    if (np % 8 == 0) i = (i % 8) * (np / 8) + i / 8;  // an XCD's workgroups share key ranges
    const int64_t tile = i % pl.ptiles, rest = i / pl.ptiles;
    it.split = rest % pl.psplits;
    it.h = rest / pl.psplits;
    it.b = -1;
    it.k = (const uint16_t*)a.p.pk + it.h * a.p.pk_sh;
    it.v = (const uint16_t*)a.p.pv + it.h * a.p.pv_sh;
    it.k_sl = a.p.pk_sl;
    it.v_sl = a.p.pv_sl;
    it.count = a.p.B * pl.req_rows;
    it.r0 = tile * 16 * (NBP & ~1 ? NBP & ~1 : 1);
    it.len = a.p.P;
    it.k0 = it.split * pl.pkeys;
    it.k1 = min(it.k0 + pl.pkeys, it.len);
    Form<D, NBP>::type::run(a, it, sh);
    return;
  }
  i -= np;
  const int64_t tile = i % pl.stiles, rest = i / pl.stiles, split = rest % pl.ssplits, bh = rest / pl.ssplits;
  it.b = bh / a.p.Hkv;
  it.h = bh - it.b * a.p.Hkv;
  it.split = pl.psplits + split;
  it.k = (const uint16_t*)a.p.k + it.b * a.p.k_sb + it.h * a.p.k_sh;
  it.v = (const uint16_t*)a.p.v + it.b * a.p.v_sb + it.h * a.p.v_sh;
  it.k_sl = a.p.k_sl;
  it.v_sl = a.p.v_sl;
  it.count = pl.req_rows;
  it.r0 = tile * 16 * (NBS & ~1 ? NBS & ~1 : 1);
  const int64_t len = a.p.lengths ? a.p.lengths[it.b] : a.p.S;
  it.len = len < 0 ? 0 : min(len, a.p.S);
  it.k0 = min(split * pl.skeys, it.len);
  it.k1 = min(it.k0 + pl.skeys, it.len);
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
  const int splits = (int)(a.pl.psplits + a.pl.ssplits);
  float top = -INFINITY, total = 0.f;
  if (ok) {
    if (splits <= 4) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s < splits) top = fmaxf(top, a.ml[s * a.pl.rows + row].x);
    } else {
      for (int s = tr; s < splits; s += TR) top = fmaxf(top, a.ml[s * a.pl.rows + row].x);
    }
  }
  if (splits > 4) {  // (TR lanes of a row: 32 or more of one wave, or whole waves)
    for (int o = 1; o < (TR < 64 ? TR : 64); o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if (TR > 64) {
      if (threadIdx.x % 64 == 0) fac[rl][threadIdx.x % TR / 64] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < TR / 64; ++w) top = fmaxf(top, fac[rl][w]);
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
      const f32x4 x = *(const f32x4*)(p + (int64_t)s * a.pl.rows * D);
      if (f != 0.f) sum += x * f;  // (a range without keys leaves zeros)
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
  const float inv = total > 0.f ? 1.f / total : 0.f;
  const uint2 w = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
  *(uint2*)((uint16_t*)a.p.out + row * D + 4 * c) = w;
  if (a.p.lse && c == 0) a.p.lse[row] = total > 0.f ? (top + log2f(total)) * 0.69314718055994531f : -INFINITY;
}

int64_t cdiv(int64_t x, int64_t y) { return (x + y - 1) / y; }

PrefixArgs args_for(const PrefixProblem& pp, const PrefixPlan& pl, const void* ws) {
  PrefixArgs a;
  a.p = pp;
  a.pl = pl;
  a.po = (float*)ws;
  a.ml = (float2*)((char*)ws + (size_t)(pl.psplits + pl.ssplits) * pl.rows * pp.d * 4);
  a.c = pp.scale * 1.4426950408889634f;
  return a;
}

int blocks_for(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 8; }

}  // namespace

PrefixPlan prefix_plan(const PrefixProblem& pp) {
  PrefixPlan pl = {};
  pl.rows = pp.B * pp.H * pp.Lq;
  pl.req_rows = pp.H / pp.Hkv * pp.Lq;
  pl.sblocks = blocks_for(pl.req_rows);
  pl.pblocks = pp.P ? blocks_for(pp.B * pl.req_rows) : pl.sblocks;
  pl.ptiles = cdiv(pp.B * pl.req_rows, 16 * pl.pblocks);
  pl.stiles = cdiv(pl.req_rows, 16 * pl.sblocks);
  // ranges of equal length, as many as give two workgroups a CU, of 256 keys at least
  const int64_t keys = pp.Hkv * pl.ptiles * pp.P + pp.B * pp.Hkv * pl.stiles * pp.S;
  int64_t range = std::max<int64_t>(256, cdiv(cdiv(keys, 512), 128) * 128);
  range = std::max(range, cdiv(std::max(pp.P, pp.S), JOIN_MAX / 2 * 128) * 128);
  pl.psplits = cdiv(pp.P, range);
  pl.ssplits = cdiv(pp.S, range);
  pl.pkeys = pl.psplits ? cdiv(cdiv(pp.P, pl.psplits), 128) * 128 : 128;
  pl.skeys = pl.ssplits ? cdiv(cdiv(pp.S, pl.ssplits), 128) * 128 : 128;
  pl.psplits = cdiv(pp.P, pl.pkeys);
  pl.ssplits = cdiv(pp.S, pl.skeys);
  return pl;
}

size_t prefix_bytes(const PrefixProblem& pp, const PrefixPlan& pl) {
  const int64_t splits = pl.psplits + pl.ssplits;
  return splits == 1 ? 0 : (size_t)splits * pl.rows * (pp.d + 2) * 4;
}

template <int D>
static void launch_d(const PrefixArgs& a, unsigned grid, hipStream_t st) {
  const int np = a.pl.pblocks, ns = a.pl.sblocks;
  if (np == 1) k_prefix<D, 1, 1><<<grid, NT, 0, st>>>(a);
  else if (np == 2 && ns == 1) k_prefix<D, 2, 1><<<grid, NT, 0, st>>>(a);
  else if (np == 2) k_prefix<D, 2, 2><<<grid, NT, 0, st>>>(a);
  else if (ns == 1) k_prefix<D, 9, 1><<<grid, NT, 0, st>>>(a);
  else if (ns == 2) k_prefix<D, 9, 2><<<grid, NT, 0, st>>>(a);
  else if (a.pl.req_rows < 64) k_prefix<D, 9, 9><<<grid, NT, 0, st>>>(a);
  else k_prefix<D, 8, 8><<<grid, NT, 0, st>>>(a);
}

hipError_t launch_prefix(const PrefixProblem& pp, const PrefixPlan& pl, void* ws, hipStream_t st) {
  const int64_t items = pp.Hkv * pl.psplits * pl.ptiles + pp.B * pp.Hkv * pl.ssplits * pl.stiles;
  if (items > 0xFFFFFF) return hipErrorInvalidValue;
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
  if (a.pl.rows <= 2048 || a.pl.psplits + a.pl.ssplits > JOIN_FEW) k_prefix_join<D, 1><<<(unsigned)a.pl.rows, NT, 0, st>>>(a);
  else k_prefix_join<D, MANY><<<(unsigned)cdiv(a.pl.rows, MANY), NT, 0, st>>>(a);
}

hipError_t launch_prefix_join(const PrefixProblem& pp, const PrefixPlan& pl, const void* ws, hipStream_t st) {
  if (pl.psplits + pl.ssplits == 1) return hipSuccess;
  if (pl.rows > 0xFFFFFF) return hipErrorInvalidValue;
  const PrefixArgs a = args_for(pp, pl, ws);
  if (pp.d == 64) join_d<64>(a, st);
  else join_d<128>(a, st);
  return hipGetLastError();
}

}  // namespace topk
