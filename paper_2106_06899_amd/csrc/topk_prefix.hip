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

template <int D, int NR>
struct Body {
  static constexpr int NS = D / 32;  // steps over the features of the scores
  static constexpr int NC = D / 16;  // blocks of 16 output features; columns of V a lane reads
  static constexpr int VB = NC * 2;  // their bytes
  static constexpr int LD = D + 4;
  struct Shared {
    float o[WAVES][16][LD];
    float2 ml[WAVES][16 * NR];
  };

  static __device__ __forceinline__ void run(const PrefixArgs& a, const Item& it, Shared& sh) {
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
        for (int c = 0; c < NC; ++c) sh.o[wave][n][(4 * g + v) * NC + c] = o[r][c][v] * f;
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
          sum += *(const f32x4*)&sh.o[w][row][col];
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

template <int D, int NRP, int NRS>
__global__ __launch_bounds__(NT, NRP > 2 ? 1 : 2) void k_prefix(PrefixArgs a) {
  union Both {
    typename Body<D, NRP>::Shared p;
    typename Body<D, NRS>::Shared s;
  };
  __shared__ __attribute__((aligned(16))) Both sh;
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
    it.r0 = tile * 16 * NRP;
    it.len = a.p.P;
    it.k0 = it.split * pl.pkeys;
    it.k1 = min(it.k0 + pl.pkeys, it.len);
    Body<D, NRP>::run(a, it, sh.p);
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
  it.r0 = tile * 16 * NRS;
  const int64_t len = a.p.lengths ? a.p.lengths[it.b] : a.p.S;
  it.len = len < 0 ? 0 : min(len, a.p.S);
  it.k0 = min(split * pl.skeys, it.len);
  it.k1 = min(it.k0 + pl.skeys, it.len);
  Body<D, NRS>::run(a, it, sh.s);
}

// Joins a row's partial results: D / 4 lanes a row.
template <int D>
__global__ __launch_bounds__(NT) void k_prefix_join(PrefixArgs a) {
  constexpr int LR = D / 4;
  const int64_t row = (int64_t)blockIdx.x * (NT / LR) + threadIdx.x / LR;
  const int col = (threadIdx.x % LR) * 4;
  if (row >= a.pl.rows) return;
  const int splits = (int)(a.pl.psplits + a.pl.ssplits);
  float top = -INFINITY;
  for (int s = 0; s < splits; ++s) top = fmaxf(top, a.ml[s * a.pl.rows + row].x);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float2 x = a.ml[s * a.pl.rows + row];
    if (x.x == -INFINITY) continue;  // saw no key
    const float f = exp2f(x.x - top);
    sum += *(const f32x4*)(a.po + (s * a.pl.rows + row) * D + col) * f;
    total += x.y * f;
  }
  const float inv = total > 0.f ? 1.f / total : 0.f;
  const uint2 w = make_uint2(pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv));
  *(uint2*)((uint16_t*)a.p.out + row * D + col) = w;
  if (a.p.lse && col == 0) a.p.lse[row] = total > 0.f ? (top + log2f(total)) * 0.69314718055994531f : -INFINITY;
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

int blocks_for(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

}  // namespace

PrefixPlan prefix_plan(const PrefixProblem& pp) {
  PrefixPlan pl = {};
  pl.rows = pp.B * pp.H * pp.Lq;
  pl.req_rows = pp.H / pp.Hkv * pp.Lq;
  pl.nr = blocks_for(pp.P ? pp.B * pl.req_rows : pl.req_rows);
  const int ns = blocks_for(pl.req_rows);
  pl.ptiles = cdiv(pp.B * pl.req_rows, 16 * pl.nr);
  pl.stiles = cdiv(pl.req_rows, 16 * ns);
  // ranges of equal length, as many as give two workgroups a CU, of 256 keys at least
  const int64_t keys = pp.Hkv * pl.ptiles * pp.P + pp.B * pp.Hkv * pl.stiles * pp.S;
  const int64_t range = std::max<int64_t>(256, cdiv(cdiv(keys, 512), 128) * 128);
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
static void launch_d(const PrefixArgs& a, int np, int ns, unsigned grid, hipStream_t st) {
  if (np == 1) k_prefix<D, 1, 1><<<grid, NT, 0, st>>>(a);
  else if (np == 2 && ns == 1) k_prefix<D, 2, 1><<<grid, NT, 0, st>>>(a);
  else if (np == 2) k_prefix<D, 2, 2><<<grid, NT, 0, st>>>(a);
  else if (ns == 1) k_prefix<D, 4, 1><<<grid, NT, 0, st>>>(a);
  else if (ns == 2) k_prefix<D, 4, 2><<<grid, NT, 0, st>>>(a);
  else k_prefix<D, 4, 4><<<grid, NT, 0, st>>>(a);
}

hipError_t launch_prefix(const PrefixProblem& pp, const PrefixPlan& pl, void* ws, hipStream_t st) {
  const int64_t items = pp.Hkv * pl.psplits * pl.ptiles + pp.B * pp.Hkv * pl.ssplits * pl.stiles;
  if (items > 0xFFFFFF) return hipErrorInvalidValue;
  if (!items) return hipSuccess;
  const PrefixArgs a = args_for(pp, pl, ws);
  const int ns = blocks_for(pl.req_rows);
  if (pp.d == 64) launch_d<64>(a, pl.nr, ns, (unsigned)items, st);
  else launch_d<128>(a, pl.nr, ns, (unsigned)items, st);
  return hipGetLastError();
}

hipError_t launch_prefix_join(const PrefixProblem& pp, const PrefixPlan& pl, const void* ws, hipStream_t st) {
  if (pl.psplits + pl.ssplits == 1) return hipSuccess;
  const PrefixArgs a = args_for(pp, pl, ws);
  const int64_t blocks = cdiv(pl.rows, NT / (pp.d / 4));
  if (blocks > 0xFFFFFF) return hipErrorInvalidValue;
  if (pp.d == 64) k_prefix_join<64><<<(unsigned)blocks, NT, 0, st>>>(a);
  else k_prefix_join<128><<<(unsigned)blocks, NT, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace topk
