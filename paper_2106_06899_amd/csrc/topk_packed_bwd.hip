// Gradients of packed attention. With P = exp(scale S - lse), recomputed from the inputs, and
// D_i = d_out_i . out_i (which is sum_j P_ij (d_out_i . v_j)):
//   dV = P^T d_out,  dS = P (d_out V^T - D),  dQ = scale dS K,  dK = scale dS^T Q.
// D is taken from out and what rounding it to bf16 took (its rounding alone would put dQ and dK off by 2.8e-3 in place
// of 2.4e-3, of which their own rounding is 1.66e-3).
// Three launches: the rows' lse and D (and zeros for the tokens of no sequence); dQ, a workgroup a tile of 128 queries,
// over the keys; dK and dV, a workgroup a tile of 128 keys and key head, over the queries of all its query heads. Each gradient is summed
// where it ends up, in a fixed order, without atomics, which costs a second S and d_out V^T: seven products in
// place of five.
//
// Both kernels keep their own 128 rows' numbers in registers (32 rows a wave, a row in lanes l and l + 32) and
// take the other side's rows through LDS in tiles of 64, read straight for the products over features and
// transposed for those over rows (see PackedTile). Weights and score gradients come out of the first products
// in the order in which the second take them; they are rounded to bf16 on the way (relative 2^-9 at most, as
// the weights of the forward pass), sums are in fp32. Where that costs little (packed_short) they are the sum of two
// bf16 numbers: dQ, dK and dV are then off by what their own rounding is, in place of 1.4 times that (and, of few
// numbers, up to 1.6). A pass over 1000 tokens takes 3 us more for it, over 2000 sequences of 30 tokens 545 -> 575; over
// 14000 tokens, heads of 128, it would be 1670 -> 2330.
// Bound as the forward pass: 3 texts of 1000 to 8192 tokens, causal, 16 heads of 128 on 4, 1.05 PFLOP/s: dQ 507 us, dK
// and dV 682 and the sum of their shares 48, of a pass of 1640 with the forward's 368.
#include "topk_packed_device.h"

#include <math.h>

#include <type_traits>

namespace topk {
namespace {

#define TOPK_INLINE __attribute__((always_inline))  // (a lambda that is called captures through memory)
constexpr int NT = 256, WAVES = 4, ROWS = 64;  // ROWS: of a tile in LDS

struct BackwardArgs {
  PackedProblem p;
  float c;  // scale * log2(e)
};

__device__ __forceinline__ void clear_part(const PackedRows& to, int64_t h, int64_t t, int c) {
  *(uint4*)((uint16_t*)to.p + h * to.head + t * to.token + c) = make_uint4(0, 0, 0, 0);
}

// The rows' lse to base 2 and D, in one pass over out, rest and d_out: 16 rows a workgroup (D = 128) or 32, 16 bytes a
// lane. Bound by memory: 16 heads of 128 of 13788 tokens 21 to 28 us, 169 MB.
template <int D>
__global__ __launch_bounds__(NT) void k_packed_stat(BackwardArgs a) {
  constexpr int LR = D / 8;  // lanes of a row
  const uint32_t row = blockIdx.x * (NT / LR) + threadIdx.x / LR, head = row / (uint32_t)a.p.N;  // (fewer than 2^28 rows)
  const int64_t i = row, h = head, t = row - head * (uint32_t)a.p.N;
  if (h >= a.p.H) return;
  const int c = threadIdx.x % LR * 8, N = (int)a.p.N;
  if (t < min(max(a.p.offsets[0], 0), N) || t >= min(max(a.p.offsets[a.p.n], 0), N)) {  // a token of no sequence
    clear_part(a.p.dq, h, t, c);
    if (h < a.p.Hkv && a.p.splits == 1) {  // (else the sums' launch does it)
      clear_part(a.p.dk, h, t, c);
      clear_part(a.p.dv, h, t, c);
    }
    return;
  }
  const int64_t at = h * a.p.out.head + t * a.p.out.token + c;
  const u32x4 x = *(const u32x4*)((const uint16_t*)a.p.out.p + at);
  const u32x4 y = a.p.rest ? *(const u32x4*)((const uint16_t*)a.p.rest + at) : (u32x4){};
  const u32x4 g = *(const u32x4*)((const uint16_t*)a.p.d_out.p + h * a.p.d_out.head + t * a.p.d_out.token + c);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sum = fmaf(__uint_as_float(x[e] << 16) + __uint_as_float(y[e] << 16), __uint_as_float(g[e] << 16), sum);
    sum = fmaf(__uint_as_float(x[e] & 0xFFFF0000u) + __uint_as_float(y[e] & 0xFFFF0000u), __uint_as_float(g[e] & 0xFFFF0000u), sum);
  }
#pragma unroll
  for (int o = 1; o < LR; o <<= 1) sum += __shfl_xor(sum, o, 64);
  if (c == 0) {
    const float lse = a.p.lse[i] * 1.4426950408889634f;
    a.p.stat[i] = lse == -INFINITY ? INFINITY : lse;  // (a row without a weight has none here, too)
    a.p.stat[a.p.H * a.p.N + i] = sum;
  }
}

// Loads a tile of 64 rows to LDS, LPW parts a lane; rows past `left` load row `left`. Only the first part's place is
// held: part j lies 64 / CH rows further on, and swz differs by a constant there.
template <int D, int LPW>
struct Loader {
  static constexpr int CH = 2 * D / 16, STEP = 64 / CH, FLIP = D == 128 ? 1 : 2;
  uint32_t row, part;
  uint32_t sl;  // bytes from one row to the next
  __device__ __forceinline__ Loader(int64_t token) {
    sl = (uint32_t)token * 2;
    row = (threadIdx.x >> 6) * LPW * STEP + (threadIdx.x & 63) / CH;
    part = (threadIdx.x & 63) % CH ^ PackedTile<D>::swz(row);
  }
  __device__ __forceinline__ void operator()(const unsigned char* from, unsigned char* to, int left, int wave) const {
    uint32_t r = row, c = part;
    asm volatile("" : "+v"(r), "+v"(c));  // (the places of the other parts are formed anew for every tile)
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const uint32_t o = (left < ROWS - 1 ? min(r + j * STEP, (uint32_t)left) : r + j * STEP) * sl + (c ^ (j * FLIP)) * 16;
      __builtin_amdgcn_global_load_lds((const void*)(from + o), (TOPK_LDS void*)&to[(wave * LPW + j) * 1024], 16, 0, 0);
    }
  }
};

// Numbers of a tile that are not finite: the wave's own part of it.
template <int LPW>
__device__ __forceinline__ bool part_not_finite(unsigned char* b, int wave, int lane) {
  uint32_t bad = 0;
#pragma unroll 1
  for (int j = 0; j < LPW; ++j) {
    const u32x4 x = *(TOPK_LDS u32x4*)&b[(wave * LPW + j) * 1024 + lane * 16];
    bad |= not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3]);
  }
  return __builtin_amdgcn_ballot_w64(bad != 0) != 0;
}
template <int LPW>
__device__ __forceinline__ void part_clear(unsigned char* b, int wave, int lane) {
#pragma unroll 1
  for (int j = 0; j < LPW; ++j) {
    TOPK_LDS u32x4* at = (TOPK_LDS u32x4*)&b[(wave * LPW + j) * 1024 + lane * 16];
    u32x4 x = *at;
#pragma unroll
    for (int w = 0; w < 4; ++w) x[w] &= ~(not_finite(x[w]) * 0xFFFFu);
    *at = x;
  }
}
// Which of the lane's sums (bit 16 f + v: feature 32 f + 8 (v / 4) + 4 half + v % 4) row j of the tile, which its row
// sees, makes NaN: those where it holds a number that is not finite. They are kept in LDS, apart from the sums,
// which branches would make the compiler hold twice.
template <int D>
__device__ __forceinline__ void mark_row(TOPK_LDS uint64_t* marks, const unsigned char* b, int j, bool sees, int half) {
  uint64_t m = 0;
#pragma unroll 1
  for (int f = 0; f < D / 32; ++f)
#pragma unroll 1
    for (int v = 0; v < 16; v += 4) {
      const TOPK_LDS uint32_t* x = (const TOPK_LDS uint32_t*)&b[j * 2 * D + ((4 * f + v / 4) ^ PackedTile<D>::swz(j)) * 16 + 8 * half];
#pragma unroll
      for (int w = 0; w < 4; ++w) m |= (uint64_t)(not_finite(x[w / 2]) >> 16 * (w & 1) & 1) << (16 * f + v + w);
    }
  if (sees) *marks |= m;
}
template <int D>
__device__ __forceinline__ void apply_marks(f32x16 (&o)[D / 32], const TOPK_LDS uint64_t* at) {
  const uint64_t marks = *at;
  if (!__builtin_amdgcn_ballot_w64(marks != 0)) return;
#pragma unroll
  for (int f = 0; f < D / 32; ++f)
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (marks >> (16 * f + v) & 1) o[f][v] = NAN;
}

// 32 rows of a wave, times `by`, through its 16 (D = 128) or 8 KiB of LDS to rows first .. of `to`, those before n.
// (T float: as they are, past the cache.)
template <int D, typename T>
__device__ __forceinline__ void store_rows(const f32x16 (&o)[D / 32], float by, TOPK_LDS f32x4* mine, T* to, int64_t token, int first, int n) {
  const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
  constexpr int PARTS = D / 4, RPS = 64 / PARTS;
#pragma unroll
  for (int f = 0; f < D / 32; ++f)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      mine[row * PARTS + ((8 * f + v / 2 + half) ^ (row & 15))] = (f32x4){o[f][v] * by, o[f][v + 1] * by, o[f][v + 2] * by, o[f][v + 3] * by};
  wave_sync_lds();
  const int part = lane % PARTS;
#pragma unroll 4
  for (int u = 0; u < 32 / RPS; ++u) {
    const int r = u * RPS + lane / PARTS;
    const f32x4 x = mine[r * PARTS + (part ^ (r & 15))];
    if (first + r >= n) continue;
    if constexpr (std::is_same<T, float>::value) __builtin_nontemporal_store(x, (f32x4*)(to + (first + r) * token + 4 * part));
    else *(uint2*)(to + (first + r) * token + 4 * part) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  }
  wave_sync_lds();
}

// KS = 2: half the rows a workgroup, and two waves share each 32, one taking the first and one the last 32 keys of
// every tile, as in the forward pass. TWO: score gradients as the sum of two bf16 numbers.
template <int D, bool CAUSAL, int KS, bool TWO>
__global__ __launch_bounds__(NT, TWO ? 1 : 2) void k_packed_dq(BackwardArgs a) {
  typedef PackedTile<D> Tile;
  constexpr int TROWS = PACKED_TILE / KS, NB = 2 / KS;  // rows of the workgroup; blocks of 32 of a tile that a wave takes
  constexpr int NS = D / 16, TILEB = ROWS * 2 * D, LPW = TILEB / 1024 / WAVES, FB = D / 32;
  __shared__ __attribute__((aligned(16))) unsigned char k0[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char k1[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char v0[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char v1[TILEB];
  __shared__ int flag[WAVES][2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
  const int group = wave % (WAVES / KS), share = wave / (WAVES / KS);  // of rows; of a tile's keys
  const int2 item = packed_item(a.p.H);
  const int h = item.x;
  const PackedPlace at = packed_place(a.p, item.y, TROWS, a.p.H, CAUSAL, false);
  if (!at.n) return;
  const int hk = h / (a.p.H / a.p.Hkv);
  const int row = at.tile * TROWS + group * 32 + n;
  const bool work = at.tile * TROWS + group * 32 < at.n;
  const int64_t token = at.first + min(row, at.n - 1);
  bf16x8 bq[NS], bo[NS];
  {
    const uint16_t* q = (const uint16_t*)a.p.q.p + h * a.p.q.head + token * a.p.q.token + (D / 2) * half;
    const uint16_t* g = (const uint16_t*)a.p.d_out.p + h * a.p.d_out.head + token * a.p.d_out.token + (D / 2) * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      bq[s] = *(const bf16x8*)(q + 8 * s);
      bo[s] = *(const bf16x8*)(g + 8 * s);
    }
  }
  const float lse = a.p.stat[h * a.p.N + token], D_row = a.p.stat[(a.p.H + h) * a.p.N + token];
  f32x16 o[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) o[f] = (f32x16){};

  const int keys = CAUSAL ? min(at.n, at.tile * TROWS + TROWS) : at.n;
  const int all_see = CAUSAL ? at.tile * TROWS + 1 : at.n, seen = CAUSAL ? min(at.n, row + 1) : at.n;
  const int tiles = (keys + ROWS - 1) / ROWS;
  const Loader<D, LPW> load_k(a.p.k.token), load_v(a.p.v.token);
  const unsigned char* kt = (const unsigned char*)((const uint16_t*)a.p.k.p + hk * a.p.k.head + at.first * a.p.k.token);
  const unsigned char* vt = (const unsigned char*)((const uint16_t*)a.p.v.p + hk * a.p.v.head + at.first * a.p.v.token);
  auto issue = [&](int t, unsigned char* kd, unsigned char* vd) TOPK_INLINE {
    const int left = min(ROWS, keys - t * ROWS) - 1;
    load_k(kt, kd, left, wave);
    load_v(vt, vd, left, wave);
    kt += ROWS * (int64_t)load_k.sl;
    vt += ROWS * (int64_t)load_v.sl;
  };
  auto tile = [&](bool edge, int t, const unsigned char* kbuf, const unsigned char* vbuf) TOPK_INLINE {
    const TOPK_LDS unsigned char *kb = (const TOPK_LDS unsigned char*)kbuf + (KS > 1 ? share * 32 * 2 * D : 0),
                                 *vb = (const TOPK_LDS unsigned char*)vbuf + (KS > 1 ? share * 32 * 2 * D : 0);
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
      uint32_t row0 = Tile::straight_base(), col0 = Tile::across_base();
      asm volatile("" : "+v"(row0), "+v"(col0));  // (the places that follow from them are not held)
      f32x16 s = {}, g = {};
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::straight(kb, row0, rb, i), bq[i], s, 0, 0, 0);
        g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::straight(vb, row0, rb, i), bo[i], g, 0, 0, 0);
      }
      bf16x8 ds[2], lo[2];
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.c, -lse)) * (g[v] - D_row);
      if (edge) {
        const int last = seen - t * ROWS - (KS > 1 ? share : rb) * 32 - 4 * half;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v >> 2) + (v & 3) >= last) s[v] = 0.f;
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        ds[v >> 3][v & 7] = (__bf16)s[v];
        if (TWO) lo[v >> 3][v & 7] = (__bf16)(s[v] - (float)ds[v >> 3][v & 7]);
      }
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int f = 0; f < FB; ++f) {
          const bf16x8 x = Tile::across(kb, col0, f, rb * 2 + st);
          o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, ds[st], o[f], 0, 0, 0);
          if (TWO) o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, lo[st], o[f], 0, 0, 0);
        }
    }
  };
  const int whole = min(keys, all_see) / ROWS;  // tiles that every row sees whole come first
  __shared__ uint64_t marks[CAUSAL ? NT : 1];
  TOPK_LDS uint64_t* mark = (TOPK_LDS uint64_t*)&marks[tid];
  if (CAUSAL) *mark = 0;
  // tile t, in the buffers that it is in; the next one's loads go to the others
  auto step = [&](auto works, int t, unsigned char* kb, unsigned char* vb, unsigned char* kn, unsigned char* vn) TOPK_INLINE {
    __builtin_amdgcn_s_waitcnt(PACKED_WAIT_VM0);
    const bool diagonal = CAUSAL && t >= whole;
    if (diagonal) {  // keys that are not finite reach only the rows that see them, which become NaN there
      const bool any = part_not_finite<LPW>(kb, wave, lane);
      if (lane == 0) flag[wave][t & 1] = any;
    }
    __syncthreads();
    if (t + 1 < tiles) issue(t + 1, kn, vn);
    if (diagonal && (flag[0][t & 1] | flag[1][t & 1] | flag[2][t & 1] | flag[3][t & 1])) {
#pragma unroll 1
      for (int j = 0; j < ROWS; ++j) mark_row<D>(mark, kb, j, j < seen - t * ROWS, half);
      __syncthreads();
      part_clear<LPW>(kb, wave, lane);
      __syncthreads();
    }
    if (decltype(works)::value) tile(t >= whole, t, kb, vb);
  };
  issue(0, k0, v0);
  auto all = [&](auto works) TOPK_INLINE {
    for (int t = 0; t < tiles; t += 2) {
      step(works, t, k0, v0, k1, v1);
      if (t + 1 < tiles) step(works, t + 1, k1, v1, k0, v0);
    }
  };
  if (work) all(std::true_type{});
  else all(std::false_type{});
  if (CAUSAL) apply_marks<D>(o, mark);
  __syncthreads();
  TOPK_LDS unsigned char *p0 = (TOPK_LDS unsigned char*)k0, *p1 = (TOPK_LDS unsigned char*)k1, *p2 = (TOPK_LDS unsigned char*)v0,
                         *p3 = (TOPK_LDS unsigned char*)v1;
  if (KS > 1) {  // the second half of the waves hand their sums over, four numbers a lane at a time
    TOPK_LDS f32x4* to = (TOPK_LDS f32x4*)(group ? p1 : p0) + lane;
    if (share) {
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int v = 0; v < 16; v += 4) to[(4 * f + v / 4) * 64] = (f32x4){o[f][v], o[f][v + 1], o[f][v + 2], o[f][v + 3]};
    }
    __syncthreads();
    if (share) return;
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const f32x4 y = to[(4 * f + v / 4) * 64];
#pragma unroll
        for (int w = 0; w < 4; ++w) o[f][v + w] += y[w];
      }
    wave_sync_lds();
  }
  TOPK_LDS f32x4* mine = (TOPK_LDS f32x4*)(KS > 1 ? group ? p1 : p0 : wave == 0 ? p0 : wave == 1 ? p1 : wave == 2 ? p2 : p3);
  store_rows<D>(o, a.p.scale, mine, (uint16_t*)a.p.dq.p + h * a.p.dq.head + at.first * a.p.dq.token, a.p.dq.token,
                at.tile * TROWS + group * 32, at.n);
}

// TWO: weights and score gradients as sums of two bf16 numbers.
template <int D, bool CAUSAL, bool TWO>
__global__ __launch_bounds__(NT, TWO ? 1 : 2) void k_packed_dkv(BackwardArgs a) {
  typedef PackedTile<D> Tile;
  constexpr int NS = D / 16, TILEB = ROWS * 2 * D, LPW = TILEB / 1024 / WAVES, FB = D / 32;
  __shared__ __attribute__((aligned(16))) unsigned char q0[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char q1[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char g0[TILEB];
  __shared__ __attribute__((aligned(16))) unsigned char g1[TILEB];
  __shared__ __attribute__((aligned(16))) float s0[2 * ROWS];
  __shared__ __attribute__((aligned(16))) float s1[2 * ROWS];
  __shared__ int flag[WAVES][2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
  const int splits = a.p.splits;
  const int2 item = packed_item(a.p.Hkv * splits);
  const int hk = item.x / splits, split = item.x - hk * splits;
  const PackedPlace at = packed_place(a.p, item.y, PACKED_TILE, a.p.Hkv * splits, CAUSAL, true);
  if (!at.n) return;
  const int G = a.p.H / a.p.Hkv;
  const int key = at.tile * PACKED_TILE + wave * 32 + n;
  const bool work = at.tile * PACKED_TILE + wave * 32 < at.n;
  // D = 128: the last parts of the values' rows lie in LDS, for which the registers do not last
  constexpr int NR = D == 128 ? NS - (CAUSAL ? 3 : 2) : NS;
  __shared__ __attribute__((aligned(16))) bf16x8 bv_rest[NS > NR ? (NS - NR) * NT : 1];
  TOPK_LDS bf16x8* rest = (TOPK_LDS bf16x8*)&bv_rest[tid];
  bf16x8 bk[NS], bv[NR];
  {
    const int64_t token = at.first + min(key, at.n - 1);
    const uint16_t* k = (const uint16_t*)a.p.k.p + hk * a.p.k.head + token * a.p.k.token + (D / 2) * half;
    const uint16_t* v = (const uint16_t*)a.p.v.p + hk * a.p.v.head + token * a.p.v.token + (D / 2) * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      bk[s] = *(const bf16x8*)(k + 8 * s);
      const bf16x8 x = *(const bf16x8*)(v + 8 * s);
      if (s < NR) bv[s < NR ? s : 0] = x;
      else rest[(s - NR) * NT] = x;  // (read by its own lane alone)
    }
  }
  f32x16 dk[FB], dv[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) dk[f] = dv[f] = (f32x16){};

  // query tiles of each head, from the first that sees a key of the workgroup on; of all heads' as one list the
  // workgroup's share
  const int first = CAUSAL ? at.tile * (PACKED_TILE / ROWS) : 0, per = (at.n + ROWS - 1) / ROWS - first;
  const int begin = (int)((int64_t)per * G * split / splits), tiles = (int)((int64_t)per * G * (split + 1) / splits) - begin;
  const Loader<D, LPW> load_q(a.p.q.token), load_g(a.p.d_out.token);
  // the next tile to load: its place in its head, and where its rows lie
  const int h = hk * G + begin / per;
  int next_t = first + begin % per;
  int t = next_t;  // the current tile's place in its head
  const int64_t token = at.first + next_t * ROWS;
  const unsigned char* qp = (const unsigned char*)((const uint16_t*)a.p.q.p + h * a.p.q.head + token * a.p.q.token);
  const unsigned char* gp = (const unsigned char*)((const uint16_t*)a.p.d_out.p + h * a.p.d_out.head + token * a.p.d_out.token);
  const float* sp = a.p.stat + ((int64_t)(wave & 1) * a.p.H + h) * a.p.N + token;  // lse by the first wave, D by the second
  auto issue = [&](unsigned char* qd, unsigned char* gd, float* sd) TOPK_INLINE {
    const int left = min(ROWS, at.n - next_t * ROWS) - 1;
    load_q(qp, qd, left, wave);
    load_g(gp, gd, left, wave);
    if (wave < 2) __builtin_amdgcn_global_load_lds((const void*)(sp + min(lane, left)), (TOPK_LDS void*)&sd[wave * ROWS], 4, 0, 0);
    qp += ROWS * (int64_t)load_q.sl;
    gp += ROWS * (int64_t)load_g.sl;
    sp += ROWS;
    if (++next_t == first + per) {
      next_t = first;
      qp += a.p.q.head * 2 - per * ROWS * (int64_t)load_q.sl;
      gp += a.p.d_out.head * 2 - per * ROWS * (int64_t)load_g.sl;
      sp += a.p.N - per * ROWS;
    }
  };
  auto tile = [&](bool edge, int t, const unsigned char* qbuf, const unsigned char* gbuf, const float* sbuf) TOPK_INLINE {
    const TOPK_LDS unsigned char *qb = (const TOPK_LDS unsigned char*)qbuf, *gb = (const TOPK_LDS unsigned char*)gbuf;
    const TOPK_LDS float* sb = (const TOPK_LDS float*)sbuf;
    constexpr int AHEAD = 2, AHEAD_T = 4;  // products by which LDS reads run ahead of their use
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      uint32_t row0 = Tile::straight_base(), col0 = Tile::across_base();
      asm volatile("" : "+v"(row0), "+v"(col0));  // (the places that follow from them are not held)
      f32x16 s = {}, g = {};
      auto straight = [&](const TOPK_LDS unsigned char* b, auto&& own, f32x16& to, auto&& also) TOPK_INLINE {
        bf16x8 x[AHEAD + 1];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) x[i] = Tile::straight(b, row0, rb, i);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          if (i + AHEAD < NS) x[(i + AHEAD) % (AHEAD + 1)] = Tile::straight(b, row0, rb, i + AHEAD);
          to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i % (AHEAD + 1)], own(i), to, 0, 0, 0);
          also(i);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      auto weight = [&](int u) TOPK_INLINE {  // of rows 8 u + 4 half ..
        const f32x4 l = *(const TOPK_LDS f32x4*)(sb + rb * 32 + 8 * u + 4 * half);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int v = 4 * u + w;
          s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.c, -l[w]));
        }
      };
      straight(qb, [&](int i) TOPK_INLINE { return bk[i]; }, s, [](int) TOPK_INLINE {});
      straight(gb, [&](int i) TOPK_INLINE { return i < NR ? bv[i < NR ? i : 0] : rest[(i - NR) * NT]; }, g, [&](int i) TOPK_INLINE {
        if (i % (NS / 4) == NS / 4 - 1) weight(i / (NS / 4));
      });
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 e = *(const TOPK_LDS f32x4*)(sb + ROWS + rb * 32 + 8 * u + 4 * half);
#pragma unroll
        for (int w = 0; w < 4; ++w) g[4 * u + w] = s[4 * u + w] * (g[4 * u + w] - e[w]);
      }
      if (edge) {  // the row of register v in the block is 4 half + 8 (v / 4) + v % 4
        const int first_row = t * ROWS + rb * 32 + 4 * half, over = at.n - first_row, under = CAUSAL ? key - first_row : -1;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 8 * (v >> 2) + (v & 3);
          if (r >= over || (CAUSAL && r < under)) s[v] = g[v] = 0.f;
        }
      }
      bf16x8 pb[2], ds[2], pb_lo[2], ds_lo[2];
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        pb[v >> 3][v & 7] = (__bf16)s[v];
        ds[v >> 3][v & 7] = (__bf16)g[v];
        if (TWO) {
          pb_lo[v >> 3][v & 7] = (__bf16)(s[v] - (float)pb[v >> 3][v & 7]);
          ds_lo[v >> 3][v & 7] = (__bf16)(g[v] - (float)ds[v >> 3][v & 7]);
        }
      }
      bf16x8 x[AHEAD_T + 1];
      auto xp = [&](int i) TOPK_INLINE { return Tile::across(i & 1 ? qb : gb, col0, i / 2 % FB, rb * 2 + i / 2 / FB); };
#pragma unroll
      for (int i = 0; i < AHEAD_T; ++i) x[i] = xp(i);
#pragma unroll
      for (int i = 0; i < 4 * FB; ++i) {  // dV and dK in turn
        if (i + AHEAD_T < 4 * FB) x[(i + AHEAD_T) % (AHEAD_T + 1)] = xp(i + AHEAD_T);
        f32x16& to = (i & 1 ? dk : dv)[i / 2 % FB];
        to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i % (AHEAD_T + 1)], (i & 1 ? ds : pb)[i / 2 / FB], to, 0, 0, 0);
        if (TWO) to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i % (AHEAD_T + 1)], (i & 1 ? ds_lo : pb_lo)[i / 2 / FB], to, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // tile i of the list, in the buffers that it is in; the next one's loads go to the others
  __shared__ uint64_t marks[CAUSAL ? NT : 1];
  TOPK_LDS uint64_t* mark = (TOPK_LDS uint64_t*)&marks[tid];
  if (CAUSAL) *mark = 0;
  auto step = [&](auto works, int i, unsigned char* qb, unsigned char* gb, float* sb, unsigned char* qn, unsigned char* gn, float* sn) TOPK_INLINE {
    const bool diagonal = CAUSAL && t * ROWS < at.tile * PACKED_TILE + PACKED_TILE;
    __builtin_amdgcn_s_waitcnt(PACKED_WAIT_VM0);
    // Queries, and gradients of theirs, that are not finite reach only the keys that they see. (To dK by the
    // weights, which lse makes NaN.)
    if (diagonal) {
      const bool any = (int)part_not_finite<LPW>(qb, wave, lane) | (int)part_not_finite<LPW>(gb, wave, lane);
      if (lane == 0) flag[wave][i & 1] = any;
    }
    __syncthreads();
    if (i + 1 < tiles) issue(qn, gn, sn);
    if (diagonal && (flag[0][i & 1] | flag[1][i & 1] | flag[2][i & 1] | flag[3][i & 1])) {
#pragma unroll 1
      for (int j = 0; j < ROWS; ++j) mark_row<D>(mark, gb, j, t * ROWS + j >= key && t * ROWS + j < at.n, half);
      __syncthreads();
      part_clear<LPW>(qb, wave, lane);
      part_clear<LPW>(gb, wave, lane);
      __syncthreads();
    }
    if (decltype(works)::value) tile(diagonal || t * ROWS + ROWS > at.n, t, qb, gb, sb);
    if (++t == first + per) t = first;
  };
  if (tiles > 0) issue(q0, g0, s0);
  auto all = [&](auto works) TOPK_INLINE {
    for (int i = 0; i < tiles; i += 2) {
      step(works, i, q0, g0, s0, q1, g1, s1);
      if (i + 1 < tiles) step(works, i + 1, q1, g1, s1, q0, g0, s0);
    }
  };
  if (work) all(std::true_type{});
  else all(std::false_type{});
  if (CAUSAL) apply_marks<D>(dv, mark);
  __syncthreads();
  TOPK_LDS unsigned char *p0 = (TOPK_LDS unsigned char*)q0, *p1 = (TOPK_LDS unsigned char*)q1, *p2 = (TOPK_LDS unsigned char*)g0,
                         *p3 = (TOPK_LDS unsigned char*)g1;
  TOPK_LDS f32x4* mine = (TOPK_LDS f32x4*)(wave == 0 ? p0 : wave == 1 ? p1 : wave == 2 ? p2 : p3);
  const int r0 = at.tile * PACKED_TILE + wave * 32;
  if (splits > 1) {
    float* part = a.p.part + ((int64_t)(2 * split) * a.p.Hkv + hk) * a.p.N * D + at.first * D;
    store_rows<D>(dk, a.p.scale, mine, part, D, r0, at.n);
    store_rows<D>(dv, 1.f, mine, part + a.p.Hkv * a.p.N * D, D, r0, at.n);
    return;
  }
  store_rows<D>(dk, a.p.scale, mine, (uint16_t*)a.p.dk.p + hk * a.p.dk.head + at.first * a.p.dk.token, a.p.dk.token, r0, at.n);
  store_rows<D>(dv, 1.f, mine, (uint16_t*)a.p.dv.p + hk * a.p.dv.head + at.first * a.p.dv.token, a.p.dv.token, r0, at.n);
}

// The sums of a key tile's shares: eight features a thread. Bound by memory: 254 MB in 48 us.
template <int D>
__global__ __launch_bounds__(NT) void k_packed_sum(BackwardArgs a) {
  const int64_t all = a.p.Hkv * a.p.N * (D / 8), i0 = (int64_t)blockIdx.x * NT + threadIdx.x;
  if (i0 >= 2 * all) return;
  const bool is_v = i0 >= all;
  const int64_t i = is_v ? i0 - all : i0, hk = i / (a.p.N * (D / 8)), r = i - hk * (a.p.N * (D / 8)), t = r / (D / 8);
  const int c = (int)(r % (D / 8)) * 8, N = (int)a.p.N;
  f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
  const int z0 = min(max(a.p.offsets[0], 0), N), z1 = max(z0, min(max(a.p.offsets[a.p.n], 0), N));
  if (t >= z0 && t < z1) {
    const float* p = a.p.part + ((is_v ? a.p.Hkv : 0) + hk) * a.p.N * D + t * D + c;
    for (int s = 0; s < a.p.splits; ++s, p += 2 * a.p.Hkv * a.p.N * D) {
      x += *(const f32x4*)p;
      y += *(const f32x4*)(p + 4);
    }
  }
  const PackedRows& to = is_v ? a.p.dv : a.p.dk;
  *(uint4*)((uint16_t*)to.p + hk * to.head + t * to.token + c) =
      make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
}

template <int D, bool CAUSAL>
void launch_d(const BackwardArgs& a, hipStream_t st) {
  const int64_t rows = a.p.H * a.p.N, per = NT / (D / 8);
  k_packed_stat<D><<<(unsigned)((rows + per - 1) / per), NT, 0, st>>>(a);
  const unsigned q_wgs = (unsigned)(packed_tiles(a.p) * a.p.H), half_q_wgs = (unsigned)(packed_tiles(a.p, PACKED_TILE / 2) * a.p.H),
                 kv_wgs = (unsigned)(packed_tiles(a.p) * a.p.Hkv * a.p.splits);
  if (packed_short(a.p)) {
    k_packed_dq<D, CAUSAL, 2, true><<<half_q_wgs, NT, 0, st>>>(a);
    k_packed_dkv<D, CAUSAL, true><<<kv_wgs, NT, 0, st>>>(a);
  } else {
    if (packed_few(a.p, a.p.H)) k_packed_dq<D, CAUSAL, 2, false><<<half_q_wgs, NT, 0, st>>>(a);
    else k_packed_dq<D, CAUSAL, 1, false><<<q_wgs, NT, 0, st>>>(a);
    k_packed_dkv<D, CAUSAL, false><<<kv_wgs, NT, 0, st>>>(a);
  }
  if (a.p.splits > 1) k_packed_sum<D><<<(unsigned)((2 * a.p.Hkv * a.p.N * (D / 8) + NT - 1) / NT), NT, 0, st>>>(a);
}

}  // namespace

// Shares of a key tile's queries. With sequences of N / n tokens the longest workgroup goes over (N / n) / 64 tiles
// of each of G heads, and the chip's 512 (two a CU) over H n (N / n)^2 / 8192 in all, half of it where causal;
// a tile is shared out until the longest has no more than three quarters of the average, or into SPLITS.
static int packed_splits(const PackedProblem& p) {
  constexpr int SPLITS = 8;
  const double L = (double)p.N / p.n, longest = L / ROWS * (p.H / p.Hkv), all = (double)p.H * p.n * L * L / (ROWS * PACKED_TILE) / (p.causal ? 2 : 1) / 512;
  int s = 1;
  while (s < SPLITS && longest / s > 0.75 * all && longest / s > 8) ++s;
  return s;
}

static size_t stat_bytes(const PackedProblem& p) { return ((size_t)p.H * p.N * 2 * sizeof(float) + 255) / 256 * 256; }
size_t packed_backward_bytes(const PackedProblem& p) {
  const int s = packed_splits(p);
  return stat_bytes(p) + (s > 1 ? (size_t)s * 2 * p.Hkv * p.N * p.d * sizeof(float) : 0);
}

hipError_t launch_packed_backward(PackedProblem p, void* ws, hipStream_t st) {
  p.splits = packed_splits(p);
  p.stat = (float*)ws;
  p.part = (float*)((char*)ws + stat_bytes(p));
  const BackwardArgs a = {p, p.scale * 1.4426950408889634f};
  if (p.d == 64 && p.causal) launch_d<64, true>(a, st);
  else if (p.d == 64) launch_d<64, false>(a, st);
  else if (p.causal) launch_d<128, true>(a, st);
  else launch_d<128, false>(a, st);
  return hipGetLastError();
}

}  // namespace topk
