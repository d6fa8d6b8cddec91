// What happens to heads between the projection and the attention: the packed [q | k | v] row
// of each token is taken apart into heads, query and key heads are divided by their root mean
// square, scaled and rotated by the token's positions.
//
//   r = (sum_f x_f^2 / d + eps)^(-1/2),  u = x r,  n = w u  (each a head of d features)
//   y_a = n_a cos t - n_b sin t,  y_b = n_a sin t + n_b cos t   for each pair (a, b) = p,
//   t = position[axis(p)] * freq[p]
// and backward, with m = the rotation by -t of the incoming gradient:
//   dw = sum over tokens and heads of m u,   dx = r (m w - u mean(m w u)).
// Without a norm dx = m, which x has no part in (an infinite x would make 0 x of it NaN).
//
// Bound by memory: every element is read once and written once (backward: x and the gradient
// read, one gradient written), so the design is about whole cache lines and few instructions.
// A group of T lanes holds one head, each lane VEC pairs (both features of a pair, so the
// rotation needs no exchange) by two accesses of VEC elements. A workgroup works on `tok` consecutive
// tokens and `hp` heads at a time, each lane staying with its token and features: the angles of
// the workgroup's tokens are computed once, by all its lanes, and go through LDS to registers,
// where every head reuses them. Input is read in runs of hp heads, and each head is written in
// runs of tok tokens. Angles are products in 64 bits, reduced to a turn there (32 bits would
// lose 0.06 rad at position 10^6), and only the fraction of a turn goes to a 32-bit sine. Squares,
// means and the weights' gradients are sums in 32 bits; results are rounded once.
//
// Measured (a device copy reaches 4.94 TB/s): 4 x 8192 tokens of 16 + 16 + 16 heads of 128, bf16,
// 169 us (4.8 TB/s); rotation of 2 x 16 heads of 8192 tokens, three axes, 29 us (4.6 TB/s); 8 x 512
// tokens of 12 + 12 + 12 heads of 64, where latency counts, 11 us forward (3.4 TB/s), 16 + 4 us
// backward (4 x 8192: 91 + 5, 5.0 TB/s; without a norm 73 in all, 84 where x was read all the same).
// With the angles formed by each lane for itself, one head at a time: 188, 30, 16, 31 + 9. Measured and
// left: the next head's loads issued ahead of this one's arithmetic (11.4 us forward, 13.4; the
// backward the same).
#include "topk_device.h"
#include "topk_heads.h"

#include <algorithm>

namespace topk {
namespace {

constexpr int NT = 256;  // threads of a workgroup

template <typename T, int N> struct Vec {
  T e[N];
};
template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<uint16_t>(uint16_t v) { return bf16_to_f32(v); }

// VEC consecutive elements, at an address that is a multiple of their size
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(float (&o)[VEC], const T* p) {
  Vec<T, VEC> v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p, sizeof(T) * VEC), sizeof(T) * VEC);
#pragma unroll
  for (int e = 0; e < VEC; ++e) o[e] = widen(v.e[e]);
}
// What a lane holds of a head as it lies in memory: both runs of VEC of each chunk.
template <typename T, int VEC, int NC> struct Raw {
  Vec<T, VEC> a[NC], b[NC];
};
template <typename T, int VEC>
__device__ __forceinline__ void widen_vec(float (&o)[VEC], const Vec<T, VEC>& v) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) o[e] = widen(v.e[e]);
}
template <int VEC>
__device__ __forceinline__ void store_vec(float* p, const float (&o)[VEC]) {
  __builtin_memcpy(__builtin_assume_aligned(p, 4 * VEC), o, 4 * VEC);
}
template <int VEC>
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&o)[VEC]) {
  typedef __bf16 bf16;
  bf16 v[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) v[e] = (bf16)o[e];  // nearest-even
  __builtin_memcpy(__builtin_assume_aligned(p, 2 * VEC), v, 2 * VEC);
}

constexpr int64_t WGS = 768;     // workgroups that fill the chip

struct Grid {
  int T;             // lanes of a head: a power of two, at least d / (2 VEC NC)
  int hp;            // heads at a time (a power of two)
  int tok;           // tokens of a workgroup: NT / (T hp)
  int64_t tiles;     // tiles of tok tokens
  int ny[3];         // workgroups that share the heads of q, k, v
  int per[3];        // heads of each
};

// A lane's place: its chunks' features and its token.
template <int VEC, int NC, bool ADJ>
struct Lane {
  int lo[NC], hi[NC];  // first features of the two runs of VEC (of pairs p .. p + VEC - 1, or not rotated)
  bool in[NC], turn[NC];
  int pair[NC];
  __device__ Lane(int c0, int T, int d, int half) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = c0 + j * T, p = c * VEC;
      in[j] = 2 * p < d;
      turn[j] = in[j] && p < half;
      pair[j] = turn[j] ? p : 0;
      if (ADJ || p >= half) {
        lo[j] = in[j] ? 2 * p : 0;
        hi[j] = lo[j] + (in[j] ? VEC : 0);
      } else {
        lo[j] = p;
        hi[j] = p + half;
      }
    }
  }
};

template <typename T, int VEC, int NC, bool ADJ>
__device__ __forceinline__ void fetch(Raw<T, VEC, NC>& r, const T* p, const Lane<VEC, NC, ADJ>& ln) {
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    r.a[j] = r.b[j] = Vec<T, VEC>{};
    if (ln.in[j]) {
      __builtin_memcpy(&r.a[j], __builtin_assume_aligned(p + ln.lo[j], sizeof(T) * VEC), sizeof(T) * VEC);
      __builtin_memcpy(&r.b[j], __builtin_assume_aligned(p + ln.hi[j], sizeof(T) * VEC), sizeof(T) * VEC);
    }
  }
}

// cos and sin of all pairs of the workgroup's tokens, from token t0 on, to LDS: [token][pair]
__device__ __forceinline__ void angles(const HeadsProblem& hp, const Grid& g, int64_t t0, float2* out) {
  const Rotation& r = hp.rot;
  const int64_t left = hp.B * hp.L - t0;
  const int n = (int)min((int64_t)g.tok, left) * r.half;
  for (int i = threadIdx.x; i < n; i += NT) {
    const int t = i / r.half, p = i - t * r.half;
    const int64_t b = (t0 + t) / hp.L, l = t0 + t - b * hp.L;
    const int a = (r.axis[p >> 4] >> (2 * (p & 15))) & 3;
    const int64_t o = b * r.pos_sb + l * r.pos_sl + a * r.pos_sa;
    const double pos = r.pos64 ? (double)((const int64_t*)r.positions)[o] : (double)((const int32_t*)r.positions)[o];
    const double turns = pos * r.freqs[p] * 0.15915494309189533577;  // 1 / (2 pi)
    const float f = 2.f * (float)(turns - rint(turns));              // in half turns, [-1, 1]
    float sn, cs;
    sincospif(f, &sn, &cs);
    out[i] = make_float2(cs, r.inverse ? -sn : sn);
  }
}
// the lane's, from there
template <int VEC, int NC, bool ADJ>
__device__ __forceinline__ void lane_angles(const Rotation& r, const Lane<VEC, NC, ADJ>& ln, const float2* of_token, float (&co)[NC][VEC],
                                            float (&si)[NC][VEC]) {
#pragma unroll
  for (int j = 0; j < NC; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float2 x = ln.turn[j] ? of_token[ln.pair[j] + e] : make_float2(1.f, 0.f);
      co[j][e] = x.x;
      si[j][e] = x.y;
    }
}

// Rotates the lane's pairs by (co, si). Chunks that are not rotated do not come here: x 1 - x' 0 is
// NaN where x' is not finite.
template <int VEC, bool ADJ>
__device__ __forceinline__ void turn_pairs(float (&a)[VEC], float (&b)[VEC], const float (&co)[VEC], const float (&si)[VEC]) {
  float x[2 * VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = a[e], x[VEC + e] = b[e];
  float y[2 * VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int i = ADJ ? 2 * e : e, k = ADJ ? 2 * e + 1 : VEC + e;
    y[i] = fmaf(x[i], co[e], -x[k] * si[e]);
    y[k] = fmaf(x[i], si[e], x[k] * co[e]);
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = y[e], b[e] = y[VEC + e];
}

__device__ __forceinline__ float group_sum(float v, int T) {
  for (int o = T >> 1; o; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// which of q, k, v a workgroup works on, and its heads
struct Share {
  int seg;
  int64_t h0, h1, first;  // heads [h0, h1) of the part, whose first head is `first` of the packed row
  __device__ Share(const HeadsProblem& hp, const Grid& g, int y) {
    seg = 0;
    first = 0;
    while (seg < 2 && y >= g.ny[seg]) {
      first += hp.heads[seg];
      y -= g.ny[seg++];
    }
    h0 = (int64_t)y * g.per[seg];
    h1 = min(h0 + g.per[seg], hp.heads[seg]);
  }
};

// A workgroup takes one part's heads of a tile of tokens (more tiles only where a grid cannot hold
// them all).
template <typename T, int VEC, int NC, bool ADJ>
__global__ __launch_bounds__(NT) void k_heads(HeadsProblem hp, Grid g) {
  __shared__ __attribute__((aligned(16))) float2 ang[NT * VEC * NC];  // (a lane's pairs are NC chunks of VEC)
  const Share sh(hp, g, blockIdx.y);
  const int lane = threadIdx.x & (g.T - 1), unit = threadIdx.x / g.T, tl = unit & (g.tok - 1), first = unit / g.tok;
  const Lane<VEC, NC, ADJ> ln(lane, g.T, hp.d, hp.rot.half);
  const bool value = sh.seg == 2;
  float wa[NC][VEC], wb[NC][VEC];
  const T* w = value ? nullptr : (const T*)hp.w[sh.seg];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) wa[j][e] = wb[j][e] = 1.f;
    if (w && ln.in[j]) {
      load_vec<T, VEC>(wa[j], w + ln.lo[j]);
      load_vec<T, VEC>(wb[j], w + ln.hi[j]);
    }
  }
  const float inv_d = 1.f / (float)hp.d;
  for (int64_t t = blockIdx.x; t < g.tiles; t += gridDim.x) {
    const int64_t token = t * g.tok + tl, b = token / hp.L, l = token - b * hp.L, h0 = sh.h0 + first;
    bool live = token < hp.B * hp.L && h0 < sh.h1;  // (of whole groups)
    int64_t row = l;
    if (live && hp.lengths && sh.seg > 0) {
      row = (int64_t)hp.lengths[b] + l;
      live = row >= 0 && row < hp.S;  // (otherwise there is no place in the cache)
    }
    const HeadRows& o = hp.part[sh.seg];
    const T* src = (const T*)hp.x.p + b * hp.x.sb + l * hp.x.sl + (sh.first + h0) * hp.x.sh;
    T* dst = (T*)o.p + b * o.sb + row * o.sl + h0 * o.sh;
    float co[NC][VEC], si[NC][VEC];
    if (!value && hp.rot.half) {
      if (t != blockIdx.x) __syncthreads();
      angles(hp, g, t * g.tok, ang);
      __syncthreads();
    }
    if (!value) lane_angles(hp.rot, ln, ang + tl * hp.rot.half, co, si);
    if (!live) continue;
    for (int64_t h = h0; h < sh.h1; h += g.hp, src += g.hp * hp.x.sh, dst += g.hp * o.sh) {
      Raw<T, VEC, NC> raw;
      fetch(raw, src, ln);
      float a[NC][VEC], c[NC][VEC];
      float sq = 0.f;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        widen_vec(a[j], raw.a[j]);
        widen_vec(c[j], raw.b[j]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sq = fmaf(a[j][e], a[j][e], fmaf(c[j][e], c[j][e], sq));
      }
      if (!value) {
        const float r = hp.norm ? rsqrtf(fmaf(group_sum(sq, g.T), inv_d, hp.eps)) : 1.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            a[j][e] *= r * wa[j][e];
            c[j][e] *= r * wb[j][e];
          }
          if (ln.turn[j]) turn_pairs<VEC, ADJ>(a[j], c[j], co[j], si[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < NC; ++j)
        if (ln.in[j]) {
          store_vec<VEC>(dst + ln.lo[j], a[j]);
          store_vec<VEC>(dst + ln.hi[j], c[j]);
        }
    }
  }
}

// Backward: workgroups walk over tiles of tokens (gridDim.x apart) so that the weights'
// gradients stay in registers; each writes its own sum, in a fixed order over its groups.
template <typename T, int VEC, int NC, bool ADJ>
__global__ __launch_bounds__(NT) void k_heads_backward(HeadsProblem hp, Grid g) {
  __shared__ __attribute__((aligned(16))) float2 ang[NT * VEC * NC];  // (a lane's pairs are NC chunks of VEC)
  __shared__ float red[NT * NC * VEC];
  const Share sh(hp, g, blockIdx.y);
  const int lane = threadIdx.x & (g.T - 1), unit = threadIdx.x / g.T, tl = unit & (g.tok - 1), first = unit / g.tok;
  const Lane<VEC, NC, ADJ> ln(lane, g.T, hp.d, hp.rot.half);
  const bool value = sh.seg == 2, norm = !value && hp.norm;  // (the gradient depends on x through the norm alone)
  float wa[NC][VEC], wb[NC][VEC], ga[NC][VEC], gb[NC][VEC];
  const T* w = value ? nullptr : (const T*)hp.w[sh.seg];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      wa[j][e] = wb[j][e] = 1.f;
      ga[j][e] = gb[j][e] = 0.f;
    }
    if (w && ln.in[j]) {
      load_vec<T, VEC>(wa[j], w + ln.lo[j]);
      load_vec<T, VEC>(wb[j], w + ln.hi[j]);
    }
  }
  const float inv_d = 1.f / (float)hp.d;
  for (int64_t t = blockIdx.x; t < g.tiles; t += gridDim.x) {
    const int64_t token = t * g.tok + tl, b = token / hp.L, l = token - b * hp.L, h0 = sh.h0 + first;
    const bool live = token < hp.B * hp.L && h0 < sh.h1;  // (of whole groups)
    const HeadRows& gr = hp.part[sh.seg];
    const T* src = (const T*)hp.x.p + b * hp.x.sb + l * hp.x.sl + (sh.first + h0) * hp.x.sh;
    const T* grad = (const T*)gr.p + b * gr.sb + l * gr.sl + h0 * gr.sh;
    T* dst = (T*)hp.dx.p + b * hp.dx.sb + l * hp.dx.sl + (sh.first + h0) * hp.dx.sh;
    float co[NC][VEC], si[NC][VEC];
    if (!value && hp.rot.half) {
      if (t != blockIdx.x) __syncthreads();
      angles(hp, g, t * g.tok, ang);
      __syncthreads();
    }
    if (!value) lane_angles(hp.rot, ln, ang + tl * hp.rot.half, co, si);
    if (!live) continue;
    for (int64_t h = h0; h < sh.h1; h += g.hp, dst += g.hp * hp.dx.sh) {
      Raw<T, VEC, NC> rawx, rawg;
      fetch(rawg, grad, ln);
      if (norm) fetch(rawx, src, ln);
      src += g.hp * hp.x.sh;
      grad += g.hp * gr.sh;
      float ma[NC][VEC], mb[NC][VEC];
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        widen_vec(ma[j], rawg.a[j]);
        widen_vec(mb[j], rawg.b[j]);
        if (!value && ln.turn[j]) turn_pairs<VEC, ADJ>(ma[j], mb[j], co[j], si[j]);  // (the launch asks for the opposite angles)
      }
      if (norm) {
        float xa[NC][VEC], xb[NC][VEC];
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          widen_vec(xa[j], rawx.a[j]);
          widen_vec(xb[j], rawx.b[j]);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            sq = fmaf(xa[j][e], xa[j][e], fmaf(xb[j][e], xb[j][e], sq));
            dot = fmaf(ma[j][e] * wa[j][e], xa[j][e], fmaf(mb[j][e] * wb[j][e], xb[j][e], dot));
          }
        }
        const float r = rsqrtf(fmaf(group_sum(sq, g.T), inv_d, hp.eps)), mean = r * group_sum(dot, g.T) * inv_d;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {  // dx = r (m w - u mean)
            const float ua = xa[j][e] * r, ub = xb[j][e] * r;
            ga[j][e] = fmaf(ma[j][e], ua, ga[j][e]);
            gb[j][e] = fmaf(mb[j][e], ub, gb[j][e]);
            ma[j][e] = r * fmaf(wa[j][e], ma[j][e], -mean * ua);
            mb[j][e] = r * fmaf(wb[j][e], mb[j][e], -mean * ub);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < NC; ++j)
        if (ln.in[j]) {
          store_vec<VEC>(dst + ln.lo[j], ma[j]);
          store_vec<VEC>(dst + ln.hi[j], mb[j]);
        }
    }
  }
  if (value || !hp.dw_part) return;
  // the groups' sums: [group][lane][NC][VEC], first features then second ones
  const int y = blockIdx.y - (sh.seg ? g.ny[0] : 0);
  float* out = hp.dw_part + ((sh.seg ? (int64_t)gridDim.x * g.ny[0] : 0) + (int64_t)y * gridDim.x + blockIdx.x) * hp.d;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    if (part) __syncthreads();
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) red[(j * VEC + e) * NT + threadIdx.x] = part ? gb[j][e] : ga[j][e];
    __syncthreads();
    // (one thread per lane place and value; NT threads cover T * NC * VEC values)
    for (int i = threadIdx.x; i < g.T * NC * VEC; i += NT) {
      const int c = i % g.T, v = i / g.T, j = v / VEC, e = v % VEC;
      float s = 0.f;
      for (int q = c; q < NT; q += g.T) s += red[v * NT + q];
      const Lane<VEC, 1, ADJ> at(c + j * g.T, 1, hp.d, hp.rot.half);
      if (at.in[0]) out[(part ? at.hi[0] : at.lo[0]) + e] = s;
    }
  }
}

// The weights' gradients, 16 columns of one a workgroup: the workgroups' sums, in a fixed order.
template <typename T>
__global__ __launch_bounds__(1024) void k_heads_weights(const float* part, T* dq, T* dk, int64_t nq, int64_t nk, int d) {
  __shared__ float red[64][17];
  T* dw = blockIdx.y ? dk : dq;
  if (!dw) return;
  const int64_t n = blockIdx.y ? nk : nq;
  if (blockIdx.y) part += nq * d;
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float s = 0.f;
  if (col < d) {
#pragma unroll 4
    for (int64_t i = q; i < n; i += 64) s += part[i * d + col];
  }
  red[q][c] = s;
  __syncthreads();
  for (int o = 32; o; o >>= 1) {
    if (q < o) red[q][c] += red[q + o][c];
    __syncthreads();
  }
  if (q == 0 && col < d) store_elem<T>(dw, col, red[0][c]);
}

// Whether sizes, strides and addresses let a lane move four elements at once (8 bytes of bf16; 16 are no
// faster). One at a time takes 273 us where four take 169 (8192-token prefill), 11.1 and 9.4 in 32 bits
// (2 x 1511 tokens of 4 + 2 + 2 heads of 96).
bool rows_fit(const HeadRows& r, int es) {
  return !r.p || (((uintptr_t)r.p) % (4 * es) == 0 && r.sb % 4 == 0 && r.sh % 4 == 0 && r.sl % 4 == 0);
}
int vector_for(const HeadsProblem& hp) {
  const int es = hp.dtype ? 2 : 4;
  bool ok = hp.rot.half % 4 == 0 && hp.d % 8 == 0 && rows_fit(hp.x, es) && rows_fit(hp.dx, es);
  for (int s = 0; s < 3; ++s) ok = ok && rows_fit(hp.part[s], es);
  for (int s = 0; s < 2; ++s) ok = ok && ((uintptr_t)hp.w[s]) % (4 * es) == 0;
  return ok ? 4 : 1;
}

Grid grid_for(const HeadsProblem& hp, int vec) {
  Grid g = {};
  const int chunks = hp.d / 2 / vec, nc = vec == 1 ? 4 : 1;
  g.T = 1;
  while (g.T * nc < chunks && g.T < 64) g.T *= 2;
  // four heads at a time, fewer where there are fewer or where a head takes a wave: the angles are
  // then a small part, and runs stay long (two: 172 us where four take 165, eight: 31 for 28 us)
  g.hp = 1;
  while (g.hp < 4 && g.hp < hp.heads[0] && g.T * g.hp < NT / 4) g.hp *= 2;
  g.tok = NT / (g.T * g.hp);
  const int64_t tokens = hp.B * hp.L;
  g.tiles = (tokens + g.tok - 1) / g.tok;
  // heads of a workgroup: as many as leave WGS workgroups (8 x 512 tokens: 11.3 us, 14.4 with 2048)
  const int64_t total = hp.heads[0] + hp.heads[1] + hp.heads[2];
  int64_t per = g.tiles >= WGS ? total : g.tiles * total / WGS;
  per = std::max<int64_t>(g.hp, per / g.hp * g.hp);
  for (int s = 0; s < 3; ++s) {
    g.ny[s] = (int)((hp.heads[s] + per - 1) / per);
    g.per[s] = g.ny[s] ? (int)((hp.heads[s] + g.ny[s] - 1) / g.ny[s]) : 1;
  }
  return g;
}
int backward_blocks(const Grid& g) {
  // each walks over as many tiles as the next, and as leaves 4096 workgroups: parts differ in heads, and values
  // take less (2 x 8192 tokens of 48 heads of 128, 32 of them queries: 127 us, 186 with 1024, 230 with 768; 2 x 1511
  // of 8 heads of 96 in fp32: 13.4, 12.0 with 1024)
  const int64_t y = g.ny[0] + g.ny[1] + g.ny[2], each = std::max<int64_t>(1, g.tiles * y / 4096);
  return (int)((g.tiles + each - 1) / each);
}

template <typename T, int VEC, int NC>
void launch_adj(const HeadsProblem& hp, const Grid& g, dim3 grid, bool backward, hipStream_t st) {
  if (backward) {
    if (hp.rot.adjacent) k_heads_backward<T, VEC, NC, true><<<grid, NT, 0, st>>>(hp, g);
    else k_heads_backward<T, VEC, NC, false><<<grid, NT, 0, st>>>(hp, g);
  } else {
    if (hp.rot.adjacent) k_heads<T, VEC, NC, true><<<grid, NT, 0, st>>>(hp, g);
    else k_heads<T, VEC, NC, false><<<grid, NT, 0, st>>>(hp, g);
  }
}
void launch_any(const HeadsProblem& hp, int vec, const Grid& g, dim3 grid, bool backward, hipStream_t st) {
  if (hp.dtype) {
    if (vec == 4) launch_adj<uint16_t, 4, 1>(hp, g, grid, backward, st);
    else launch_adj<uint16_t, 1, 4>(hp, g, grid, backward, st);
  } else {
    if (vec == 4) launch_adj<float, 4, 1>(hp, g, grid, backward, st);
    else launch_adj<float, 1, 4>(hp, g, grid, backward, st);
  }
}

}  // namespace

hipError_t launch_heads(const HeadsProblem& hp, hipStream_t st) {
  const int vec = vector_for(hp);
  const Grid g = grid_for(hp, vec);
  launch_any(hp, vec, g, dim3((unsigned)std::min<int64_t>(g.tiles, 1 << 20), g.ny[0] + g.ny[1] + g.ny[2]), false, st);
  return hipGetLastError();
}

size_t heads_backward_bytes(const HeadsProblem& hp) {
  // of either form: which one runs depends on the addresses
  size_t most = 0;
  for (int vec : {4, 1}) {
    if (vec > 1 && (hp.rot.half % vec || (hp.d / 2) % vec)) continue;
    const Grid g = grid_for(hp, vec);
    most = std::max(most, (size_t)backward_blocks(g) * (g.ny[0] + g.ny[1]) * hp.d * 4);
  }
  return most;
}

hipError_t launch_heads_backward(const HeadsProblem& hp, hipStream_t st) {
  const int vec = vector_for(hp);
  const Grid g = grid_for(hp, vec);
  const int gx = backward_blocks(g);
  launch_any(hp, vec, g, dim3(gx, g.ny[0] + g.ny[1] + g.ny[2]), true, st);
  if (hp.dw[0] || hp.dw[1]) {
    const dim3 grid((hp.d + 15) / 16, 2);
    const int64_t nq = (int64_t)gx * g.ny[0], nk = (int64_t)gx * g.ny[1];
    if (hp.dtype) k_heads_weights<uint16_t><<<grid, 1024, 0, st>>>(hp.dw_part, (uint16_t*)hp.dw[0], (uint16_t*)hp.dw[1], nq, nk, hp.d);
    else k_heads_weights<float><<<grid, 1024, 0, st>>>(hp.dw_part, (float*)hp.dw[0], (float*)hp.dw[1], nq, nk, hp.d);
  }
  return hipGetLastError();
}

}  // namespace topk
