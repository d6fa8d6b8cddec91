// Internal interface between the host side (topk_api.hip) and the kernels of the head
// preparation (topk_rope.hip) and of shared-prefix attention (topk_prefix.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace topk {

constexpr int ROPE_MAX_D = 512;
constexpr int ROPE_MAX_AXES = 4;

// A tensor of head rows: row (b, h, l) starts at p + b * sb + h * sh + l * sl elements.
struct HeadRows {
  void* p;
  int64_t sb, sh, sl;
};

// The rotation: pair p of a token turns by positions[axis(p)] * freqs[p].
struct Rotation {
  const void* positions;
  const double* freqs;
  int64_t pos_sa, pos_sb, pos_sl;
  int half;      // pairs
  int pos64;     // positions are int64 (int32 otherwise)
  int adjacent;  // pair p = features 2p, 2p + 1 (p, p + half otherwise)
  int inverse;   // turn by the opposite angles
  uint32_t axis[ROPE_MAX_D / 2 / 16];  // two bits a pair
};

// Heads [0, H) are queries, [H, H + Hkv) keys, [H + Hkv, H + 2 Hkv) values of one packed row;
// rope alone is H query heads without norm or weight.
struct HeadsProblem {
  HeadRows x;         // packed input, heads in order
  HeadRows part[3];   // q, k, v: outputs of a forward call, incoming gradients of a backward call
  HeadRows dx;        // backward: gradient of the packed input
  const void* w[2];   // norm weights of q and k heads (NULL: ones)
  void* dw[2];        // backward: their gradients (NULL: not wanted)
  float* dw_part;     // backward: sums of each workgroup
  int64_t B, L, heads[3];
  int d, dtype, norm;
  float eps;
  const int32_t* lengths;  // append: keys and values go to rows lengths[b] + l of caches of S rows
  int64_t S;
  Rotation rot;
};

hipError_t launch_heads(const HeadsProblem& hp, hipStream_t st);
hipError_t launch_heads_backward(const HeadsProblem& hp, hipStream_t st);
size_t heads_backward_bytes(const HeadsProblem& hp);

}  // namespace topk
