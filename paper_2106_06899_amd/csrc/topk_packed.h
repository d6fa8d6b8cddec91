// Internal interface of packed attention (topk_packed.hip, topk_packed_bwd.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace topk {

// Heads of packed tokens: head h, token t at h * head + t * token elements.
struct PackedRows {
  void* p;
  int64_t head, token;
};

struct PackedProblem {
  PackedRows q, k, v, out;
  PackedRows d_out, dq, dk, dv;  // (backward)
  float* lse;                    // [H, N], contiguous; NULL: not written
  void* rest;                    // laid out as out, or NULL: what rounding took from it
  const int32_t* offsets;        // [n + 1]
  int64_t N;
  int n, H, Hkv, d, causal;
  float scale;
  // (backward) workspace
  float* stat;  // [2, H, N]: lse to base 2; sum of d_out * out
  float* part;  // splits > 1: [splits, 2, Hkv, N, d] shares of dK and dV
  int splits;
};

constexpr int PACKED_TILE = 128;  // rows of a workgroup
// workgroups of a head at most, of so many rows, and one more, so that one is left for the tokens of no sequence
int64_t packed_tiles(const PackedProblem& p, int rows = PACKED_TILE);
// so few workgroups of PACKED_TILE rows that half as many rows are better
bool packed_few(const PackedProblem& p, int heads);
// so few tokens, or so short sequences, that the training pass may as well have its weights and score gradients as two
// bf16 numbers
bool packed_short(const PackedProblem& p);
size_t packed_backward_bytes(const PackedProblem& p);
hipError_t launch_packed(const PackedProblem& p, hipStream_t st);
hipError_t launch_packed_backward(PackedProblem p, void* ws, hipStream_t st);

}  // namespace topk
