// Internal interface of shared-prefix attention (topk_prefix.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace topk {

struct PrefixProblem {
  const void* q;             // [B, H, Lq, d]
  void* out;                 // [B, H, Lq, d]
  float* lse;                // [B, H, Lq] or NULL
  const void *pk, *pv;       // shared: head h, key j at h * p?_sh + j * p?_sl
  int64_t pk_sh, pk_sl, pv_sh, pv_sl;
  const void *k, *v;         // own: request b, head h, key j at b * ?_sb + h * ?_sh + j * ?_sl
  int64_t k_sb, k_sh, k_sl, v_sb, v_sh, v_sl;
  const int32_t* lengths;    // own keys of each request (NULL: S of each)
  int64_t B, H, Hkv, Lq, P, S;
  int d, causal;
  float scale;
};

// How the work is cut: row tiles, and key ranges whose partial results are joined.
struct PrefixPlan {
  int pform, sform;        // forms of the items on the prefix and on own keys (see k_prefix)
  int both;                // items of one request take both, ranges of pkeys of the two as one list
  int64_t rows;            // B * H * Lq
  int64_t req_rows;        // rows of one request and key head: (H / Hkv) * Lq
  int64_t ptiles, psplits, pkeys;  // prefix: row tiles of a key head, key ranges, keys of a range
  int64_t stiles, ssplits, skeys;  // own keys: row tiles of a request and key head, ...
  int64_t splits;          // partial results of a row
};

PrefixPlan prefix_plan(const PrefixProblem& pp);
constexpr int64_t PREFIX_MAX_ITEMS = 0xFFFFFF;  // workgroups of a launch
int64_t prefix_items(const PrefixProblem& pp, const PrefixPlan& pl);
size_t prefix_bytes(const PrefixProblem& pp, const PrefixPlan& pl);
hipError_t launch_prefix(const PrefixProblem& pp, const PrefixPlan& pl, void* ws, hipStream_t st);
hipError_t launch_prefix_join(const PrefixProblem& pp, const PrefixPlan& pl, const void* ws, hipStream_t st);

}  // namespace topk
