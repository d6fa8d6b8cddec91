// Internal interface of attention over a cache in pages (topk_tree.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace topk {

struct TreeProblem {
  const void* q;           // [B, H, T, d]
  void* out;               // [B, H, T, d]
  float* lse;              // [B, H, T] or NULL
  const void* pool[2];     // keys, values: head h, row r of page p at p * page + h * head + r * row
  int64_t page[2], head[2], row[2];
  const int32_t* table;    // [B, M] at b * table_stride; NULL: request b has page b
  int64_t table_stride;
  const int32_t* lengths;  // [B]
  const int32_t* parents;  // [B, T] at b * parents_stride; NULL: each draft follows the one before it
  int64_t parents_stride;
  int64_t B, M, n_pages, page_rows;
  int H, Hkv, T, d;
  float scale;
};

// How the work is cut: row tiles of a request and key head, and key ranges. Which request a range is of is
// found on the device from the lengths: there are `ranges` + B of them at most.
struct TreePlan {
  int form;        // 1, 2: blocks of 16 rows; 3, 4: the same, pages of whole groups of four keys; 8, 9: 128 rows
                   // (weights as two bf16 numbers, as one)
  int tiles;       // row tiles of (H / Hkv) * T rows
  int64_t ranges;  // wanted, of all requests together; 0: one a request
  int round;       // ranges whose workgroups fill the chip once
};

constexpr int TREE_MAX = 64;  // drafts of a request
TreePlan tree_plan(const TreeProblem& p);
int64_t tree_workgroups(const TreeProblem& p, const TreePlan& pl);
size_t tree_bytes(const TreeProblem& p, const TreePlan& pl);
hipError_t launch_tree(const TreeProblem& p, const TreePlan& pl, void* ws, hipStream_t st);
hipError_t launch_tree_join(const TreeProblem& p, const TreePlan& pl, const void* ws, hipStream_t st);

}  // namespace topk
