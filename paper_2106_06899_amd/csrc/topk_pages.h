// Internal interface of the page calls (topk_pages.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace topk {

// Pools of keys and values: row r of page p, head h, layer l at l * layer + p * page + h * head + r * row
// elements of each.
struct PagePool {
  void* p[2];  // keys, values
  int64_t layer[2], page[2], head[2], row[2];
};
struct PageShape {
  int64_t layers, heads, n_pages;
  int page_rows;
  int pieces;  // 16-byte pieces of a row
  int es;      // bytes of an element
};
// Which pages each request holds: entry e of request b at table[b * stride + e], -1 where it holds none.
struct PageTable {
  int32_t* at;
  int64_t stride;
  int B, M;
};

constexpr int KEEP_MAX = 64;  // accepted drafts of a request

struct ReserveArgs {
  PagePool pool;
  PageShape s;
  PageTable t;
  int32_t *refs, *missing;
  const int32_t *lengths, *rows_each;
  int64_t rows;
  int32_t *kind, *free_list;  // workspace: an entry of the tables each; pages found free
  int4* copies;               // [B + 1]: how many follow; from, to, rows of each
  int32_t* listed;            // large pools: [cdiv(n_pages, FREE_BLOCK)] free pages of a block; and which, [n_pages]
};
struct AppendArgs {
  PagePool pool, from;  // from: `page` is a request's stride (or unused), `row` a token's
  PageShape s;
  PageTable t;
  const int32_t *lengths, *offsets;
  int64_t T;  // tokens of each request; with offsets: of all
};
struct KeepArgs {
  PagePool pool;
  PageShape s;
  PageTable t;
  const int32_t *lengths, *kept;
  int32_t* new_lengths;
  int64_t kept_stride;
  int A;
};
struct ForkArgs {
  PageTable t;
  int32_t *refs, *lengths;
  const int32_t* parents;
  int64_t n_pages;
  int page_rows;
  int32_t* tmp;  // [B][M + 1]: the new entries and length
};
struct CompactArgs {
  PagePool pool, to;
  PageShape s;
  PageTable t;
  const int32_t* refs;
  int32_t *new_table, *new_refs, *missing;
  int64_t n_to;
  int32_t *number, *live;  // workspace: [n_pages] new numbers; [n_to + 1] old ones, and how many
};

size_t reserve_bytes(const PageShape& s, const PageTable& t);
size_t fork_bytes(const PageTable& t);
size_t compact_bytes(const PageShape& s, int64_t n_to);
hipError_t launch_reserve(ReserveArgs a, void* ws, hipStream_t st);
hipError_t launch_append(const AppendArgs& a, hipStream_t st);
hipError_t launch_keep(const KeepArgs& a, hipStream_t st);
hipError_t launch_fork(ForkArgs a, void* ws, hipStream_t st);
hipError_t launch_release(const PageTable& t, int32_t* refs, const int32_t* lengths, int64_t n_pages, int page_rows, hipStream_t st);
hipError_t launch_compact(CompactArgs a, void* ws, hipStream_t st);
int64_t pages_parts(const PageShape& s, int64_t pages);  // pieces of work of a copy of so many pages

}  // namespace topk
