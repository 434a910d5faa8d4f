// Launchers of the kernels behind nvfp4_paging.h (called by paging_api.cpp after
// argument validation) and the parameters they pass by value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention_plan.h"

namespace nvfp4 {

struct TablesArgs {
  int32_t* table;
  int32_t* kv_len;
  int32_t* free_pages;
  int32_t* free_count;
  const int32_t* new_rows;
  const int32_t* drop;         // may be null, and so
  const int32_t* kept;
  int32_t* cu_rows;
  int32_t* positions;          // these two
  int64_t* slots;
  int64_t table_stride;
  int max_pages, seqs, num_pages, page_shift, rows;
  int32_t* plan;               // workspace: step_tables.hip
};

// Attention with shared prefixes: AttentionArgs of the pass over own tokens, and the groups.
struct SharedArgs : AttentionArgs {
  const int32_t* cu_seqs;
  const int32_t* prefix;
  int groups, max_prefix, max_own;
};

// How the pass over the prefixes left its results.
struct PrefixPieces {
  int tiles, chunk, splits;
  const float* part;
};

// The two passes' plans (attention_plan.h) and the bytes of their partial results.
struct SharedPlan {
  AttentionPlan prefix, own;
  size_t prefix_bytes, bytes;
};

// The groups, as the sequences of a step.
inline KvBatchArgs prefix_batch(const SharedArgs& a) {
  KvBatchArgs b = a.batch;
  b.cu_rows = a.cu_seqs;
  b.seqs = a.groups;
  b.max_kv_len = a.max_prefix;
  return b;
}

inline size_t all_part_bytes(const KvCacheArgs& c, const KvBatchArgs& b, int group, const AttentionPlan& p) {
  return (size_t)(host_tiles(b, group, 16 * p.tiles) * c.heads * p.splits * 16 * p.tiles) * (c.dim + 2) * sizeof(float);
}

inline SharedPlan shared_plan(const SharedArgs& a) {
  SharedPlan p = {};
  if (a.groups > 0) {
    const KvBatchArgs groups = prefix_batch(a);
    p.prefix = attention_plan(a.cache, groups, a.group, 0, kAnyRoom);
    p.prefix_bytes = all_part_bytes(a.cache, groups, a.group, p.prefix);
  }
  KvBatchArgs own = a.batch;
  own.max_kv_len = a.max_own;
  p.own = attention_plan(a.cache, own, a.group, 0, kAnyRoom);
  p.bytes = p.prefix_bytes + all_part_bytes(a.cache, own, a.group, p.own);
  return p;
}

// Whether every launch of a plan is in range.
inline bool shared_fits(const SharedArgs& a, const SharedPlan& p) {
  const int64_t own = host_tiles(a.batch, a.group, 16 * p.own.tiles) * a.cache.heads;
  if (!one_grid(own * p.own.splits, 64 * p.own.waves) || !one_grid(own * p.own.tiles * 4, 256)) return false;
  return a.groups == 0 ||
         one_grid(host_tiles(prefix_batch(a), a.group, 16 * p.prefix.tiles) * a.cache.heads * p.prefix.splits, 256);
}

// Bounds of pages' keys.
struct PageBoundsArgs {
  int8_t* codes;               // [page][head][largest, smallest][dim]
  float* step;
  int64_t page_stride, step_stride;
};

struct BoundsArgs {
  KvCacheArgs cache;
  KvBatchArgs batch;
  PageBoundsArgs bounds;
};

struct SelectArgs {
  KvCacheArgs cache;
  KvBatchArgs batch;
  PageBoundsArgs bounds;
  const uint16_t* q;
  int64_t ldq;
  int group, count, first, recent, causal, max_pages;
  int32_t* index;              // [row][head][count], and
  int32_t* pages;              // the pages themselves
  int32_t* tokens;             // [row]: of the pages taken; -1: a row behind the last sequence
  uint32_t* scores;            // workspace
};

// Attention over chosen pages: the batch's sequences are its rows, kv_len their tokens.
struct SelectedArgs : AttentionArgs {
  const int32_t* pages;
  int count;
};

size_t step_tables_workspace_bytes(int64_t seqs);
hipError_t launch_step_tables(const TablesArgs& a, hipStream_t stream);
hipError_t launch_kv_attention_shared(const SharedArgs& a, const SharedPlan& p, hipStream_t stream);      // (a.part: its workspace)
bool bounds_fit(const BoundsArgs& a);      // (each launch in range)
hipError_t launch_kv_page_bounds(const BoundsArgs& a, hipStream_t stream);
size_t kv_select_workspace_bytes(int64_t rows, int64_t heads, int64_t max_pages);
bool select_fits(const SelectArgs& a);
hipError_t launch_kv_select(const SelectArgs& a, hipStream_t stream);
hipError_t launch_kv_attention_selected(const SelectedArgs& a, hipStream_t stream);      // (a.part: its workspace)

}  // namespace nvfp4
