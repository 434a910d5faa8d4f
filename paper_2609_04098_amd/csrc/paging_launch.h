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
  float* part;
};

// The workgroups of both passes (kv_attention_shared.hip).
struct SharedWork {
  uint32_t own, prefix;        // workgroups
  uint32_t prefix_eighth;      // of the prefix's for each die
  int own_tiles, prefix_tiles;
};

// The two passes' plans and the bytes of their partial results; or that of the attention
// without sharing (attention_plan.h), if it is taken to be faster.
struct SharedPlan {
  bool apart;
  AttentionPlan whole, prefix, own;
  size_t prefix_bytes, bytes;
};

// Numbers of a group pass's tiles of `rows` packed rows, for n packed rows in all: group g's
// begin at first row * group / rows + g.
__host__ __device__ inline int64_t prefix_tile_numbers(int64_t n, int rows, int groups) {
  return groups == 1 ? (n + rows - 1) / rows : n / rows + groups;
}

inline int64_t prefix_tiles(const SharedArgs& a, int form) {
  return prefix_tile_numbers((int64_t)a.batch.rows * a.group, 16 * form, a.groups);
}

inline size_t all_part_bytes(const KvCacheArgs& c, int64_t tiles, const AttentionPlan& p) {
  return (size_t)(tiles * c.heads * p.splits * 16 * p.tiles) * (c.dim + 2) * sizeof(float);
}

// What a step takes, from 18 measured steps (times without and with sharing, in its best
// form, us; sequences x new rows, prefix, own tokens up to, query / key heads of dim):
//   4 x 1, 608, 90, 40 / 8 of 128       8.2  9.9     150 x 1, 512, 100, 40 / 8 of 128    21.1 25.8
//   100 x 1, 1024, 200, 64 / 8 of 64   17.9 21.6     8 x 1, 2048, 300, 32 / 8 of 128     14.0 11.1
//   60 x 1 (3 groups), 2000, 24 / 4    18.8 17.2     2 x 1, 30000, 500, 40 / 8 of 128    21.9 20.9
//   16 x 1, 8192, 200, 40 / 8          37.1 17.8     32 x 4, 4096, 500, 32 / 8           43.9 29.7
//   150 x 1, 4160, 777, 24 / 4 of 256  99.0 49.0     64 x 1, 32768, 1000, 40 / 8          377 76.0
//   64 x 8 (2 groups), 4000, 64 / 8    94.9  112
// Pages that sequences share are in the caches after the first one has read them, so what
// sharing saves is not memory's but the caches' reads; it costs partial results and a join.
// So it begins at prefixes of 1536 tokens, and not where a sequence's own rows fill 64.
// Rows of the prefix's workgroups: by the rows of a group,
//   320 of 128: 85 us with 16, 76 with 32, 79 with 128    512 (4096 tokens): 30.0 29.7 32.9
//   1024: 126 112 105     2048: 133 128 112     2048 of 64: 97 85 84
//   900 of 256: 49 (16), 54 (128)     512 of 256 (30000 tokens): 59 (16), 65 (128)
// Pieces: the number of them for which an estimate is least, in the time of a token for a
// workgroup that has its compute unit to itself (3.7 ns for 32 rows of 128): 1400 for its
// beginning and end; two of them on a unit take 1.5 times as long (1.8 with heads of 256), a
// few units with two or three, where there is not one for every half, twice; and a piece's partial
// results, written and read, at 4 TB/s, with a wave's eighth of a load's latency.  (20 users, 64 / 4 heads, a prefix of 30000: 49 us in six
// pieces, 43 in twelve, 48 in 24; two groups of 20 with 64 / 8 heads, 16000: 69 in two, 43 in
// six; 900 rows of 256: 49 in one of 4160, 56 in two; 32 x 4: 30 in two, 33 in four.)
// Tiles of 128 rows: three to a unit (1024 rows, 16000 tokens: 131 us in four, 92 in twelve).
inline AttentionPlan shared_pieces(int tokens, int64_t work, int64_t packed_rows, int dim, bool wide, int least) {
  AttentionPlan q = {};
  const auto chunk_of = [&](int64_t n) {
    const int c = (int)(((tokens + n - 1) / n + 127) / 128 * 128);
    return c < least ? least : c;
  };
  int64_t best = 1;
  if (wide) {
    best = work < 256 ? 256 / work : 1;
    if (tokens / best > 1000) best = work < 768 ? 768 / work : 1;
  } else {
    const double both = dim == 256 ? 1.8 : 1.5, part = 25.0 + (double)packed_rows * (dim + 2) * 8.0 / 4e6 / 3.7e-3;
    double least_time = 0.0;
    for (int64_t n = 1; n <= 128 && (n == 1 || tokens / n >= least); ++n) {
      const int64_t all = work * n;
      const double each = (double)chunk_of(n);
      const double time = (all <= 256 ? each + 1400.0 : all < 448 ? 2.0 * each + 1400.0
                                                                  : (double)((all + 511) / 512) * (both * each + 1400.0)) + n * part;
      if (n == 1 || time < least_time) least_time = time, best = n;
    }
  }
  q.chunk = chunk_of(best);
  q.splits = tokens > 0 ? (tokens + q.chunk - 1) / q.chunk : 1;
  q.waves = 4;
  return q;
}

inline SharedPlan shared_plan(const SharedArgs& a) {
  SharedPlan p = {};
  const int64_t rows = (int64_t)a.batch.rows * a.group;
  const int64_t of_seq = (rows + a.batch.seqs - 1) / a.batch.seqs, of_group = a.groups > 0 ? (rows + a.groups - 1) / a.groups : 0;
  p.apart = a.groups == 0 || a.max_prefix < 1536 || of_seq >= 64;
  if (p.apart) {
    p.whole = attention_plan(a.cache, a.batch, a.group, 0, kAnyRoom);
    p.bytes = part_bytes(a.cache, a.batch, a.group, p.whole);
    return p;
  }
  const int own_form = of_seq <= 16 ? 1 : a.cache.dim == 256 ? 8 : 2;
  int form = a.cache.dim == 256 || of_group < 256 ? 1 : of_group < 768 ? 2 : 8;
  if (form < own_form) form = own_form;
  const int64_t all_rows = rows * a.cache.heads;
  p.prefix = shared_pieces(a.max_prefix, prefix_tiles(a, form) * a.cache.heads, all_rows, a.cache.dim, form == 8, 128);
  p.prefix.tiles = form;
  p.prefix_bytes = all_part_bytes(a.cache, prefix_tiles(a, form), p.prefix);
  const int64_t own_tiles = host_tiles(a.batch, a.group, 16 * own_form);
  p.own = shared_pieces(a.max_own, own_tiles * a.cache.heads, all_rows, a.cache.dim, own_form == 8, 256);
  p.own.tiles = own_form;
  p.bytes = p.prefix_bytes + all_part_bytes(a.cache, own_tiles, p.own);
  return p;
}

inline SharedWork shared_work(const SharedArgs& a, const SharedPlan& p) {
  SharedWork w = {};
  w.own_tiles = (int)host_tiles(a.batch, a.group, 16 * p.own.tiles);
  w.own = (uint32_t)((int64_t)w.own_tiles * a.cache.heads * p.own.splits);
  w.prefix_tiles = (int)prefix_tiles(a, p.prefix.tiles);
  w.prefix = (uint32_t)((int64_t)w.prefix_tiles * a.cache.heads * p.prefix.splits);
  w.prefix_eighth = (w.prefix + 7) / 8;
  return w;
}

inline int64_t shared_workgroups(const SharedWork& w) { return (int64_t)w.own + 8 * (int64_t)w.prefix_eighth; }

// Whether every launch of a plan is in range.
inline bool shared_fits(const SharedArgs& a, const SharedPlan& p) {
  if (p.apart) return attention_fits(a.cache, a.batch, a.group, p.whole);
  const int64_t own = host_tiles(a.batch, a.group, 16 * p.own.tiles) * a.cache.heads;
  const int64_t prefix = prefix_tiles(a, p.prefix.tiles) * a.cache.heads;
  return one_grid(((int64_t)a.batch.rows * a.q_heads + 3) / 4, 256) && one_grid(own * p.own.splits + prefix * p.prefix.splits + 16, 256);
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
size_t kv_select_workspace_bytes(const SelectArgs& a);
bool select_fits(const SelectArgs& a);
hipError_t launch_kv_select(const SelectArgs& a, hipStream_t stream);
hipError_t launch_kv_attention_selected(const SelectedArgs& a, hipStream_t stream);      // (a.part: its workspace)

}  // namespace nvfp4
