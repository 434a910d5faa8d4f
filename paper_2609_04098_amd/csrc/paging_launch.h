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
  int join_share;              // waves that join a row's query head
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
//   60 x 1 (3 groups), 2000, 24 / 4    18.8 17.2     2 x 1, 30000, 500, 40 / 8 of 128    22.6 19.5
//   16 x 1, 8192, 200, 40 / 8          37.1 17.8     32 x 4, 4096, 500, 32 / 8           43.9 29.7
//   150 x 1, 4160, 777, 24 / 4 of 256  99.0 49.0     64 x 1, 32768, 1000, 40 / 8          377 76.4
//   64 x 8 (2 groups), 4000, 64 / 8    94.9  112
// Pages that sequences share are in the caches after the first one has read them, so what
// sharing saves is not memory's but the caches' reads; it costs partial results and a join.
// So it begins at prefixes of 1536 tokens, and not where an average sequence's own rows fill 64.
// (The average is all that the host has, and a bad one for a prompt among single tokens: 64 x 1 behind 32768,
// 40 / 8 heads of 128, take 80 us alone, 110 beside a prompt of 256 rows, 289 of 512, and 513 of 1024, where
// nothing is shared any more; without sharing 378, 513, 394, 513.)
// Rows of a prefix's workgroups, and pieces of either pass: those for which an estimate is
// least, of what hangs on them.  m workgroups of a compute unit side by side take
// `alone` + m `each` for a token of their piece and `start` for their beginning and end; those
// that a unit has no room for come behind them; and partial results are written and read at
// 2.6 TB/s.  Fitted to 210 measured steps (1 to 4 groups of 36 to 900 rows, prefixes of 2000 to
// 32000 tokens, 1 to 8 key heads, each in 1 to 48 pieces): what it takes is slower than
// the fastest of them by 3% (heads of 64), 4% (128) and 2% (256) on the average, timed anew by 6, 7 and 5%.
//   us of the fastest with 16, 32, 48 and 128 rows; groups x rows, prefix, key heads of 128:
//   1 x 160, 2000, 2    11.8  14.3  16.3        1 x 320, 32768, 8   78.5  77.7  72.4  92.3
//   4 x 256, 32000, 4    116   112   103   120  1 x 696, 32000, 8    158   140   125   136
//   2 x 320, 4000, 4    24.9  25.2  25.7  31.1  4 x 510, 8000, 8     183   173   159   141
//   of 64: 2 x 696, 32000, 4   94.7  80.7  77.1  98.3     2 x 512, 8000, 4   35.2  31.9  32.6  36.7
// (48 rows of 128 fill the registers that two waves of a SIMD have; of 64 they gain nothing
// on 32, and 32 of 128 less than 2% on the better of 16 and 48.  128 rows, through LDS, gain 2 to 12%
// only at a thousand rows and more.  Heads of 256, 900 rows: 49 with 16, 54 with 128, 69 with 32.)
struct Pace {
  double alone, each, start;            // us
  int slots;                            // workgroups that a unit has room for
};

inline Pace pace_of(int dim, int form) {
  if (dim == 64) return form == 1 ? Pace{1.3e-3, 1.8e-3, 0.3, 4} : Pace{2.1e-3, 2.5e-3, 0.5, 4};
  if (dim == 256) return {1.5e-3, 3.5e-3, 0.0, 2};
  return form == 1 ? Pace{1.8e-3, 1.3e-3, 0.3, 4} : form == 2 ? Pace{2.8e-3, 1.4e-3, 0.6, 2} : Pace{4.0e-3, 1.45e-3, 1.0, 2};
}

// The pieces of `tokens` for `work` tiles of a form (16 rows times it), at least `least` tokens
// each, and the estimate.  Tiles of 128 rows: three to a unit.
inline AttentionPlan shared_pieces(int tokens, int64_t work, int64_t packed_rows, int dim, int form, int least, double* time) {
  AttentionPlan q = {};
  const auto chunk_of = [&](int n) {
    const int c = (tokens / n + (tokens % n != 0) + 127) / 128 * 128;
    return c < least ? least : c;
  };
  int best = 1;
  if (form == 8) {
    if (work < 256) best = (int)(256 / work);
    if (tokens / best > 1000) best = work < 768 ? (int)(768 / work) : 1;
  } else {
    const Pace p = pace_of(dim, form);
    const double part = (double)packed_rows * (dim + 2) * 8.0 / 2.6e6;
    for (int n = 1; n <= 128 && (n == 1 || (tokens / n >= least && work * n <= 12 * 256)); ++n) {
      const double chunk = chunk_of(n);
      const int64_t m = (work * n + 255) / 256, full = m / p.slots, rest = m % p.slots;
      const auto side_by_side = [&](int64_t w) { return chunk * (p.alone + w * p.each) + p.start; };
      const double t = full * side_by_side(p.slots) + (rest > 0 ? side_by_side(rest) : 0.0) + n * part;
      if (n == 1 || t < *time) *time = t, best = n;
    }
  }
  q.tiles = form;
  q.chunk = chunk_of(best);
  q.splits = tokens > 0 ? (tokens + q.chunk - 1) / q.chunk : 1;
  q.waves = 4;
  return q;
}

inline SharedPlan shared_plan(const SharedArgs& a) {
  SharedPlan p = {};
  const int64_t rows = (int64_t)a.batch.rows * a.group;
  const int64_t of_seq = (rows + a.batch.seqs - 1) / a.batch.seqs;
  p.apart = a.groups == 0 || a.max_prefix < 1536 || of_seq >= 64;
  if (p.apart) {
    p.whole = attention_plan(a.cache, a.batch, a.group, 0, kAnyRoom);
    p.bytes = part_bytes(a.cache, a.batch, a.group, p.whole);
    return p;
  }
  const int dim = a.cache.dim, own_form = of_seq <= 16 ? 1 : dim == 256 ? 8 : 2;
  const int64_t all_rows = rows * a.cache.heads, of_group = (rows + a.groups - 1) / a.groups;
  double time = 0.0;
  const auto prefix = [&](int form, double* t) {      // (as if the groups were of one size)
    return shared_pieces(a.max_prefix, a.groups * ((of_group + 16 * form - 1) / (16 * form)) * a.cache.heads, all_rows, dim, form, 128, t);
  };
  const int more = dim == 64 ? 2 : dim == 128 ? 3 : 8;      // the form of more rows
  if (own_form > 1) {
    p.prefix = prefix(more, &time);
  } else {
    p.prefix = prefix(1, &time);
    double other = 0.0;
    const AttentionPlan q = dim < 256 ? prefix(more, &other) : p.prefix;
    if (dim < 256 && other < time) p.prefix = q;
  }
  p.prefix_bytes = all_part_bytes(a.cache, prefix_tiles(a, p.prefix.tiles), p.prefix);
  const int64_t own_tiles = host_tiles(a.batch, a.group, 16 * own_form);
  p.own = shared_pieces(a.max_own, own_tiles * a.cache.heads, all_rows, dim, own_form, 256, &time);
  p.bytes = p.prefix_bytes + all_part_bytes(a.cache, own_tiles, p.own);
  // Few rows of many pieces by four waves (by one and by four, us; rows x query heads, pieces of the prefix:
  // 16, 128 31.1 19.9;  80, 32 21.6 19.0;  640, 24 34.5 33.5;  720, 5 29.7 35.6;  2048, 6 29.5 32.8).
  p.join_share = (int64_t)a.batch.rows * a.q_heads <= 1024 && p.prefix.splits + p.own.splits > 8 ? 4 : 1;
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
