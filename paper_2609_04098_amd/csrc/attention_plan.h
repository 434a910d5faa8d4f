// How a step is divided over workgroups, from what the host knows of it: the
// attention's rows of a workgroup, its waves and pieces of long sequences, the
// append's form.  Host code.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "attention_launch.h"

namespace nvfp4 {

// A launch has fewer than 2^32 work-items.
inline bool one_grid(int64_t workgroups, int threads) { return workgroups * threads < (int64_t)1 << 32; }

inline int64_t host_tiles(const KvBatchArgs& b, int group, int rows) {
  return b.cu_rows == nullptr ? (int64_t)b.seqs * ((group + rows - 1) / rows) : (int64_t)b.rows * group / rows + b.seqs;
}

constexpr int64_t kAnyRoom = (int64_t)1 << 62;

struct AttentionPlan {
  int tiles;               // of 16 rows, for a workgroup
  int waves;
  int chunk, splits;
};

// Row tiles: a workgroup takes 16 rows where an average sequence has no more.  It
// takes 128 where sequences have over 64 and there are enough rows to fill the
// compute units with such workgroups (heads of 256, whose smaller tiles have a compute
// unit's registers to themselves: few), more of them for long sequences,
// where a workgroup that is alone takes long; else 32.  Full tiles times key heads, and
// the times in tiles of 32 and of 128 rows: heads of 128, 400 of 1500 tokens 74 and 62
// us, 503 of 447 39 and 22 us, 375 of 3000 104 and 107 us, 192 of 967 29 and 31 us;
// heads of 256, 81 of 856 40 and 36 us, 31 of 8000 98 and 59 us, 62 of 1000 27 and 31.
// Pieces: the number of them for which an estimate of the time is least, of a
// step whose sequences all have the largest length and of one that has 0.55 times
// as many workgroups (lengths of all sizes), together.  (Its figures are those that
// fit measured times best; 8 sequences of 30000 tokens, a window of 3000, 4 key
// heads of 128: 18.0 us in one piece with eight waves, 12.4 us in six.)
// A window bounds what a tile sees, and a step's workspace is sized without it:
// with one, only numbers of pieces that fit `room` partial results are looked at.
inline AttentionPlan attention_plan(const KvCacheArgs& c, const KvBatchArgs& b, int group, int window, int64_t room) {
  AttentionPlan p;
  const int64_t seqs = b.seqs > 0 ? b.seqs : 1, rows = ((int64_t)b.rows * group + seqs - 1) / seqs;
  const auto of_rows = [&](int tile) { return (rows + tile - 1) / tile; };
  const double full = (double)b.rows * group * c.heads / 128.0;
  const double enough = c.dim == 256 ? (b.max_kv_len < 2000 ? 64.0 : 24.0) : (b.max_kv_len < 1600 ? 330.0 : 480.0);
  p.tiles = rows <= 16 ? 1 : rows > 64 && full >= enough ? 8 : 2;
  const int64_t each_seq = of_rows(16 * p.tiles), work = each_seq * seqs * c.heads;
  // Workgroups of four waves that the estimate counts on a compute unit at a time.
  const auto fit = [&](int s) {
    return p.tiles == 8   ? (c.dim == 256 ? 2 : c.dim == 128 ? 3 : 4)
                  : p.tiles == 2 ? (c.dim == 256 ? 1 : c.dim == 128 ? 2 : 3)
                                 : (c.dim == 256 ? (s == 1 ? 2 : 1) : c.dim == 128 ? 3 : 4);
  };
  // Tokens that a workgroup takes in a microsecond alone, and that all of them
  // take together (5.5 TB/s of memory; 0.9 PFLOP/s of products).
  const double alone = p.tiles == 8   ? 35.0 * 128 / c.dim
                       : p.tiles == 2 ? 160.0 * 128 / c.dim
                       : c.dim == 64  ? 180.0
                       : c.dim == 128 ? 150.0
                                      : 80.0;
  const double join = p.tiles != 1 ? 6.0 : c.dim == 256 ? 2.0 : 5.0;
  // Eight waves: their rate, and their later start where there are many.
  const double eight = c.dim == 256 ? 1.1 : 1.3, start = c.dim == 256 ? 8.0 : 2.5;
  // (The tiles of one sequence share its keys and values.)
  const double together = p.tiles == 8 ? 0.9e9 / (512.0 * c.dim)
                                       : 5.5e6 / (2.0 * c.dim) * (each_seq < 2.4 ? (double)each_seq : 2.4);
  // A piece's results, written and read (tiles of 128 rows: two thirds of it behind
  // the products).
  const double part = (double)(rows < 16 * p.tiles ? rows : 16 * p.tiles) * c.dim * 8.0 / (p.tiles == 8 ? 12e6 : 4e6);
  static const int candidates[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64, 96, 128};
  double best = 0.0;
  p.waves = 4;
  p.splits = 1;
  const int64_t reach = (int64_t)window + 16 * p.tiles + 64;
  const int length = window > 0 && reach < b.max_kv_len ? (int)reach : b.max_kv_len;
  p.chunk = length > 0 ? length : 1;
  for (const int s : candidates) {
    const int64_t each = ((int64_t)length + 128 * s - 1) / (128 * s) * 128;
    if (s > 1 && (each < 256 || s > room)) break;
    // (One piece: also with eight waves, of which a compute unit holds one workgroup.
    // 24 sequences of up to 6 rows of 4 key heads of 64, a window of 4096: 23.5 us
    // with four, 18.2 us with eight, 18.3 us with sixteen.  A ring of three tiles
    // ahead in LDS for four waves: 20.5 us.  They start later where there are many:
    // 30 sequences of 8 key heads of 128, 400 tokens: 8.0 us with four, 11.1 us with
    // eight; and have twice the loads in flight: 32 of 3000, 45.2 and 38.1 us.)
    for (const int waves : {4, 8}) {
      if (waves > 4 && (s > 1 || p.tiles != 1)) continue;
      const double slots = 256.0 * (waves > 4 ? 1 : fit(s));
      double time = 0.0;
      for (const double share : {1.0, 0.55}) {
        const double n = share * (double)(work * s), longest = (double)each / (waves > 4 ? eight * alone : alone);
        const double all = n * (double)each / together;
        const double work_time = all > longest ? all : longest;
        time += waves > 4 ? 0.75 * work_time + start * n / slots : work_time;
        if (n > slots)                                             // the last ones; beginnings and ends
          time += (p.tiles == 8 ? 0.25 : 0.5) * longest + 6.0 * 256.0 * n / (slots * slots);
        if (s > 1) time += 0.05 * all + join + n * part;                           // the join
      }
      if ((s == 1 && waves == 4) || time < best) {
        best = time;
        p.waves = waves;
        p.splits = s;
        p.chunk = each > 0 ? (int)each : 1;
      }
    }
  }
  if (p.splits > 1) p.splits = (length + p.chunk - 1) / p.chunk;
  return p;
}

// Whether the attention's launches, and the numbers of its workgroups, are in range.
inline bool attention_fits(const KvCacheArgs& c, const KvBatchArgs& b, int group, const AttentionPlan& p) {
  const int64_t work = host_tiles(b, group, 16 * p.tiles) * c.heads;
  const int64_t joins = p.splits == 1 ? 0 : work * p.tiles * (p.splits > 8 ? 16 : 4);
  return one_grid(work * p.splits, 64 * p.waves) && one_grid(joins, 256);
}

inline size_t part_bytes(const KvCacheArgs& c, const KvBatchArgs& b, int group, const AttentionPlan& p) {
  if (p.splits == 1) return 0;
  return (size_t)(host_tiles(b, group, 16 * p.tiles) * c.heads * p.splits * 16 * p.tiles) * (c.dim + 2) * sizeof(float);
}

// The append's form and workgroups.
struct AppendPlan {
  bool tokens;             // a token at a time (few rows)
  int each;                // many rows: heads of a workgroup
  int threads;
  int64_t workgroups;
};

inline AppendPlan append_plan(const KvCacheArgs& c, const KvBatchArgs& b) {
  const int64_t items = b.cu_rows == nullptr ? b.seqs : (b.rows >> c.page_shift) + 2 * (int64_t)b.seqs;
  AppendPlan p;
  p.tokens = b.cu_rows == nullptr || b.rows < 5 * (int64_t)b.seqs;
  p.each = 0;
  p.threads = 256;
  if (p.tokens) {
    p.workgroups = 2 * items * ((c.heads * c.dim + 511) / 512);
    return p;
  }
  // Heads of a workgroup: as many as leave one round of workgroups on 256 compute
  // units, four of 4096 elements each (pages that are written, about rows / page_size).
  const int elements = c.page_size * c.dim;
  const int64_t pages = (b.rows >> c.page_shift) + b.seqs;
  const int64_t fit = elements <= 4096 ? 1024 : 1024 * 4096 / elements;
  int64_t each = (pages * c.heads + fit - 1) / fit;
  if (each > c.heads) each = c.heads;
  const int64_t parts = (c.heads + each - 1) / each;
  p.each = (int)((c.heads + parts - 1) / parts);
  p.threads = elements <= 4096 ? 256 : elements / 16;
  p.workgroups = items * parts;
  return p;
}

}  // namespace nvfp4
