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
// takes 128 where sequences have over 64 and the full tiles of 128 rows times key
// heads are enough, by the largest length; else 32.  Largest length, full
// tiles, and the times in tiles of 32 and of 128 rows (us); the last of each line has
// ragged lengths:
//   heads of 64     447 tokens, 260: 18.1 20.0   447, 400: 22.6 19.8   700, 260: 22.6 27.7
//                   700, 900: 47.4 40.5   3000, 600: 108 121   3000, 1000: 160 150
//                   16000, 512: 420 409 (one sequence 330 402)   40000, 512: 1028 963
//                   40000, 800: 1628 1809   40000, 900: 1864 1827   3000, 806: 83 99
//                   (beyond 10000 tokens neither form is the faster one throughout)
//   heads of 128    447, 130: 22.1 20.1   447, 260: 31.1 26.9   967, 260: 42.9 46.1
//                   967, 400: 56.9 46.7   1500, 260: 55.0 68.5   1500, 560: 93.8 83.8
//                   3000, 260: 91 105   3000, 650: 186 164   8000, 512: 347 391   1500, 346: 51 70
//   heads of 256    (32 rows have a compute unit to themselves: one round of 256 workgroups up
//                   to 64)  967, 50: 27.4 37.8   967, 66: 50.5 43.1   2500, 50: 45.9 64.6
//                   2500, 66: 87 64   4000, 66: 124 87   16000, 30: 159 97   16000, 46: 208 144
// Of 440 such steps (1 to 8 sequences, half of them ragged) the rule takes the faster
// form, or one within 5%, in 387, and one within 15% in 423; the worst are (128, 24000
// tokens, 130 full tiles) 374 us for 271 and (64, 40000, 556, ragged) 1270 for 939.
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
  const double enough = c.dim == 256   ? (b.max_kv_len < 3500 ? 65.0 : 24.0)
                        : c.dim == 128 ? (b.max_kv_len < 600 ? 150.0 : b.max_kv_len < 1600 ? 400.0 : 480.0)
                                       : (b.max_kv_len < 600 ? 330.0 : b.max_kv_len < 10000 ? 850.0 : 500.0);
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

// The append's form and workgroups.  Few rows: under 5 for a sequence, of which the
// host knows no more.  128 sequences of the same n rows, 8 heads of 128, a token at a
// time and in whole pages (us), pages of 16, 32, 64 and 128:
//   n = 1    8.1  9.3     8.0  9.1     7.9 12.4     8.1 24.9
//   n = 4    8.1  9.1     8.1  9.8     8.0 12.1    11.5 15.4
//   n = 8    8.7 13.2    10.2 10.7    11.1 20.1    11.0 17.9
//   n = 16  15.9 14.8    16.8 12.0    16.8 15.0    18.9 19.5
// but a prompt among single tokens, whose pages are a workgroup's of four waves each,
//   100 x 1 + 500 (5.9 on average)  11.3 11.0   18.5 12.3   33.1 19.5   63.7 38.3
//   30 x 1 + 100 (4.2)              10.5  8.2   17.9  8.2   32.6  9.1   40.3 15.4
// so that 5 gives up the former from 5 to 8 rows, and the latter below 5.
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
