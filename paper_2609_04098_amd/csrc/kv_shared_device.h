// Sequences that share prefixes: the rows and tokens of the attention's two passes
// (kv_attention_shared.hip), over a group's prefix with the rows of all its sequences,
// and over each sequence's own tokens.
//
// A sequence shares where its rows all lie behind the prefix; any other takes all of
// its tokens for its own, and its part of the first pass is not looked at.  A prefix's
// pages are those of the group's first sequence that shares.
#pragma once

#include "kv_attention_device.h"
#include "paging_launch.h"

namespace nvfp4 {

struct PrefixArgs : SharedArgs {
  static constexpr bool kParts = true;
};

struct OwnArgs : SharedArgs {
  static constexpr bool kParts = true;
};

__device__ __forceinline__ int group_start(const SharedArgs& a, int g) { return min(max(a.cu_seqs[g], 0), a.batch.seqs); }

// The first row of sequence s (of the last one's end: s = seqs).
__device__ __forceinline__ int start_row(const KvBatchArgs& b, int s) { return b.cu_rows == nullptr ? s : row_bound(b, s); }

__device__ __forceinline__ int prefix_tokens(const SharedArgs& a, int g) {
  return min(max(a.prefix[g], 0), a.batch.max_tokens);
}

// The group of sequence b, whose rows begin at token `first`, its first sequence, and the
// prefix that b shares (0: none).  All lanes of a wave call it with the same arguments.
__device__ __forceinline__ int shared_prefix(const SharedArgs& a, int b, int first, int& g, int& group_seq) {
  g = group_seq = 0;
  if (a.groups == 0) return 0;
  if (a.groups < 64) {      // all there is to know of them in one load's latency
    const int lane = threadIdx.x & 63;
    const int start = group_start(a, min(lane, a.groups)), tokens = prefix_tokens(a, min(lane, a.groups - 1));
    const unsigned long long hit = __ballot(lane < a.groups && start <= b);
    if (hit == 0) return 0;
    g = 63 - __builtin_clzll(hit);
    if (b >= __builtin_amdgcn_readlane(start, g + 1)) return 0;
    group_seq = __builtin_amdgcn_readlane(start, g);
    const int p = __builtin_amdgcn_readlane(tokens, g);
    return first >= p ? p : 0;
  }
  group_seq = last_at_most(a.groups, b, g, [&](int x) { return group_start(a, x); });
  if (b < group_seq || b >= group_start(a, g + 1)) return 0;
  const int p = prefix_tokens(a, g);
  return first >= p ? p : 0;
}

// The number of the first of group g's tiles of kRows packed rows.
template <int kRows>
__device__ __forceinline__ int first_prefix_tile(const SharedArgs& a, int row, int g) {
  return (int)((uint32_t)row * (uint32_t)a.group / kRows) + g;      // (below 2^31 packed rows)
}

// A tile of a group's rows over its prefix.
template <int kRows>
__device__ __forceinline__ bool find_tile(const PrefixArgs& a, int number, Tile& t) {
  const int lane = threadIdx.x & 63;
  int g, s0, s1, row0, row1;
  if (a.groups < 64) {
    const int s = group_start(a, min(lane, a.groups)), row = start_row(a.batch, s);
    const unsigned long long hit = __ballot(lane < a.groups && first_prefix_tile<kRows>(a, row, lane) <= number);
    if (hit == 0) return false;
    g = 63 - __builtin_clzll(hit);
    s0 = __builtin_amdgcn_readlane(s, g), s1 = __builtin_amdgcn_readlane(s, g + 1);
    row0 = __builtin_amdgcn_readlane(row, g), row1 = __builtin_amdgcn_readlane(row, g + 1);
  } else {
    last_at_most(a.groups, number, g, [&](int x) {
      return first_prefix_tile<kRows>(a, start_row(a.batch, group_start(a, x)), x);
    });
    s0 = group_start(a, g), s1 = group_start(a, g + 1);
    row0 = start_row(a.batch, s0), row1 = start_row(a.batch, s1);
  }
  const int ordinal = number - first_prefix_tile<kRows>(a, row0, g), prefix = prefix_tokens(a, g);
  t.row0 = row0;
  t.rows = row1 - row0;
  t.first = 0;
  if (prefix == 0 || ordinal < 0 || (int64_t)ordinal * kRows >= (int64_t)t.rows * a.group) return false;
  t.r0 = ordinal * kRows;
  t.n = min(kRows, t.rows * a.group - t.r0);
  t.begin = 0;
  t.end = prefix;
  for (int s = s0; s < s1; s += 64) {
    const int at = min(s + lane, s1 - 1);
    const SeqRows r = seq_rows(a.batch, a.batch.cu_rows == nullptr ? at : a.batch.cu_rows[at],
                               a.batch.cu_rows == nullptr ? at + 1 : a.batch.cu_rows[at + 1], a.batch.kv_len[at]);
    const unsigned long long hit = __ballot(s + lane < s1 && r.first >= prefix);
    if (hit != 0) {
      t.b = s + __builtin_ctzll(hit);
      return true;
    }
  }
  return false;
}

__device__ __forceinline__ int64_t part_tiles(const PrefixArgs& a, int rows) {
  return prefix_tile_numbers((int64_t)a.batch.rows * a.group, rows, a.groups);
}

// A tile of a sequence's rows over its own tokens.
template <int kRows>
__device__ __forceinline__ bool find_tile(const OwnArgs& a, int number, Tile& t) {
  if (!find_tile<kRows>(static_cast<const AttentionArgs&>(a), number, t)) return false;
  int g, group_seq;
  t.begin = min(shared_prefix(a, t.b, t.first, g, group_seq), max(0, t.end));
  return true;
}

}  // namespace nvfp4
