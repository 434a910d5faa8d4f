// The attention of one workgroup of few rows (kv_attention.hip; with shared prefixes
// kv_attention_shared.hip, over selected pages kv_attention_selected.hip).  Args says which
// rows and tokens a workgroup takes and where pages stand: find_tile(), group_pages()
// and part_tiles() of its type; Args::kParts: all results are partial ones.
#pragma once

#include "kv_attention_device.h"

namespace nvfp4 {

// Registers: the waves of a SIMD that a kernel of these forms is compiled for.
constexpr int rows_waves(int dim, int tiles, int waves, bool split) {
  return waves > 4 ? 2 : dim == 256 && split ? 1 : dim == 256 ? 3 - tiles : tiles > 1 ? 2 : 3;
}

// Keys and values of one tile of 32 tokens, as loaded: [group of 16][64
// elements of the head].
template <int D>
struct TileCodes {
  u32x4 k[2][D / 64], v[2][D / 64];
};

template <int D>
__device__ __forceinline__ void load_codes(const AttentionArgs& a, int kind, int h, int token, int page0, int page1,
                                           int lane, u32x4 (&to)[2][D / 64]) {
  const int mask = a.cache.page_size - 1;
  const int64_t head = (int64_t)h * a.cache.page_size * D;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int page = g ? page1 : page0, slot = (token + 16 * g) & mask;
    const uint8_t* from = a.cache.kv[kind] + (int64_t)max(page, 0) * a.cache.page_stride[kind] + head + slot * D;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) to[g][c] = *reinterpret_cast<const u32x4*>(from + c * 1024 + lane * 16);
  }
}

// The next tile's keys are loaded where this one's have been read, and so the values:
// one tile's registers, and a load's latency to cover either.  (Two tiles' registers,
// loaded a whole tile ahead: 60 sequences of 2000 tokens, 4 key heads of 64, 17.0 us;
// so 13.7.  Heads of 256 through a ring of two tiles in LDS: 40 of up to 2500, 3 key
// heads, 32 us; so 25.)
// Workgroups of eight waves, and those that take pieces of heads of 256, have a
// compute unit to themselves, though registers would let in two: those that short
// sequences leave empty make room for others then, and two long ones do not share a
// unit (16 sequences of up to 32768, 4 key heads of 256, in four pieces: 105 us, two
// to a unit 173; 32 of 3000, 8 key heads of 128, eight waves: 38 and 48 us).
template <int D, int kTiles, int kWaves>
struct RowsLds {
  static constexpr int kPart = kWaves > 4 ? 64 : (D > 128 ? 128 : D);      // elements of a row that are joined at a time
  float joined[kWaves][16][kPart + 4];
  float2 stats[kWaves][16 * kTiles];
};

// LDS that a kernel asks for and does not use, to have a compute unit to itself.
constexpr int alone_bytes(int dim, int tiles, int waves, bool split) {
  return waves > 4 || (dim == 256 && tiles == 1 && split) ? 65536 : 16;
}

// Key head h, piece `piece` (0, unless kSplit) of the tile with that number.
template <int D, int kTiles, int kWaves, bool kSplit, typename Args>
__device__ __forceinline__ void attention_rows(Args a, int h, int number, int piece, RowsLds<D, kTiles, kWaves>& lds) {
  constexpr int kRows = 16 * kTiles, kThreads = kWaves * 64, kPart = RowsLds<D, kTiles, kWaves>::kPart;
  auto& stats = lds.stats;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  Tile t;
  if (!find_tile<kRows>(a, number, t)) return;
  int begin = t.begin, end = t.end;
  bool whole = !Args::kParts;    // this piece is all that the rows see
  if (kSplit) {
    const int pieces = pieces_of(a, t);
    if (piece >= pieces) return;
    whole = whole && pieces == 1;
    piece_tokens(a, t, piece, begin, end);
  }

  RowTiles<D, kTiles> rows;
  rows.start(a, t, h, t.r0, t.n, lane, begin, end);
  const float scale = fabsf(a.scale);

  const int step = kWaves * kTileTokens;
  int token = (begin & ~(kTileTokens - 1)) + wave * kTileTokens;
  GroupPages pages = group_pages(a, t.b, h, (int64_t)token + (lane >> 1) * step + (lane & 1) * 16, begin, end);
  int in_batch = 0;
  // The tile's scales; then the next batch of pages, if the next tile needs it.
  const auto scales = [&](bool (&there)[2], float (&ks)[2], float (&vs)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      there[g] = __builtin_amdgcn_readlane(pages.page, 2 * in_batch + g) >= 0;
      ks[g] = fmaxf(lane_of(pages.k_scale, 2 * in_batch + g) * scale, 1e-37f);      // (not 0: -infinity stays)
      vs[g] = lane_of(pages.v_scale, 2 * in_batch + g);
    }
    if (++in_batch == 32) {
      pages = group_pages(a, t.b, h, (int64_t)token + step + (lane >> 1) * step + (lane & 1) * 16, begin, end);
      in_batch = 0;
      // (Waited for here, or the compiler would, and with them for the tile's values,
      // in front of every tile.)
      __builtin_amdgcn_s_waitcnt(wait_loads(0));
    }
  };
  bool there[2];
  float ks[2], vs[2];
  const auto load = [&](int kind, int at, u32x4(&to)[2][D / 64]) __attribute__((always_inline)) {
    load_codes<D>(a, kind, h, at, __builtin_amdgcn_readlane(pages.page, 2 * in_batch),
                  __builtin_amdgcn_readlane(pages.page, 2 * in_batch + 1), lane, to);
  };
  // (No branch around the loads, where the compiler would wait for whatever may be
  // outstanding on one of its paths: behind the end they read a page that is there.)
  TileCodes<D> now;
  load(0, token, now.k);
  load(1, token, now.v);
  while (token < end) {
    scales(there, ks, vs);
    rows.pass(
        a, token, there[0], there[1], ks, vs, lane, [&](int g, int c) { return now.k[g][c]; },
        [&](int g, int c) { return now.v[g][c]; }, [&]() __attribute__((always_inline)) { load(0, token + step, now.k); },
        [&]() __attribute__((always_inline)) { load(1, token + step, now.v); });
    token += step;
  }

  // The waves' results, joined: Y = sum_w 2^(m_w - m) Y_w.
  rows.finish();
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (quarter == 0) stats[wave][16 * i + col] = make_float2(rows.m[i], rows.l[i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    float m_all = kNone, l_all = 0.0f;
    for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, stats[w][16 * i + col].x);
    const float zero_m = m_all == kNone ? 0.0f : m_all;
    for (int w = 0; w < kWaves; ++w)
      l_all += stats[w][16 * i + col].y * __builtin_amdgcn_exp2f(stats[w][16 * i + col].x - zero_m);
    float mine = __builtin_amdgcn_exp2f(rows.m[i] - zero_m) * rows.s_ref;
    if (whole) mine *= l_all == 0.0f ? 0.0f : 1.0f / l_all;
    const int r = t.r0 + 16 * i + col;
    if (threadIdx.x < 16 && 16 * i + col < t.n) {
      if (!whole) {
        float2* to = reinterpret_cast<float2*>(a.part) + (((int64_t)number * a.cache.heads + h) * a.splits + piece) * kRows;
        to[16 * i + col] = make_float2(m_all, l_all);
      } else if (a.lse != nullptr) {
        a.lse[(int64_t)(t.row0 + r / a.group) * a.q_heads + h * a.group + r % a.group] =
            l_all == 0.0f ? kNone : (m_all + __builtin_amdgcn_logf(l_all)) * 0.69314718055994531f;
      }
    }
#pragma unroll
    for (int d0 = 0; d0 < D; d0 += kPart) {
      if (i > 0 || d0 > 0) __syncthreads();
#pragma unroll
      for (int j = 0; j < kPart / 16; ++j)
        *reinterpret_cast<f32x4*>(&lds.joined[wave][col][16 * j + 4 * quarter]) = rows.o[i][d0 / 16 + j] * mine;
      __syncthreads();
      // A thread takes four elements of one row.
      for (int x = threadIdx.x; x < 16 * kPart / 4; x += kThreads) {
        const int row = 16 * i + x / (kPart / 4), e = (x % (kPart / 4)) * 4;
        if (row >= t.n) continue;
        f32x4 y = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) y += *reinterpret_cast<const f32x4*>(&lds.joined[w][x / (kPart / 4)][e]);
        if (!whole) {
          const int64_t stats_floats = part_tiles(a, kRows) * a.cache.heads * a.splits * (2 * kRows);
          float* to = a.part + stats_floats +
                      ((((int64_t)number * a.cache.heads + h) * a.splits + piece) * kRows + row) * D + d0 + e;
          *reinterpret_cast<f32x4*>(to) = y;
        } else {
          const int rr = t.r0 + row;
          uint16_t* to = a.y + (int64_t)(t.row0 + rr / a.group) * a.ldy + (int64_t)(h * a.group + rr % a.group) * D + d0 + e;
          *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
        }
      }
    }
  }
}

// What a workgroup takes: heads side by side, then a tile's pieces.
template <bool kSplit>
__device__ __forceinline__ void work_of(const AttentionArgs& a, int& h, int& number, int& piece) {
  int id = blockIdx.x;
  h = id % a.cache.heads;
  id /= a.cache.heads;
  number = kSplit ? id / a.splits : id;
  piece = kSplit ? piece_of(id % a.splits, number, a.splits) : 0;
}

// A whole kernel of it.
template <int D, int kTiles, int kWaves, bool kSplit, typename Args>
__device__ __forceinline__ void attention_rows_kernel(Args a) {
  __shared__ struct {
    RowsLds<D, kTiles, kWaves> rows;
    char alone[alone_bytes(D, kTiles, kWaves, kSplit)];
  } lds;
  int h, number, piece;
  work_of<kSplit>(a, h, number, piece);
  attention_rows<D, kTiles, kWaves, kSplit>(a, h, number, piece, lds.rows);
}

// Joins the pieces of a sequence.  kShare waves take a packed row, each its
// share of the pieces, four pieces' loads in flight.
template <int D, int kTiles, int kShare, typename Args>
__device__ __forceinline__ void attention_join(Args a) {
  constexpr int kRows = 16 * kTiles, kEach = D / 64, kAhead = 4, kBlockRows = 4 / kShare;
  __shared__ float sums[kShare > 1 ? 4 : 1][kShare > 1 ? D : 1];
  __shared__ float totals[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, share = wave % kShare;
  const int row = (int)(blockIdx.x % (kRows / kBlockRows)) * kBlockRows + wave / kShare;
  const int h = (int)(blockIdx.x / (kRows / kBlockRows)) % a.cache.heads;
  const int number = (int)(blockIdx.x / (kRows / kBlockRows)) / a.cache.heads;
  Tile t;
  if (!find_tile<kRows>(a, number, t) || row >= t.n) return;      // (with kShare 4, the whole workgroup)
  const int pieces = pieces_of(a, t);
  if (pieces == 1) return;      // its rows are written already
  const int64_t first = ((int64_t)number * a.cache.heads + h) * a.splits;
  const float2* stats = reinterpret_cast<const float2*>(a.part) + first * kRows + row;
  const float* part = a.part + part_tiles(a, kRows) * a.cache.heads * a.splits * (2 * kRows) +
                      (first * kRows + row) * D + lane * kEach;
  float m = kNone, l = 0.0f, y[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) y[i] = 0.0f;
  for (int p = share; p < pieces; p += kShare * kAhead) {
    float2 st[kAhead];
    float v[kAhead][kEach];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int at = p + u * kShare;
      st[u] = make_float2(kNone, 0.0f);
#pragma unroll
      for (int i = 0; i < kEach; ++i) v[u][i] = 0.0f;
      if (at < pieces) {
        st[u] = stats[at * kRows];
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[u][i] = part[(int64_t)at * kRows * D + i];
      }
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) top = fmaxf(top, st[u].x);
    const float base = top == kNone ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - base);
    m = top;
    l *= f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) y[i] *= f;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const float g = __builtin_amdgcn_exp2f(st[u].x - base);
      l = fmaf(st[u].y, g, l);
#pragma unroll
      for (int i = 0; i < kEach; ++i) y[i] = fmaf(v[u][i], g, y[i]);
    }
  }
  const int r = t.r0 + row, head = h * a.group + r % a.group;
  const int64_t token_row = t.row0 + r / a.group;
  uint16_t* to = a.y + token_row * a.ldy + (int64_t)head * D;
  if (kShare > 1) {
    if (lane == 0) totals[wave] = m;
    __syncthreads();
    const float top = fmaxf(fmaxf(totals[0], totals[1]), fmaxf(totals[2], totals[3]));
    const float g = __builtin_amdgcn_exp2f(m - (top == kNone ? 0.0f : top));
    __syncthreads();
    if (lane == 0) totals[wave] = l * g;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sums[kShare > 1 ? wave : 0][kShare > 1 ? lane * kEach + i : 0] = y[i] * g;
    __syncthreads();
    m = top;
    l = (totals[0] + totals[1]) + (totals[2] + totals[3]);
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = kShare > 1 ? lane * kEach + i : 0;
      y[i] = (sums[0][e] + sums[kShare > 1 ? 1 : 0][e]) + (sums[kShare > 1 ? 2 : 0][e] + sums[kShare > 1 ? 3 : 0][e]);
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (D == 64)
    to[lane] = __builtin_bit_cast(uint16_t, (__bf16)(y[0] * inv));
  else
#pragma unroll
    for (int i = 0; i + 1 < kEach; i += 2)
      *reinterpret_cast<uint32_t*>(to + lane * kEach + i) = bf16_pair(y[i] * inv, y[i + 1] * inv);
  if (a.lse != nullptr && lane == 0)
    a.lse[token_row * a.q_heads + head] = l == 0.0f ? kNone : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

}  // namespace nvfp4
