// Attention of few rows over the paged E4M3 cache for gfx950 (layout and
// definition: nvfp4_attention.h; the products: kv_attention_device.h).
//
// A workgroup takes 16 or 32 packed rows of one sequence and key head; its
// waves take turns with tiles of 32 tokens, and join their results in LDS at
// the end.  Keys and values go from memory to registers.  Long sequences are
// divided further, into pieces for several workgroups, which a second launch joins.
//
// Bound by HBM where there are enough workgroups: 128 sequences of up to 8000
// tokens, 8 key heads of 128: 192 us, 5.3 TB/s; one of 131072: 53 us with its join,
// 5.05 TB/s.  Else by a wave's 250 instructions for a tile and its loads' latency.
#include "attention_plan.h"
#include "kv_attention_device.h"

namespace nvfp4 {

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
template <int D, int kTiles, int kWaves, bool kSplit>
__global__ __launch_bounds__(kWaves * 64, kWaves > 4                ? 2
                                                  : D == 256 && kSplit ? 1
                                                  : D == 256           ? 3 - kTiles
                                                                       : 4 - kTiles) void
kv_attention_rows_kernel(AttentionArgs a) {
  constexpr int kRows = 16 * kTiles, kThreads = kWaves * 64;
  constexpr int kPart = kWaves > 4 ? 64 : (D > 128 ? 128 : D);            // elements of a row that are joined at a time
  __shared__ struct {
    float joined[kWaves][16][kPart + 4];
    char alone[kWaves > 4 || (D == 256 && kTiles == 1 && kSplit) ? 65536 : 1];      // (so that they have)
  } lds;
  __shared__ float2 stats[kWaves][kRows];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  int id = blockIdx.x;
  const int h = id % a.cache.heads;
  id /= a.cache.heads;
  const int number = kSplit ? id / a.splits : id;
  const int piece = kSplit ? piece_of(id % a.splits, number, a.splits) : 0;
  Tile t;
  if (!find_tile<kRows>(a, number, t)) return;
  int begin = t.begin, end = t.end;
  bool whole = true;             // this piece is all that the rows see
  if (kSplit) {
    const int pieces = pieces_of(a, t);
    if (piece >= pieces) return;
    whole = pieces == 1;
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
          const int64_t stats_floats = tiles_of(a.batch, a.group, kRows) * a.cache.heads * a.splits * (2 * kRows);
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

// Joins the pieces of a sequence.  kShare waves take a packed row, each its
// share of the pieces, four pieces' loads in flight.
template <int D, int kTiles, int kShare>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a) {
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
  const float* part = a.part + tiles_of(a.batch, a.group, kRows) * a.cache.heads * a.splits * (2 * kRows) +
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

namespace {

template <int D, int kTiles>
hipError_t launch_join(const AttentionArgs& a, int64_t work, hipStream_t stream) {
  if (a.splits == 1) return hipSuccess;
  if (a.splits > 8)
    kv_attention_join_kernel<D, kTiles, 4><<<dim3((unsigned)(work * 16 * kTiles)), 256, 0, stream>>>(a);
  else
    kv_attention_join_kernel<D, kTiles, 1><<<dim3((unsigned)(work * 4 * kTiles)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <int D, int kTiles, int kWaves>
hipError_t launch_rows(const AttentionArgs& a, int64_t work, hipStream_t stream) {
  if constexpr (kWaves == 4) {      // (eight waves take one piece)
    if (a.splits > 1) {
      kv_attention_rows_kernel<D, kTiles, kWaves, true><<<dim3((unsigned)(work * a.splits)), kWaves * 64, 0, stream>>>(a);
      const hipError_t e = hipGetLastError();
      return e != hipSuccess ? e : launch_join<D, kTiles>(a, work, stream);
    }
  }
  kv_attention_rows_kernel<D, kTiles, kWaves, false><<<dim3((unsigned)work), kWaves * 64, 0, stream>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_attention(const AttentionArgs& a, hipStream_t stream) {
  const int64_t work = host_tiles(a.batch, a.group, 16 * a.row_tiles) * a.cache.heads;
  if (a.row_tiles == 8) {
    const hipError_t e = launch_kv_attention_tile(a, work / a.cache.heads, stream);
    return e != hipSuccess ? e : launch_join<D, 8>(a, work, stream);
  }
  if (a.row_tiles == 2) return launch_rows<D, 2, 4>(a, work, stream);
  if (a.waves == 8) return launch_rows<D, 1, 8>(a, work, stream);
  return launch_rows<D, 1, 4>(a, work, stream);
}

}  // namespace

hipError_t launch_kv_attention(const AttentionArgs& args, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  AttentionArgs a = args;
  const AttentionPlan p = {a.row_tiles, a.waves, a.chunk, a.splits};
  if (part_bytes(a.cache, a.batch, a.group, p) > workspace_bytes) return hipErrorInvalidValue;      // (by the plan, never)
  a.part = static_cast<float*>(workspace);
  return a.cache.dim == 64    ? launch_attention<64>(a, stream)
         : a.cache.dim == 128 ? launch_attention<128>(a, stream)
                              : launch_attention<256>(a, stream);
}

}  // namespace nvfp4
