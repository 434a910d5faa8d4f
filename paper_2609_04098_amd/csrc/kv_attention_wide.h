// The attention of one workgroup of 128 rows (kv_attention_tile.hip, whose comment
// says how; with shared prefixes kv_attention_shared.hip).  Args: as in kv_attention_rows.h.
#pragma once

#include "kv_attention_device.h"

namespace nvfp4 {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTileRows = 128;
constexpr int kStageTokens = 64;
constexpr int kOneOfRoom = 0x3F800000 + (7 << 23);      // the bits of kValueRoom

// Maximum and sum over lanes lane % 32 and lane % 32 + 32.
__device__ __forceinline__ float over_halves_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

__device__ __forceinline__ float over_halves_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// The 32 rows of one wave.
template <int D>
struct WideRows {
  static constexpr int kSteps = D / 16;       // of the first product
  bf16x8 q[kSteps];
  f32x16 o[D / 32];
  float m, l;
  int first, r0, rows;           // token of the first new row; first packed row, packed rows
  int begin, end, all0, all1;
  float s_ref;

  __device__ __forceinline__ void start(const AttentionArgs& a, const Tile& t, int h, int row, int n, int lane,
                                        int from, int to) {
    first = t.first;
    r0 = row;
    rows = n;
    const int r = r0 + min(lane & 31, n - 1);
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;      // the scale's sign goes into Q
    // Steps 2 x and 2 x + 1: the halves of piece 2 x + lane / 32 of 16 elements.
    const uint16_t* src = a.q + (int64_t)(t.row0 + r / a.group) * a.ldq + (int64_t)(h * a.group + r % a.group) * D +
                          (lane >> 5) * 16;
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(src + (x / 2) * 32 + (x & 1) * 8);
      q[x] = __builtin_bit_cast(bf16x8, w ^ flip);
    }
    m = kNone;
    l = 0.0f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) o[j] = (f32x16)(0.0f);
    begin = from;
    end = to;
    const int low = t.first + r0 / a.group, high = t.first + (r0 + n - 1) / a.group;
    all1 = a.causal ? min(end, low + 1) : end;
    all0 = a.window > 0 ? max(begin, window_begin(high, a.window)) : begin;
    s_ref = kSmallest;
  }

  // Tokens token .. token + 31, whose keys and values are the two groups at
  // keys and values (16 D bytes each, in the cache's order); f: factors of the
  // scores, vs: value scales; there: both pages are in the cache.
  __device__ __forceinline__ void pass(const AttentionArgs& a, int token, bool there0, bool there1, float f0, float f1,
                                       float vs0, float vs1, int lane, const uint8_t* keys, const uint8_t* values) {
    const int half = lane >> 5;
    f32x16 s = (f32x16)(0.0f);
    // Key lane % 32, piece 2 x + half of 16 elements.
    const uint8_t* mine = keys + ((lane >> 4) & 1) * 16 * D + (lane & 15) * 16 + half * 256;
#pragma unroll
    for (int x = 0; x < kSteps / 2; ++x) {
      const u32x4 k = *reinterpret_cast<const u32x4*>(mine + x * 512);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16_of(k[0], k[1]), q[2 * x], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16_of(k[2], k[3]), q[2 * x + 1], s, 0, 0, 0);
    }
    // Element 64 c + 16 (2 (lane / 16 % 2) + n) + lane % 16, tokens 4 half .. + 3 and 8 + 4 half .. + 3.
    const uint8_t* own = values + (half * 16 + (lane & 15)) * 16 + ((lane >> 4) & 1) * 8;
    const bool whole = token >= all0 && token + kTileTokens <= all1 && there0 && there1;
    const uint32_t v0 = __float_as_uint(vs0), v1 = __float_as_uint(vs1), ref = __float_as_uint(s_ref);
    f16x8 p[2];
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float w = __builtin_amdgcn_exp2f(fmaf(s[r], r < 8 ? f0 : f1, -m));
      sum += w;
      p[r / 8][r % 8] = (_Float16)w;
    }
    float power0 = __uint_as_float(max((int)(v0 - ref) + kOneOfRoom, 0));
    float power1 = __uint_as_float(max((int)(v1 - ref) + kOneOfRoom, 0));
    // Where all rows see all tokens and the value scales are powers of two, at
    // most the largest met, the scores need no maximum: as long as their
    // exponentials' sum fits binary16, so does each.
    // (Before a row's first token m is -infinity, and the sum does not.)
    const bool plain = whole && max(v0, v1) <= ref && ((v0 | v1 | ref) & 0x7FFFFFu) == 0;
    if (!plain || __any(!(sum <= 65504.0f))) {
      if (!whole) {
        const int at = first + (r0 + min(lane & 31, rows - 1)) / a.group;
        const int see1 = a.causal ? min(end, at + 1) : end;
        const int see0 = a.window > 0 ? max(begin, window_begin(at, a.window)) : begin;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = token + 8 * (r / 4) + 4 * half + r % 4;
          if (j < see0 || j >= see1 || !(r < 8 ? there0 : there1)) s[r] = kNone;
        }
      }
      float t0 = s[0], t1 = s[8];
#pragma unroll
      for (int r = 1; r < 8; ++r) t0 = fmaxf(t0, s[r]), t1 = fmaxf(t1, s[8 + r]);
      const float m_new = fmaxf(m, reference(over_halves_max(fmaxf(t0 * f0, t1 * f1))));
      const float f = m == m_new ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);      // (0 from nothing)
      l *= f;
      m = m_new;
      const float s_new = fmaxf(fmaxf(vs0, vs1), s_ref), less = f * (s_ref / s_new);
#pragma unroll
      for (int j = 0; j < D / 32; ++j) o[j] *= less;
      s_ref = s_new;
      const float s_inv = kValueRoom / s_new, base = m == kNone ? 0.0f : m;
      const uint32_t r0 = __float_as_uint(vs0 * s_inv), r1 = __float_as_uint(vs1 * s_inv);
      sum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[r], r < 8 ? f0 : f1, -base));
        sum += w;
        p[r / 8][r % 8] = (_Float16)(w * __uint_as_float(((r < 8 ? r0 : r1) & 0x7FFFFFu) | 0x3F800000u));
      }
      power0 = __uint_as_float(r0 & 0x7F800000u);
      power1 = __uint_as_float(r1 & 0x7F800000u);
    }
    l += sum;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float power = g ? power1 : power0;
      constexpr int kBatch = D == 256 ? 1 : D / 64;      // (registers)
#pragma unroll
      for (int c0 = 0; c0 < D / 64; c0 += kBatch) {
        u32x2 v[kBatch][2];
#pragma unroll
        for (int c = 0; c < kBatch; ++c)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            v[c][x] = *reinterpret_cast<const u32x2*>(own + g * 16 * D + (c0 + c) * 1024 + x * 512);
        if (!whole) {
#pragma unroll
          for (int c = 0; c < kBatch; ++c)
#pragma unroll
            for (int x = 0; x < 2; ++x) v[c][x] = (u32x2){without_nan(v[c][x][0]), without_nan(v[c][x][1])};
        }
#pragma unroll
        for (int c = 0; c < kBatch; ++c)
#pragma unroll
          for (int n = 0; n < 2; ++n)
            o[2 * (c0 + c) + n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f16_of(v[c][0][n], v[c][1][n], power, power), p[g],
                                                                       o[2 * (c0 + c) + n], 0, 0, 0);
      }
    }
  }
};

template <int D>
struct alignas(16) TileLds {
  uint8_t stage[2][2][kStageTokens / 16][16 * D];      // [buffer][keys, values]
};

// Key head h, piece `piece` (0, unless kSplit) of the tile with that number, of `tiles`.
template <int D, bool kSplit, typename Args>
__device__ __forceinline__ void attention_tile(Args a, int tiles, int h, int number, int piece, TileLds<D>& lds) {
  constexpr int kGroups = kStageTokens / 16;
  auto& stage = lds.stage;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Tile t;
  if (!find_tile<kTileRows>(a, number, t)) return;
  int begin = t.begin, end = t.end;
  bool whole = !Args::kParts;    // this piece is all that the rows see
  if (kSplit) {
    const int pieces = pieces_of(a, t);
    if (piece >= pieces) return;
    whole = whole && pieces == 1;
    piece_tokens(a, t, piece, begin, end);
  }

  const int first = 32 * wave, n = min(32, t.n - first);      // this wave's rows (none: it only loads)
  const int r0 = t.r0 + min(first, t.n - 1);
  WideRows<D> rows;
  rows.start(a, t, h, r0, max(n, 1), lane, begin, end);
  // Tokens that one of this wave's rows sees.
  const int low = t.first + r0 / a.group, high = t.first + (r0 + max(n, 1) - 1) / a.group;
  const int mine1 = n <= 0 ? 0 : (a.causal ? min(end, high + 1) : end);
  const int mine0 = a.window > 0 ? max(begin, window_begin(low, a.window)) : begin;

  const float scale = fabsf(a.scale);
  int token = begin & ~(kStageTokens - 1), in_batch = 0, buffer = 0;
  // 16 tiles' pages; their key scales times the softmax scale (not 0, so that a
  // masked score, -infinity, stays one).
  const auto look_up = [&](int from) __attribute__((always_inline)) {
    GroupPages g = group_pages(a, t.b, h, (int64_t)from + 16 * lane, begin, end);
    g.k_scale = fmaxf(g.k_scale * scale, 1e-37f);
    return g;
  };
  GroupPages pages = look_up(token), more = pages;
  const int mask = a.cache.page_size - 1;
  // Wave w stages group w.
  const auto issue = [&](int at, int group, int to) __attribute__((always_inline)) {
    const int page = __builtin_amdgcn_readlane(more.page, group + wave);
    stage_group<D>(a.cache, 0, page, (at + 16 * wave) & mask, h, lane, stage[to][0][wave]);
    stage_group<D>(a.cache, 1, page, (at + 16 * wave) & mask, h, lane, stage[to][1][wave]);
  };
  if (token < end) issue(token, 0, 0);
  while (token < end) {
    const int ahead = token + kStageTokens, next = (in_batch + 1) % (64 / kGroups);
    if (next == 0) more = look_up(ahead);
    // This wave's loads of the tile have landed and its reads of the other
    // buffer are done; after the barrier, everybody's.
    __builtin_amdgcn_s_waitcnt(wait_loads(0) & kWaitLds);
    __builtin_amdgcn_s_barrier();
    if (ahead < end) issue(ahead, kGroups * next, buffer ^ 1);
#pragma unroll 1
    for (int half = 0; half < kGroups / 2; ++half) {
      const int at = token + 32 * half, g = kGroups * in_batch + 2 * half;
      if (at >= mine1 || at + 32 <= mine0) continue;
      rows.pass(a, at, __builtin_amdgcn_readlane(pages.page, g) >= 0, __builtin_amdgcn_readlane(pages.page, g + 1) >= 0,
                lane_of(pages.k_scale, g), lane_of(pages.k_scale, g + 1), lane_of(pages.v_scale, g),
                lane_of(pages.v_scale, g + 1), lane, stage[buffer][0][2 * half], stage[buffer][1][2 * half]);
    }
    if (next == 0) pages = more;
    in_batch = next;
    buffer ^= 1;
    token = ahead;
  }

  // This lane's elements of its row: 64 c + 32 x + 16 n + 8 y + 4 half + 0 .. 3 in o[2 c + n][8 x + 4 y + 0 .. 3].
  // (The lane's number again, so that nothing made of it is kept through the loop.)
  const int own_lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  // (For a largest P of 1.)
  const float l = over_halves_sum(rows.l) * (1.0f / 1024.0f), m = rows.m + kAbove;
  float s_ref = rows.s_ref;
  const float down = last_factor(s_ref);
  if (down != 1.0f) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) rows.o[j] *= down;
  }
  if ((own_lane & 31) >= n) return;
  const int in_tile = first + (own_lane & 31), e0 = 4 * (own_lane >> 5);
  if (!whole) {
    const int64_t at = (((int64_t)number * a.cache.heads + h) * a.splits + piece) * kTileRows + in_tile;
    if (own_lane < 32) reinterpret_cast<float2*>(a.part)[at] = make_float2(m, l);
    float* to = a.part + (int64_t)tiles * a.cache.heads * a.splits * (2 * kTileRows) + at * D + e0;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = rows.o[j][4 * x + e] * s_ref;
        *reinterpret_cast<f32x4*>(to + 64 * (j / 2) + 32 * (x / 2) + 16 * (j & 1) + 8 * (x & 1)) = y;
      }
  } else {
    const int r = t.r0 + in_tile, head = h * a.group + r % a.group;
    const int64_t row = t.row0 + r / a.group;
    if (a.lse != nullptr && own_lane < 32)
      a.lse[row * a.q_heads + head] = l == 0.0f ? kNone : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
    const float f = l == 0.0f ? 0.0f : s_ref / l;
    uint16_t* to = a.y + row * a.ldy + (int64_t)head * D + e0;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<uint2*>(to + 64 * (j / 2) + 32 * (x / 2) + 16 * (j & 1) + 8 * (x & 1)) =
            make_uint2(bf16_pair(rows.o[j][4 * x] * f, rows.o[j][4 * x + 1] * f),
                       bf16_pair(rows.o[j][4 * x + 2] * f, rows.o[j][4 * x + 3] * f));
  }
}

// A whole kernel of it: heads side by side, then a tile's pieces, the longest rows first.
template <int D, bool kSplit, typename Args>
__device__ __forceinline__ void attention_tile_kernel(Args a, int tiles) {
  __shared__ TileLds<D> lds;
  int id = blockIdx.x;
  const int h = id % a.cache.heads;
  id /= a.cache.heads;
  const int number = tiles - 1 - (kSplit ? id / a.splits : id);
  const int piece = kSplit ? piece_of(id % a.splits, number, a.splits) : 0;
  attention_tile<D, kSplit>(a, tiles, h, number, piece, lds);
}

}  // namespace nvfp4
