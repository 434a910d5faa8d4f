// Device code that the attention kernels share: the rows of a workgroup, their
// running softmax, and the two products of one tile of 32 tokens.
//
// Rows.  The `group` query heads of one key head read the same keys, so a
// sequence's rows are packed: packed row r is new token r / group with query
// head h * group + r % group.
//
// One pass with a running maximum m and sum l (in powers of two; the scale
// holds log2 e):  S^T = K Q^T by v_mfma_f32_16x16x32_bf16 (E4M3 keys are exact
// in bf16), P = 2^(S - m), Y^T += V^T P^T by v_mfma_f32_16x16x32_f16 (E4M3
// values are exact in f16).  With the products transposed, a lane holds the
// scores of ONE row, for the tokens 4 g .. 4 g + 3 of two groups of 16 (g =
// lane / 16), and these are the elements that the second product wants of it:
// its contraction index is taken in that order, 8 g + e being token 4 g + e of
// the first group and 8 g + 4 + e of the second.  So P never leaves its lane.
// The cache's order makes both operands whole 16-byte loads of a contiguous
// kilobyte for each wave.
//
// m is kept kAbove below the largest score met, whose P is then about 2^kAbove: so
// P uses binary16's range up to its end, and a token keeps its 11 bits down to 2^-24
// of the largest P and is off by 2^-35 of that below (twice that where P takes a part
// of a value scale, below).  With a largest P of 1, tokens
// behind an attention sink were lost from Y but not from l (8192 tokens 17 nats
// below one whose values are zero: Y 41% off; now 0.1%).
//
// The page's key scale goes into the scores.  Its value scale, over the largest one
// met so far (s_ref, by which Y is multiplied at the end) and times the 2^7 that 448
// leaves of binary16's range, goes into the values' conversion to binary16 (a power
// of two) and into P (what is left of it, nothing for the powers of two that the
// append takes).  Values are exact down to a scale of 2^-22 of the largest.
#pragma once

#include "attention_device.h"

namespace nvfp4 {

constexpr int kTileTokens = 32;
constexpr float kNone = -__builtin_inff();

// The largest P is 2^kAbove where m was last set.  The tile kernel takes 16 of them
// before it looks for a maximum, so no more than 2^11 would do; with 10, a score may
// pass the largest by 6 until it does, and by 5.9 in the other kernels (to kHighest:
// 2^15.9 < 65504).
constexpr float kAbove = 10.0f, kHighest = 15.9f;
constexpr float kValueRoom = 128.0f;               // 448 * 2^7 < 65504
constexpr float kSmallest = 0x1p-119f;             // of s_ref: over kValueRoom, a normal number

// The running m for a largest score, whose own P is then 2^kAbove without a rounding
// (it weighs most; with m a whole number, 7.5 to 9% of y were one step of bf16 beside
// the rounded exact value, so 5 to 7%).  Scores that have no fraction left, and -infinity, stay.
__device__ __forceinline__ float reference(float top) { return fabsf(top) < 16777216.0f ? top - kAbove : top; }

// The first token that token t's row sees of a window of at least 1 (below 0: all).
// (A t below 0 counts as 0, so that no window below 2^31 takes it out of 32 bits.)
__device__ __forceinline__ int window_begin(int t, int window) { return max(t, 0) - (window - 1); }

// Packed rows of one tile and the tokens that they see.
struct Tile {
  int b, row0, rows, r0, n;      // sequence, its first row and rows, first packed row, packed rows of this tile
  int first;                     // token of the sequence's first new row
  int begin, end;                // tokens that some row of the tile sees
};

// Sequence b's tiles have the numbers from cu_rows[b] * group / kRows + b on
// (it has ceil(n_b * group / kRows) of them).
template <int kRows>
__device__ __forceinline__ bool find_tile(const AttentionArgs& a, int number, Tile& t) {
  int ordinal;
  const SeqRows s = find_rows(a.batch, number, (a.group + kRows - 1) / kRows, t.b, ordinal, [&](int row, int b) {
    return (int)((int64_t)row * a.group / kRows) + b;
  });
  t.row0 = s.row;
  t.rows = s.rows;
  t.first = s.first;
  if (ordinal < 0 || (int64_t)ordinal * kRows >= s.rows * a.group) return false;
  t.r0 = ordinal * kRows;
  t.n = min(kRows, s.rows * a.group - t.r0);
  const int lowest = t.first + t.r0 / a.group, highest = t.first + (t.r0 + t.n - 1) / a.group;
  t.end = a.causal ? min(s.len, highest + 1) : s.len;
  // (Not behind the end: a length that makes no sense would put it near 2^31.)
  t.begin = a.window > 0 ? min(max(0, window_begin(lowest, a.window)), max(0, t.end)) : 0;
  return true;
}

// The piece of a tile that its x-th workgroup takes: another order for each tile.
// Workgroups go to the dies and to their shader engines in turn, and the last
// pieces, which short sequences do not have, would otherwise be the same one's.
__device__ __forceinline__ int piece_of(int x, int number, int splits) {
  return (x + number + (number >> 2) + (number >> 5)) % splits;
}

// A tile's pieces of a.chunk tokens each, from the first token that one of its rows
// sees (its step of 64) on; the last one takes what is left.  A tile that sees
// nothing has one.
__device__ __forceinline__ int pieces_of(const AttentionArgs& a, const Tile& t) {
  return t.begin < t.end ? min((t.end - 1 - (t.begin & ~63)) / a.chunk, a.splits - 1) + 1 : 1;
}

// Tokens [begin, end) of a tile's piece.
__device__ __forceinline__ void piece_tokens(const AttentionArgs& a, const Tile& t, int piece, int& begin, int& end) {
  const int from = (t.begin & ~63) + piece * a.chunk;
  begin = max(t.begin, from);
  end = piece + 1 < a.splits ? min(t.end, from + a.chunk) : t.end;
}

__device__ __forceinline__ int64_t tiles_of(const KvBatchArgs& a, int group, int rows) {
  return a.cu_rows == nullptr ? (int64_t)a.seqs * ((group + rows - 1) / rows)
                              : (int64_t)a.rows * group / rows + a.seqs;
}

// Tiles that partial results are kept for.
__device__ __forceinline__ int64_t part_tiles(const AttentionArgs& a, int rows) { return tiles_of(a.batch, a.group, rows); }

// At the end: s_ref becomes what Y is multiplied by for a largest P of 1; the result,
// what Y is multiplied by before that: 1, but where s_ref over l might otherwise be no
// normal number (value scales below 2^-89).
__device__ __forceinline__ float last_factor(float& s_ref) {
  const bool tiny = s_ref < 0x1p-89f;
  s_ref *= tiny ? 0x1p+23f : 0x1p-17f;
  return tiny ? 0x1p-40f : 1.0f;
}

// 8 E4M3 values in bf16 (exact), and in f16 times a power of two.
__device__ __forceinline__ bf16x8 bf16_of(uint32_t a, uint32_t b) {
  union {
    bf16x2 p[4];
    bf16x8 v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return u.v;
}

__device__ __forceinline__ f16x8 f16_of(uint32_t a, uint32_t b, float scale_a, float scale_b) {
  union {
    f16x2 p[4];
    f16x8 v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, scale_a, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, scale_a, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, scale_b, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, scale_b, true);
  return u.v;
}

// E4M3 NaN codes (0x7F, 0xFF) to zero: a masked token's probability is zero,
// and zero times whatever its slot holds has to be.
__device__ __forceinline__ uint32_t without_nan(uint32_t x) {
  const uint32_t hit = ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;      // a byte's top bit where it is NaN
  return x & ~((hit >> 7) * 255u);
}

// Maximum and sum over the four lanes lane % 16 + 16 i.
__device__ __forceinline__ float over_quarters_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float over_quarters_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Page and scales of the groups of 16 tokens that a wave meets next: its lane
// holds those of the group at `token`, page -1 where that is past the end or in
// front of the beginning (a window's first tile may begin in pages that nobody
// sees, whose scales may be anything) or its page is not in the cache.
struct GroupPages {
  int page;
  float k_scale, v_scale;
};

__device__ __forceinline__ GroupPages group_pages(const AttentionArgs& a, int b, int h, int64_t token, int begin,
                                                  int end) {
  GroupPages g;
  g.page = -1;
  g.k_scale = g.v_scale = 0.0f;
  if (token < end && token + 16 > begin) {
    const int p = a.batch.table[(int64_t)b * a.batch.table_stride + (token >> a.cache.page_shift)];
    if (p >= 0 && p < a.cache.num_pages) {
      g.page = p;
      g.k_scale = a.cache.scale[0][(int64_t)p * a.cache.scale_stride + h];
      g.v_scale = a.cache.scale[1][(int64_t)p * a.cache.scale_stride + h];
    }
  }
  return g;
}

__device__ __forceinline__ float lane_of(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

// s_waitcnt operands: at most n vector memory operations outstanding, or no LDS
// access (the other counters are not waited for).
constexpr int wait_loads(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }
constexpr int kWaitLds = 0xC07F;

// One head's group of 16 tokens (16 D bytes) from its page to LDS, whole wave,
// D / 64 loads that write LDS directly (lane's 16 bytes at 16 lane).  A page
// that is not in the cache is read as page 0 (its tokens are masked).
template <int D>
__device__ __forceinline__ void stage_group(const KvCacheArgs& c, int kind, int page, int slot, int h, int lane,
                                            uint8_t* to) {
  const uint8_t* from = c.kv[kind] + (int64_t)max(page, 0) * c.page_stride[kind] + ((int64_t)h * c.page_size + slot) * D;
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(from), (short)0, 16 * D, 0x00020000);
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(to + i * 1024), 16, lane * 16,
                                             i * 1024, 0, 0);
}

// The rows of one wave, 16 kTiles of them, and what they have met so far.
template <int D, int kTiles>
struct RowTiles {
  static constexpr int kSteps = D / 32, kOut = D / 16;
  bf16x8 q[kTiles][kSteps];
  f32x4 o[kTiles][kOut];
  float m[kTiles], l[kTiles];
  int at[kTiles];                // each lane's tokens
  int begin, end;                // tokens that the wave looks at
  int all0, all1;                // those that every row sees
  float s_ref, s_inv;

  // Packed rows from r0 on, n of them (lanes of rows behind take the last one).
  __device__ __forceinline__ void start(const AttentionArgs& a, const Tile& t, int h, int r0, int n, int lane,
                                        int from, int to) {
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;      // the scale's sign goes into Q
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int r = r0 + min(16 * i + (lane & 15), n - 1);
      at[i] = t.first + r / a.group;
      const uint16_t* src = a.q + (int64_t)(t.row0 + r / a.group) * a.ldq +
                            (int64_t)(h * a.group + r % a.group) * D + (lane >> 4) * 16;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(src + (s / 2) * 64 + (s & 1) * 8);
        q[i][s] = __builtin_bit_cast(bf16x8, w ^ flip);
      }
      m[i] = kNone;
      l[i] = 0.0f;
#pragma unroll
      for (int j = 0; j < kOut; ++j) o[i][j] = (f32x4){0, 0, 0, 0};
    }
    begin = from;
    end = to;
    const int low = t.first + r0 / a.group, high = t.first + (r0 + n - 1) / a.group;
    all1 = a.causal ? min(end, low + 1) : end;
    all0 = a.window > 0 ? max(begin, window_begin(high, a.window)) : begin;
    s_ref = kSmallest;
    s_inv = kValueRoom / kSmallest;
  }

  // At the end: m, l and what Y is multiplied by, for a largest P of 1.
  __device__ __forceinline__ void finish() {
    const float down = last_factor(s_ref);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      l[i] = over_quarters_sum(l[i]) * (1.0f / 1024.0f);
      m[i] += kAbove;
      if (down != 1.0f) {
#pragma unroll
        for (int j = 0; j < kOut; ++j) o[i][j] *= down;
      }
    }
  }

  // Tokens token .. token + 31: the codes of keys(g, c) and values(g, c) are
  // those of group g and elements 64 c .. 64 c + 63; ks holds the key scales
  // times |scale|, vs the value scales; there: both pages are in the cache.
  // keys_done, values_done: called where the codes have been read.
  template <typename Keys, typename Values, typename KeysDone, typename ValuesDone>
  __device__ __forceinline__ void pass(const AttentionArgs& a, int token, bool there0, bool there1, const float (&ks)[2],
                                       const float (&vs)[2], int lane, Keys keys, Values values, KeysDone keys_done,
                                       ValuesDone values_done) {
    f32x4 s[kTiles][2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) s[i][g] = (f32x4){0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const u32x4 k = keys(g, c);
        const bf16x8 k0 = bf16_of(k[0], k[1]), k1 = bf16_of(k[2], k[3]);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) s[i][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[i][2 * c], s[i][g], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          s[i][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[i][2 * c + 1], s[i][g], 0, 0, 0);
      }
    }
    keys_done();
    const bool whole = token >= all0 && token + kTileTokens <= all1 && there0 && there1;
    if (!whole) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const int see1 = a.causal ? min(end, at[i] + 1) : end;
        const int see0 = a.window > 0 ? max(begin, window_begin(at[i], a.window)) : begin;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = token + 16 * g + 4 * (lane >> 4) + e;
            if (j < see0 || j >= see1 || !(g ? there1 : there0)) s[i][g][e] = kNone;
          }
      }
    }
    // m follows only where P would pass binary16's range.
    float top[kTiles];
    bool over = false;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      top[i] = fmaxf(fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3])) * ks[0],
                     fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3])) * ks[1]);
      over |= top[i] - m[i] > kHighest;
    }
    if (__any(over)) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const float m_new = fmaxf(m[i], reference(over_quarters_max(top[i])));
        const float f = m[i] == m_new ? 1.0f : __builtin_amdgcn_exp2f(m[i] - m_new);      // (0 from nothing)
        l[i] *= f;
#pragma unroll
        for (int j = 0; j < kOut; ++j) o[i][j] *= f;
        m[i] = m_new;
      }
    }
    const float v_top = fmaxf(vs[0], vs[1]);
    if (v_top > s_ref) {
      const float f = s_ref / v_top;
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < kOut; ++j) o[i][j] *= f;
      s_ref = v_top;
      s_inv = kValueRoom / v_top;
    }
    float w[kTiles][8];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const float base = m[i] == kNone ? 0.0f : m[i];
      float sum = 0.0f;      // (the tile's own first: fewer roundings at the size of the whole)
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[i][4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[i][g][e], ks[g], -base));
          sum += w[i][4 * g + e];
        }
      l[i] += sum;
    }
    float power[2];
    bool rest = false;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const uint32_t bits = __float_as_uint(vs[g] * s_inv);
      power[g] = __uint_as_float(bits & 0x7F800000u);
      rest |= (bits & 0x7FFFFFu) != 0;
    }
    if (rest) {      // the power of two above the ratio (at most kValueRoom), and 1/2 to 1 of P
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const uint32_t part = __float_as_uint(vs[g] * s_inv) & 0x7FFFFFu;
        const float f = part != 0 ? __uint_as_float(part | 0x3F000000u) : 1.0f;
        power[g] *= part != 0 ? 2.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) w[i][4 * g + e] *= f;
      }
    }
    f16x8 p[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) p[i][e] = (_Float16)w[i][e];
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      u32x4 v0 = values(0, c), v1 = values(1, c);
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v0[j] = without_nan(v0[j]), v1[j] = without_nan(v1[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f16x8 v = f16_of(v0[j], v1[j], power[0], power[1]);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          o[i][4 * c + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[i], o[i][4 * c + j], 0, 0, 0);
      }
    }
    values_done();
  }
};

}  // namespace nvfp4
