// Attention over the paged E4M3 cache for gfx950 (layout and definition:
// nvfp4_attention.h).
//
// Rows.  The `group` query heads of one key head read the same keys, so a
// sequence's rows are packed: packed row r is new token r / group with query
// head h * group + r % group.  A workgroup takes 16 packed rows of one sequence
// and key head; its four waves take turns with tiles of 32 tokens.
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
// kilobyte for each wave, without LDS.
//
// The page's key scale goes into the scores.  Its value scale goes into P,
// divided by the largest one met so far (s_ref, by which Y is multiplied at the
// end), so that P stays at most 1 in binary16: what falls below 2^-25 of the
// largest value met is dropped.
//
// Bound by HBM for few rows: the waves' loads of one tile ahead are what covers
// its latency.
#include "attention_device.h"

namespace nvfp4 {

constexpr int kRowsThreads = 256;
constexpr int kRowsWaves = kRowsThreads / 64;
constexpr int kTileTokens = 32;

// Packed rows of one tile and the tokens that they see.
struct Tile {
  int b, row0, rows, r0, n;      // sequence, its first row and rows, first packed row, packed rows of this tile
  int first;                     // token of the sequence's first new row
  int begin, end;                // tokens that some row of the tile sees
};

__device__ __forceinline__ int row_bound(const KvBatchArgs& a, int b) { return min(max(a.cu_rows[b], 0), a.rows); }

// Sequence b's tiles have the numbers from cu_rows[b] * group / kRows + b on
// (it has ceil(n_b * group / kRows) of them).
template <int kRows>
__device__ __forceinline__ bool find_tile(const AttentionArgs& a, int number, Tile& t) {
  int ordinal;
  if (a.batch.cu_rows == nullptr) {
    const int each = (a.group + kRows - 1) / kRows;
    t.b = number / each;
    ordinal = number % each;
  } else {
    int lo = 0, hi = a.batch.seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if ((int)((int64_t)row_bound(a.batch, mid) * a.group / kRows) + mid <= number)
        lo = mid;
      else
        hi = mid - 1;
    }
    t.b = lo;
    ordinal = number - ((int)((int64_t)row_bound(a.batch, lo) * a.group / kRows) + lo);
  }
  const SeqRows s = seq_rows(a.batch, t.b);
  t.row0 = s.row;
  t.rows = s.rows;
  t.first = s.first;
  t.r0 = ordinal * kRows;
  t.n = min(kRows, s.rows * a.group - t.r0);
  if (ordinal < 0 || t.n <= 0) return false;
  const int lowest = t.first + t.r0 / a.group, highest = t.first + (t.r0 + t.n - 1) / a.group;
  t.end = a.causal ? min(s.len, highest + 1) : s.len;
  t.begin = a.window > 0 ? max(0, lowest - a.window + 1) : 0;
  return true;
}

__device__ __forceinline__ int64_t tiles_of(const KvBatchArgs& a, int group, int rows) {
  return a.cu_rows == nullptr ? (int64_t)a.seqs * ((group + rows - 1) / rows)
                              : (int64_t)a.rows * group / rows + a.seqs;
}

// 8 E4M3 values in bf16 or f16 (exact).
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

__device__ __forceinline__ f16x8 f16_of(uint32_t a, uint32_t b) {
  union {
    f16x2 p[4];
    f16x8 v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
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

// Keys and values of one tile of 32 tokens, as loaded: [group of 16][64
// elements of the head].
template <int D>
struct TileCodes {
  u32x4 k[2][D / 64], v[2][D / 64];
};

// Page and scales of the groups of 16 tokens that this wave meets: lane 2 i
// and 2 i + 1 hold those of its i-th tile from `from` on, page -1 where the
// group is past the end or its page is not in the cache.
struct GroupPages {
  int page;
  float k_scale, v_scale;
};

__device__ __forceinline__ GroupPages group_pages(const AttentionArgs& a, int b, int h, int from, int step, int end,
                                                  int lane) {
  GroupPages g;
  g.page = -1;
  g.k_scale = g.v_scale = 0.0f;
  const int64_t token = (int64_t)from + (int64_t)(lane >> 1) * step + (lane & 1) * 16;
  if (token < end) {
    const int p = a.batch.table[(int64_t)b * a.batch.table_stride + (token >> a.cache.page_shift)];
    if (p >= 0 && p < a.cache.num_pages) {
      g.page = p;
      g.k_scale = a.cache.scale[0][(int64_t)p * a.cache.scale_stride + h];
      g.v_scale = a.cache.scale[1][(int64_t)p * a.cache.scale_stride + h];
    }
  }
  return g;
}

template <int D>
__device__ __forceinline__ void load_tile(const AttentionArgs& a, int h, int token, int page0, int page1, int lane,
                                          TileCodes<D>& t) {
  const int mask = a.cache.page_size - 1;
  const int64_t head = (int64_t)h * a.cache.page_size * D;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int page = g ? page1 : page0, slot = (token + 16 * g) & mask;
    const uint8_t* k = a.cache.kv[0] + (int64_t)max(page, 0) * a.cache.page_stride[0] + head + slot * D;
    const uint8_t* v = a.cache.kv[1] + (int64_t)max(page, 0) * a.cache.page_stride[1] + head + slot * D;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      t.k[g][c] = *reinterpret_cast<const u32x4*>(k + c * 1024 + lane * 16);
      t.v[g][c] = *reinterpret_cast<const u32x4*>(v + c * 1024 + lane * 16);
    }
  }
}

constexpr float kNone = -__builtin_inff();

template <int D, bool kSplit>
__global__ __launch_bounds__(kRowsThreads, 2) void kv_attention_rows_kernel(AttentionArgs a) {
  constexpr int kSteps = D / 32, kOut = D / 16;
  constexpr int kHalf = D > 128 ? 128 : D;             // elements of a row that are joined at a time
  __shared__ float joined[kRowsWaves][16][kHalf + 4];
  __shared__ float2 stats[kRowsWaves][16];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, quarter = lane >> 4;
  int id = blockIdx.x;
  const int h = id % a.cache.heads;
  id /= a.cache.heads;
  const int piece = kSplit ? id % a.splits : 0;
  const int number = kSplit ? id / a.splits : id;
  Tile t;
  if (!find_tile<16>(a, number, t)) return;
  int begin = t.begin, end = t.end;
  if (kSplit) {
    begin = max(begin, piece * a.chunk);
    if (piece + 1 < a.splits) end = min(end, (piece + 1) * a.chunk);
    if (begin >= end && !(piece == 0 && t.begin >= t.end)) return;      // (rows that see nothing: piece 0 says so)
  }

  // This lane's row; Q in the order of the keys' loads.
  const int r = t.r0 + min(col, t.n - 1);
  const int token_row = t.row0 + r / a.group, head = h * a.group + r % a.group;
  const int at = t.first + r / a.group;
  bf16x8 q[kSteps];
  {
    const uint16_t* src = a.q + (int64_t)token_row * a.ldq + (int64_t)head * D + quarter * 16;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(src + (s / 2) * 64 + (s & 1) * 8));
  }
  // Tokens [see0, see1) are seen by this lane's row; [all0, all1) by every row.
  const int see1 = a.causal ? min(end, at + 1) : end;
  const int see0 = a.window > 0 ? max(begin, at - a.window + 1) : begin;
  const int low = t.first + t.r0 / a.group, high = t.first + (t.r0 + t.n - 1) / a.group;
  const int all1 = a.causal ? min(end, low + 1) : end;
  const int all0 = a.window > 0 ? max(begin, high - a.window + 1) : begin;

  f32x4 o[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) o[i] = (f32x4){0, 0, 0, 0};
  float m = kNone, l = 0.0f, s_ref = 1.17549435e-38f, s_inv = 1.0f / 1.17549435e-38f;

  const int step = kRowsWaves * kTileTokens;
  int token = (begin & ~(kTileTokens - 1)) + wave * kTileTokens;
  GroupPages pages = group_pages(a, t.b, h, token, step, end, lane);
  int in_batch = 0;
  TileCodes<D> now, next;
  if (token < end)
    load_tile<D>(a, h, token, __builtin_amdgcn_readlane(pages.page, 0), __builtin_amdgcn_readlane(pages.page, 1), lane,
                 now);
  while (token < end) {
    const int page0 = __builtin_amdgcn_readlane(pages.page, 2 * in_batch);
    const int page1 = __builtin_amdgcn_readlane(pages.page, 2 * in_batch + 1);
    float ks[2], vs[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      ks[g] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pages.k_scale), 2 * in_batch + g)) * a.scale;
      vs[g] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pages.v_scale), 2 * in_batch + g));
    }
    const int ahead = token + step;
    if (++in_batch == 32) {
      pages = group_pages(a, t.b, h, ahead, step, end, lane);
      in_batch = 0;
    }
    if (ahead < end)
      load_tile<D>(a, h, ahead, __builtin_amdgcn_readlane(pages.page, 2 * in_batch),
                   __builtin_amdgcn_readlane(pages.page, 2 * in_batch + 1), lane, next);

    f32x4 s[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      s[g] = (f32x4){0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        s[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(now.k[g][c][0], now.k[g][c][1]), q[2 * c], s[g], 0, 0, 0);
        s[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(now.k[g][c][2], now.k[g][c][3]), q[2 * c + 1], s[g], 0, 0, 0);
      }
    }
    const bool whole = token >= all0 && token + kTileTokens <= all1 && page0 >= 0 && page1 >= 0;
    float x[8];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * g + e] = s[g][e] * ks[g];
    if (!whole) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = token + 16 * g + 4 * quarter + e;
          if (j < see0 || j >= see1 || (g ? page1 : page0) < 0) x[4 * g + e] = kNone;
        }
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) now.v[g][c][i] = without_nan(now.v[g][c][i]);
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = over_quarters_max(top);
    if (__any(top > m)) {
      const float m_new = fmaxf(m, top);
      const float f = m == m_new ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);      // (0 from nothing)
      l *= f;
#pragma unroll
      for (int i = 0; i < kOut; ++i) o[i] *= f;
      m = m_new;
    }
    const float v_top = fmaxf(vs[0], vs[1]);
    if (v_top > s_ref) {
      const float f = s_ref / v_top;
#pragma unroll
      for (int i = 0; i < kOut; ++i) o[i] *= f;
      s_ref = v_top;
      s_inv = 1.0f / v_top;
    }
    const float base = m == kNone ? 0.0f : m;
    f16x8 p;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float ratio = vs[g] * s_inv;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float w = __builtin_amdgcn_exp2f(x[4 * g + e] - base);
        l += w;
        p[4 * g + e] = (_Float16)(w * ratio);
      }
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        o[4 * c + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of(now.v[0][c][i], now.v[1][c][i]), p, o[4 * c + i],
                                                             0, 0, 0);
    now = next;
    token = ahead;
  }

  // The four waves' results, joined: Y = sum_w 2^(m_w - m) Y_w.
  l = over_quarters_sum(l);
  if (quarter == 0) stats[wave][col] = make_float2(m, l);
  __syncthreads();
  float m_all = kNone, l_all = 0.0f;
#pragma unroll
  for (int w = 0; w < kRowsWaves; ++w) m_all = fmaxf(m_all, stats[w][col].x);
  const float zero_m = m_all == kNone ? 0.0f : m_all;
#pragma unroll
  for (int w = 0; w < kRowsWaves; ++w) l_all += stats[w][col].y * __builtin_amdgcn_exp2f(stats[w][col].x - zero_m);
  float mine = __builtin_amdgcn_exp2f(m - zero_m) * s_ref;
  if (!kSplit) mine *= l_all == 0.0f ? 0.0f : 1.0f / l_all;
  if (threadIdx.x < 16 && threadIdx.x < t.n) {
    if (kSplit) {
      float2* to = reinterpret_cast<float2*>(a.part) + (((int64_t)number * a.cache.heads + h) * a.splits + piece) * 16;
      to[threadIdx.x] = make_float2(m_all, l_all);
    } else if (a.lse != nullptr) {
      a.lse[(int64_t)token_row * a.q_heads + head] =
          l_all == 0.0f ? kNone : (m_all + __builtin_amdgcn_logf(l_all)) * 0.69314718055994531f;
    }
  }
#pragma unroll
  for (int d0 = 0; d0 < D; d0 += kHalf) {
    if (d0 > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < kHalf / 16; ++i)
      *reinterpret_cast<f32x4*>(&joined[wave][col][16 * i + 4 * quarter]) = o[d0 / 16 + i] * mine;
    __syncthreads();
    // A thread takes four elements of one row.
    for (int x = threadIdx.x; x < 16 * kHalf / 4; x += kRowsThreads) {
      const int row = x / (kHalf / 4), e = (x % (kHalf / 4)) * 4;
      if (row >= t.n) continue;
      f32x4 y = (f32x4){0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < kRowsWaves; ++w) y += *reinterpret_cast<const f32x4*>(&joined[w][row][e]);
      if (kSplit) {
        const int64_t pieces = (tiles_of(a.batch, a.group, 16) * a.cache.heads) * a.splits * 32;      // floats of stats
        float* to = a.part + pieces +
                    ((((int64_t)number * a.cache.heads + h) * a.splits + piece) * 16 + row) * D + d0 + e;
        *reinterpret_cast<f32x4*>(to) = y;
      } else {
        const int rr = t.r0 + row;
        uint16_t* to = a.y + (int64_t)(t.row0 + rr / a.group) * a.ldy + (int64_t)(h * a.group + rr % a.group) * D + d0 + e;
        *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
      }
    }
  }
}

// Joins the pieces of a sequence: one wave for each packed row.
template <int D>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(task % 16);
  const int h = (int)(task / 16 % a.cache.heads);
  const int64_t number = task / 16 / a.cache.heads;
  const int64_t tiles = tiles_of(a.batch, a.group, 16);
  if (number >= tiles) return;
  Tile t;
  if (!find_tile<16>(a, (int)number, t) || row >= t.n) return;
  const int64_t first = (number * a.cache.heads + h) * a.splits;
  const float2* stats = reinterpret_cast<const float2*>(a.part) + first * 16 + row;
  const float* part = a.part + tiles * a.cache.heads * a.splits * 32 + (first * 16 + row) * D;
  int p0 = 0, p1 = 1;
  if (t.begin < t.end) {
    p0 = min(t.begin / a.chunk, a.splits - 1);
    p1 = min((t.end - 1) / a.chunk, a.splits - 1) + 1;
  }
  float m = kNone;
  for (int p = p0 + lane; p < p1; p += 64) m = fmaxf(m, stats[p * 16].x);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
  const float base = m == kNone ? 0.0f : m;
  float l = 0.0f, y[D / 64];
#pragma unroll
  for (int i = 0; i < D / 64; ++i) y[i] = 0.0f;
  for (int p = p0; p < p1; ++p) {
    const float2 st = stats[p * 16];
    const float f = __builtin_amdgcn_exp2f(st.x - base);
    l += st.y * f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) y[i] = fmaf(part[(int64_t)p * 16 * D + lane * (D / 64) + i], f, y[i]);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int r = t.r0 + row, head = h * a.group + r % a.group;
  const int64_t token_row = t.row0 + r / a.group;
  uint16_t* to = a.y + token_row * a.ldy + (int64_t)head * D + lane * (D / 64);
  if (D == 64)
    *to = __builtin_bit_cast(uint16_t, (__bf16)(y[0] * inv));
  else
#pragma unroll
    for (int i = 0; i + 1 < D / 64; i += 2) *reinterpret_cast<uint32_t*>(to + i) = bf16_pair(y[i] * inv, y[i + 1] * inv);
  if (a.lse != nullptr && lane == 0)
    a.lse[token_row * a.q_heads + head] = l == 0.0f ? kNone : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

namespace {

int64_t host_tiles(const KvBatchArgs& b, int group, int rows) {
  return b.cu_rows == nullptr ? (int64_t)b.seqs * ((group + rows - 1) / rows) : (int64_t)b.rows * group / rows + b.seqs;
}

// Pieces of a sequence: enough workgroups for four on each of 256 compute
// units, of 256 tokens at least.
void plan(const KvCacheArgs& c, const KvBatchArgs& b, int group, int& chunk, int& splits) {
  const int64_t work = host_tiles(b, group, 16) * c.heads;
  int64_t want = work > 0 ? (1024 + work - 1) / work : 1;
  int64_t each = want > 0 ? (b.max_kv_len + want - 1) / want : b.max_kv_len;
  each = (each + 127) / 128 * 128;
  if (each < 256) each = 256;
  splits = (int)((b.max_kv_len + each - 1) / each);
  if (splits < 1) splits = 1;
  chunk = (int)each;
}

}  // namespace

size_t kv_attention_workspace_bytes(const KvCacheArgs& c, const KvBatchArgs& b, int q_heads) {
  if (b.seqs == 0 || b.rows == 0) return 0;
  int chunk, splits;
  const int group = q_heads / c.heads;
  plan(c, b, group, chunk, splits);
  if (splits == 1) return 0;
  return (size_t)(host_tiles(b, group, 16) * c.heads * splits * 16) * (c.dim + 2) * sizeof(float);
}

template <int D>
hipError_t launch_attention(const AttentionArgs& a, hipStream_t stream) {
  const int64_t work = host_tiles(a.batch, a.group, 16) * a.cache.heads;
  if (work * a.splits >= (int64_t)1 << 31) return hipErrorInvalidValue;
  if (a.splits == 1) {
    kv_attention_rows_kernel<D, false><<<dim3((unsigned)work), kRowsThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  kv_attention_rows_kernel<D, true><<<dim3((unsigned)(work * a.splits)), kRowsThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  kv_attention_join_kernel<D><<<dim3((unsigned)(work * 4)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_attention(const AttentionArgs& args, void* workspace, hipStream_t stream) {
  AttentionArgs a = args;
  plan(a.cache, a.batch, a.group, a.chunk, a.splits);
  a.part = static_cast<float*>(workspace);
  return a.cache.dim == 64    ? launch_attention<64>(a, stream)
         : a.cache.dim == 128 ? launch_attention<128>(a, stream)
                              : launch_attention<256>(a, stream);
}

}  // namespace nvfp4
