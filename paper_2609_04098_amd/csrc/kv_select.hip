// The pages that an attention reads, chosen by a score of their bounds (definition:
// nvfp4_paging.h), for gfx950.
//
// Bounds: each full page's largest and smallest key elements in 8 bits, hi_e and lo_e
// in 127ths of the largest magnitude.  With a query in 8 bits, q_e,
//   sum_e max(q_e hi_e, q_e lo_e) = sum_e max(q_e, 0) hi_e + min(q_e, 0) lo_e
// bounds its products with all of the page's keys: one product of 2 D elements, by
// v_mfma_i32_16x16x64_i8 for 16 pages and 16 query heads at a time.  The sums are whole
// numbers, the factors behind them one binary32 product each, so that a choice depends
// on no order of sums and ties are ties.
//
// Bound by the bounds' bytes, 2 D + 4 of a page's page_size * 2 D, where there are many
// rows; else by launches and the selection's passes over a row's scores.  32 rows of up to 32768
// tokens, 8 key heads of 128, pages of 16: 23 us for 61 MB, the selection (7.4 where it is a launch
// of its own) among them, during which a compute unit's only workgroup loads nothing; one row of 131072, pages of 64: 4.9 and 7.4.
// The bounds of two prompts of up to 16000 tokens, 8 heads of 128, pages of 32: 10.4 us for 28 MB,
// a launch and three loads' latencies in front of them.
#include <type_traits>
#include "attention_plan.h"
#include "kv_attention_device.h"
#include "paging_launch.h"

namespace nvfp4 {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- bounds

// The other lanes of a row of 16 (all lanes active): as in kv_append.hip.
template <int kHow>
__device__ __forceinline__ uint32_t row_other(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kHow, 0xF, 0xF, true);
}

__device__ __forceinline__ f16x2 max2(f16x2 a, f16x2 b) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ f16x2 min2(f16x2 a, f16x2 b) { return __builtin_elementwise_min(a, b); }

template <bool kMax>
__device__ __forceinline__ f16x2 pick(f16x2 a, f16x2 b) { return kMax ? max2(a, b) : min2(a, b); }

template <int kHow, bool kMax>
__device__ __forceinline__ f16x2 fold(f16x2 v) {
  return pick<kMax>(v, __builtin_bit_cast(f16x2, row_other<kHow>(__builtin_bit_cast(uint32_t, v))));
}

// Of 8 pairs of elements in each of 16 lanes the largest (or smallest) over the lanes: a
// lane ends with pairs 4 (lane % 2) + 2 (lane / 2 % 2) and the one behind it.  (With a
// neighbour each gives away half of what it has; then lanes that have the same, 4, 8
// and 12 apart.)
template <bool kMax>
__device__ __forceinline__ void over_row(const f16x2 (&v)[8], bool odd, bool high, f16x2 (&to)[2]) {
  f16x2 four[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t send = __builtin_bit_cast(uint32_t, odd ? v[i] : v[i + 4]);
    four[i] = pick<kMax>(odd ? v[i + 4] : v[i], __builtin_bit_cast(f16x2, row_other<0xB1>(send)));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t send = __builtin_bit_cast(uint32_t, high ? four[i] : four[i + 2]);
    to[i] = pick<kMax>(high ? four[i + 2] : four[i], __builtin_bit_cast(f16x2, row_other<0x4E>(send)));
    to[i] = fold<0x128, kMax>(fold<0x124, kMax>(to[i]));
  }
}

// The largest value of a row of 16 lanes.
__device__ __forceinline__ float row_max(float m) {
  m = fmaxf(m, __uint_as_float(row_other<0xB1>(__float_as_uint(m))));
  m = fmaxf(m, __uint_as_float(row_other<0x4E>(__float_as_uint(m))));
  m = fmaxf(m, __uint_as_float(row_other<0x141>(__float_as_uint(m))));
  return fmaxf(m, __uint_as_float(row_other<0x140>(__float_as_uint(m))));
}

// The larger of this and of what another lane sends.
template <int kHow>
__device__ __forceinline__ float other_max(float keep, float send) {
  return fmaxf(keep, __uint_as_float(row_other<kHow>(__float_as_uint(send))));
}

// Sums over the lanes up to this one (all lanes active).
template <int kHow, int kRows>
__device__ __forceinline__ int from_below(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kHow, kRows, 0xF, false);
}

__device__ __forceinline__ int scan_up(int x) {
  x += from_below<0x111, 0xF>(x);      // one lane below, in a row of 16; two, four, eight
  x += from_below<0x112, 0xF>(x);
  x += from_below<0x114, 0xF>(x);
  x += from_below<0x118, 0xF>(x);
  x += from_below<0x142, 0xA>(x);      // the last lane of the row below, into rows 1 and 3
  x += from_below<0x143, 0xC>(x);      // lane 31, into rows 2 and 3
  return x;
}

// The sum, the smallest and the largest over a row of 16 lanes.
__device__ __forceinline__ int row_sum(int v) {
  v += (int)row_other<0xB1>((uint32_t)v);
  v += (int)row_other<0x4E>((uint32_t)v);
  v += (int)row_other<0x141>((uint32_t)v);
  return v + (int)row_other<0x140>((uint32_t)v);
}

__device__ __forceinline__ uint32_t row_low(uint32_t v) {
  v = min(v, row_other<0xB1>(v));
  v = min(v, row_other<0x4E>(v));
  v = min(v, row_other<0x141>(v));
  return min(v, row_other<0x140>(v));
}

__device__ __forceinline__ uint32_t row_high(uint32_t v) { return ~row_low(~v); }

// The smallest over the four lanes lane % 16 + 16 i.
__device__ __forceinline__ uint32_t over_quarters_low(uint32_t x) {
  const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t y = min(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  return min(b[0], b[1]);
}

// What lanes have written to LDS is there for the others of their wave.
__device__ __forceinline__ void wave_sees_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wave takes one head of one full page.  Pages of sequence b that its new rows
// completed have the numbers from cu_rows[b] / page_size + b on.
template <int D>
__global__ __launch_bounds__(256) void kv_page_bounds_kernel(BoundsArgs a, int items) {
  __shared__ __attribute__((aligned(8))) _Float16 found[4][2][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int h = (int)(id % a.cache.heads), item = (int)(id / a.cache.heads);
  const int shift = a.cache.page_shift, size = a.cache.page_size;
  if (item >= items) return;
  int b, ordinal;
  const SeqRows s = find_rows(a.batch, item, 1, b, ordinal, [&](int row, int x) { return (row >> shift) + x; });
  // (Rows before token 0 and behind the table are not there.)
  const int entry = (max(s.first, 0) >> shift) + ordinal;
  if (ordinal < 0 || s.rows == 0 || entry >= s.len >> shift || (int64_t)entry << shift >= (int64_t)s.first + s.rows) return;
  const int page = a.batch.table[(int64_t)b * a.batch.table_stride + entry];
  if (page < 0 || page >= a.cache.num_pages) return;
  const uint8_t* from = a.cache.kv[0] + (int64_t)page * a.cache.page_stride[0] + (int64_t)h * size * D + lane * 16;
  f16x2 hi[D / 64][8], lo[D / 64][8];
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) hi[c][i] = (f16x2)((_Float16)-INFINITY), lo[c][i] = (f16x2)((_Float16)INFINITY);
  for (int t = 0; t < size; t += 16, from += 16 * D) {
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(from + c * 1024);      // token lane % 16, elements 64 c + 16 (lane / 16) ..
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f16x2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
        const f16x2 y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true);
        hi[c][2 * i] = max2(hi[c][2 * i], x), lo[c][2 * i] = min2(lo[c][2 * i], x);
        hi[c][2 * i + 1] = max2(hi[c][2 * i + 1], y), lo[c][2 * i + 1] = min2(lo[c][2 * i + 1], y);
      }
    }
  }
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    union {
      f16x2 pairs[2];
      uint2 both;
    } top, low;
    over_row<true>(hi[c], odd, high, top.pairs);
    over_row<false>(lo[c], odd, high, low.pairs);
    if ((lane & 12) == 0) {
      const int at = 64 * c + 16 * (lane >> 4) + (odd ? 8 : 0) + (high ? 4 : 0);
      *reinterpret_cast<uint2*>(&found[wave][0][at]) = top.both;
      *reinterpret_cast<uint2*>(&found[wave][1][at]) = low.both;
    }
  }
  wave_sees_lds();
  constexpr int kEach = 2 * D / 64;      // elements of hi, then of lo
  float v[kEach], top = 0.0f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = (float)(&found[wave][0][0])[lane * kEach + i];
    if (fabsf(v[i]) == INFINITY) v[i] = 0.0f;      // (E4M3 has none: only NaN, which a maximum passes over)
    top = fmaxf(top, fabsf(v[i]));
  }
  top = over_quarters_max(row_max(top));
  const float over = top > 0.0f ? top : 1.0f, inv = 1.0f / over;
  uint32_t packed[(kEach + 3) / 4] = {};
#pragma unroll
  for (int i = 0; i < kEach; ++i) {      // (rounded as the exact quotient is: as in query_codes(), with 4 significant bits)
    const float y = v[i] * 127.0f;
    float q = y * inv;
    q = fmaf(fmaf(-q, over, y), inv, q);
    packed[i / 4] |= ((uint32_t)(int)rintf(q) & 255u) << (8 * (i % 4));
  }
  int8_t* to = a.bounds.codes + (int64_t)page * a.bounds.page_stride + (int64_t)h * 2 * D + lane * kEach;
  if constexpr (kEach == 2) *reinterpret_cast<uint16_t*>(to) = (uint16_t)packed[0];
  else if constexpr (kEach == 4) *reinterpret_cast<uint32_t*>(to) = packed[0];
  else *reinterpret_cast<uint2*>(to) = make_uint2(packed[0], packed[1]);
  if (lane == 0) {
    const float scale = a.cache.scale[0][(int64_t)page * a.cache.scale_stride + h];
    a.bounds.step[(int64_t)page * a.bounds.step_stride + h] = top * scale / 127.0f;
  }
}

// ---------------------------------------------------------------- scores

// The row of a step's tensors: its sequence and the pages that it sees (-1: a row behind
// the last sequence).
struct RowPages {
  int b, token, pages;
};

__device__ __forceinline__ RowPages row_pages(const SelectArgs& a, int row) {
  RowPages r;
  int ordinal;
  // (Its sequence: the last that begins at or before it; those without rows behind it do not.)
  const SeqRows s = find_rows(a.batch, row, 1, r.b, ordinal, [&](int first, int) { return first; });
  if (ordinal < 0 || ordinal >= s.rows) {
    r.token = r.pages = -1;
    return r;
  }
  r.token = a.causal ? min(s.first + ordinal, s.len - 1) : s.len - 1;
  r.pages = r.token < 0 ? 0 : (r.token >> a.cache.page_shift) + 1;
  return r;
}

// Whole numbers that order as the scores do (-0 is 0, NaN is -infinity).  A page that is
// not in the cache has key 0, which no score has.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == x ? x + 0.0f : -INFINITY);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kColumns = 16;             // query heads of one product

// Query heads in 8 bits: head x's element e at codes[x][e].
template <int D>
struct QueryCodes {
  int8_t codes[kColumns][D];
  float unit[kColumns];
};

// A lane's elements of a query head.
template <int D>
struct QueryLane {
  static constexpr int kEach = D / 64;
  uint32_t w[(kEach + 1) / 2];

  __device__ __forceinline__ void load(const SelectArgs& a, int row, int head) {
    const uint16_t* src = a.q + (int64_t)row * a.ldq + (int64_t)head * D + (threadIdx.x & 63) * kEach;
    if constexpr (kEach == 1) w[0] = src[0];
    else if constexpr (kEach == 2) w[0] = *reinterpret_cast<const uint32_t*>(src);
    else *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(src);
  }
};

// A query head, by a whole wave, into column x.  127 v / top is rounded as the exact
// quotient is: both have 8 significant bits, so it is a half (then it is representable, and
// the correction finds it) or further from one than 2^-17 of itself; the quotient is off by
// 2^-23 at most.  (Elements over 2^e, the top's power of two, keep within range.)
// A head that is not finite has a unit of NaN: so have its products, and a maximum passes
// them over.
template <int D>
__device__ __forceinline__ void query_codes(const QueryLane<D>& lanes, int x, QueryCodes<D>& to) {
  constexpr int kEach = D / 64;
  const int lane = threadIdx.x & 63;
  float v[kEach], top = 0.0f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) v[i] = i & 1 ? bf16_high(lanes.w[i / 2]) : bf16_low(lanes.w[i / 2]);
  bool finite = true;
#pragma unroll
  for (int i = 0; i < kEach; ++i) finite = finite && fabsf(v[i]) < INFINITY;
  finite = __all(finite);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = finite ? v[i] : 0.0f;
    top = fmaxf(top, fabsf(v[i]));
  }
  top = row_max(top);
  top = over_quarters_max(top);
  const int e = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
  const float over = top > 0.0f ? __builtin_amdgcn_ldexpf(top, -e) : 1.0f, inv = 1.0f / over;
  int8_t n[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const float y = __builtin_amdgcn_ldexpf(v[i], -e) * 127.0f;      // (exact)
    float q = y * inv;
    q = fmaf(fmaf(-q, over, y), inv, q);
    n[i] = (int8_t)(int)rintf(q);
  }
  if constexpr (kEach == 1) to.codes[x][lane] = n[0];
  else if constexpr (kEach == 2) *reinterpret_cast<char2*>(&to.codes[x][2 * lane]) = make_char2(n[0], n[1]);
  else *reinterpret_cast<char4*>(&to.codes[x][4 * lane]) = make_char4(n[0], n[1], n[2], n[3]);
  if (lane == 0) to.unit[x] = finite ? top / 127.0f : NAN;
}

// Scores of 16 pages at a time for up to 16 query heads.  Bounds are loaded as they lie,
// a kilobyte an instruction, and turned in LDS into the product's operands, a page to a lane
// of 16 (loaded as operands, 16 pages for 16 lanes, 8 times 2048 pages took 25.2 us in one
// compute unit each; so 18.2).  Pieces of 16 bytes change places by their page's number, so that 16 lanes
// meet 16 different bank groups.
template <int D>
struct Scorer {
  static constexpr int kSteps = D / 64, kChunks = D / 8, kLoads = D / 32;      // pieces of a page; loads of 16 pages
  static constexpr int kHalves = D == 256 ? 2 : 1, kPart = kChunks / kHalves;  // what is turned at a time
  typedef i32x4 Turn[16 * kPart];          // LDS of a wave
  i32x4 above[kSteps], below[kSteps];      // max(q, 0), min(q, 0): head lane % 16, elements 64 s + 16 (lane / 16) .. + 15
  float unit;

  // (Columns behind the n heads take the last one.)
  __device__ __forceinline__ void start(const QueryCodes<D>& q, int n) {
    const int lane = threadIdx.x & 63, col = min(lane & 15, n - 1), quarter = lane >> 4;
    unit = q.unit[col];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const i32x4 w = *reinterpret_cast<const i32x4*>(&q.codes[col][64 * s + 16 * quarter]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t negative = (((uint32_t)w[i] >> 7) & 0x01010101u) * 255u;
        below[s][i] = (int)((uint32_t)w[i] & negative);
        above[s][i] = (int)((uint32_t)w[i] & ~negative);
      }
    }
  }

  struct Round {
    i32x4 raw[kLoads];
    float step;
    int page;                              // of lane % 16 (-1: none)
  };

  static __device__ __forceinline__ int owner(int i) { return (64 / kChunks) * i + (int)(threadIdx.x & 63) / kChunks; }
  static __device__ __forceinline__ int place(int page, int chunk) {
    return page * kPart + (chunk ^ (D == 64 ? page >> 1 : page));
  }

  static __device__ __forceinline__ void load(const SelectArgs& a, int h, int page, Round& to) {
    const int chunk = (threadIdx.x & 63) % kChunks;
    const uint32_t mine = (uint32_t)max(page, 0);
    to.page = page;
    to.step = (a.bounds.step + h)[(uint64_t)mine * (uint32_t)a.bounds.step_stride];
    const int8_t* const at = a.bounds.codes + h * 2 * D + chunk * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)      // (strides below 2^31: one product each)
      to.raw[i] = *reinterpret_cast<const i32x4*>(at + (uint64_t)(uint32_t)__shfl((int)mine, owner(i)) * (uint32_t)a.bounds.page_stride);
  }

  // The page of 16 whose key a lane of columns 0 to 3 gets.
  static __device__ __forceinline__ int of_lane() {
    const int lane = threadIdx.x & 63;
    return 4 * (lane >> 4) + 2 * (lane & 1) + (lane >> 1 & 1);
  }

  // Its key.
  __device__ __forceinline__ uint32_t key(const Round& p, Turn& turn) const {
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4, chunk = lane % kChunks;
    i32x4 sum = (i32x4){0, 0, 0, 0};
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (kHalves == 1 || chunk / kPart == half) turn[place(owner(i), chunk % kPart)] = p.raw[i];
      wave_sees_lds();
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (kHalves == 1 || half == 0)
          sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(turn[place(col, 4 * s + quarter)], above[s], sum, 0, 0, 0);
        if (kHalves == 1 || half == 1)
          sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(turn[place(col, (kHalves == 1 ? D / 16 : 0) + 4 * s + quarter)], below[s], sum,
                                                      0, 0, 0);
      }
      wave_sees_lds();
    }
    // Pages 4 quarter + e of head col: the largest over the heads, of page 4 quarter + 2
    // (col % 2) + col / 2 % 2 (a lane gives away half of its pages, twice).
    const bool odd = col & 1, high = col & 2;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)sum[e] * unit;
    const float a0 = other_max<0xB1>(odd ? v[2] : v[0], odd ? v[0] : v[2]), a1 = other_max<0xB1>(odd ? v[3] : v[1], odd ? v[1] : v[3]);
    float m = other_max<0x4E>(high ? a1 : a0, high ? a0 : a1);
    m = other_max<0x124>(m, m);
    m = other_max<0x128>(m, m);
    const int mine = of_lane();
    const float step = __shfl(p.step, mine);
    return __shfl(p.page, mine) < 0 ? 0u : key_of(m * step);
  }
};

// Table entry j, of those in [first, end) (another's where it is not), and its page: -1 where it
// is not among them or not in the cache.  (No branch around the load, nor a store to memory
// in a loop that has it: the compiler would wait for all that may be on its way.)
__device__ __forceinline__ int entry_at(const int32_t* table, int j, int first, int end) {
  return table[min(max(j, first), end - 1)];
}

__device__ __forceinline__ int page_of(const SelectArgs& a, int entry, int j, int first, int end) {
  return j >= first && j < end && entry < a.cache.num_pages ? entry : -1;
}

// The scores of one row and key head's pages j0 + 16 wave .. by rounds of 16 pages a wave
// up to j1; put(j, key) from the lanes that hold them.
template <int D, int kWaves, typename Put>
__device__ __forceinline__ void score_pages(const SelectArgs& a, const QueryCodes<D>& q, int heads, int h, const int32_t* table, int first,
                                            int end, int j0, int j1, typename Scorer<D>::Turn* turns, Put put) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = threadIdx.x & 15;
  Scorer<D> scorer;
  scorer.start(q, heads);
  int j = j0 + 16 * wave;
  // Two rounds' bounds ahead (heads of 256: one, none in 16 waves; registers).  A round's entries are
  // loaded before the bounds of the round in front of it, and looked at a round later: loads are
  // waited for in order.
  constexpr int kAhead = D == 256 ? (kWaves > 4 ? 0 : 1) : 2, kRounds = kAhead + 1, kRound = 16 * kWaves;
  typename Scorer<D>::Round p[kRounds];
  int entry[kRounds];
#pragma unroll
  for (int x = 0; x < kRounds; ++x) entry[x] = entry_at(table, j + x * kRound + col, first, end);
#pragma unroll
  for (int x = 0; x < kAhead; ++x) Scorer<D>::load(a, h, page_of(a, entry[x], j + x * kRound + col, first, end), p[x]);
  int ahead = entry[kAhead];
  const auto round = [&](auto at) __attribute__((always_inline)) {
    constexpr int x = decltype(at)::value;
    if (j >= j1) return false;
    const int behind = entry_at(table, j + kRounds * kRound + col, first, end);
    Scorer<D>::load(a, h, page_of(a, ahead, j + kAhead * kRound + col, first, end), p[(x + kAhead) % kRounds]);
    const uint32_t key = scorer.key(p[x], turns[wave]);
    const int mine = j + Scorer<D>::of_lane();
    if (col < 4 && mine >= first && mine < end) put(mine, key);
    ahead = behind;
    j += kRound;
    return true;
  };
  // A round by the name of its registers: copied, they would be waited for.
  while (round(std::integral_constant<int, 0>{}) && (kRounds < 2 || round(std::integral_constant<int, 1 % kRounds>{})) &&
         (kRounds < 3 || round(std::integral_constant<int, 2 % kRounds>{}))) {}
}

// ---------------------------------------------------------------- selection

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048, kBinBits = 11;
constexpr int kHeldKeys = 8192;          // keys of a row and key head in LDS

struct SelectLds {
  int counts[2][kBins];
  int totals[2][kHeldKeys / kSelectThreads][kSelectWaves];      // of every round and wave
  uint32_t ends[2][kSelectWaves];
  int sums[kSelectWaves];
  int found[3];
};

// What is taken of n keys: those from `cut` on, and the first `ties` of those that are
// cut - 1 (64 bits, so that there is one behind the largest).
struct Cut {
  uint64_t cut;
  int ties;
};

// The want largest of key(0) .. key(n - 1) (1 <= want < n).  Their smallest is found in the
// counts of 2048 equal steps from the smallest to the largest key, then in those of
// the step that holds it: two or three times for any 32 bits, once for most.
template <typename Key>
__device__ __forceinline__ Cut find_cut(SelectLds& lds, int n, int want, Key key) {
  static_assert(kSelectWaves == 16 && kBins == 2 * kSelectThreads, "a wave for each lane of a row, two steps a thread");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15;
  const auto clear = [&](int which) {
    *reinterpret_cast<int2*>(&lds.counts[which][2 * threadIdx.x]) = make_int2(0, 0);
  };
  uint32_t lo = ~0u, hi = 0;
  for (int i = threadIdx.x; i < n; i += kSelectThreads) {
    const uint32_t k = key(i);
    lo = min(lo, k), hi = max(hi, k);
  }
  clear(0);
  lo = over_quarters_low(row_low(lo));
  hi = ~over_quarters_low(row_low(~hi));
  if (lane == 0) lds.ends[0][wave] = lo, lds.ends[1][wave] = hi;
  __syncthreads();
  lo = row_low(lds.ends[0][col]);
  hi = row_high(lds.ends[1][col]);
  int left = want;
  for (int level = 0;; level ^= 1) {
    const uint32_t range = hi - lo;
    if (range == 0) return {(uint64_t)lo + 1, left};
    const int shift = max(0, 32 - __builtin_clz(range) - kBinBits);
    for (int i = threadIdx.x; i < n; i += kSelectThreads) {
      const uint32_t k = key(i);
      if (k >= lo && k <= hi) atomicAdd(&lds.counts[level][(k - lo) >> shift], 1);      // (whole numbers: any order)
    }
    clear(level ^ 1);      // (last read before the last level's end)
    __syncthreads();
    // The largest step with at least `left` keys at or above it; a thread has two of them.
    const int top = kBins - 1 - 2 * (int)threadIdx.x;
    const int first = lds.counts[level][top], second = lds.counts[level][top - 1], up = scan_up(first + second);
    if (lane == 63) lds.sums[wave] = up;
    __syncthreads();
    const int above = row_sum(col < wave ? lds.sums[col] : 0) + up - first - second;
    if (above < left && above + first + second >= left) {
      const bool of_first = above + first >= left;
      lds.found[0] = of_first ? top : top - 1;
      lds.found[1] = left - above - (of_first ? 0 : first);
      lds.found[2] = of_first ? first : second;
    }
    __syncthreads();
    const uint32_t from = lo + ((uint32_t)lds.found[0] << shift);
    left = lds.found[1];
    if (shift == 0) return {(uint64_t)from + 1, left};
    if (left == lds.found[2]) return {from, 0};                   // all of the step
    lo = from;
    if (hi - lo >= 1u << shift) hi = lo + ((1u << shift) - 1);
  }
}

// The positions of the taken ones among all n, in order: put(position, i).
template <typename Key, typename Put>
__device__ __forceinline__ void put_taken(SelectLds& lds, int n, const Cut& c, Key key, Put put) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned long long below = (1ull << lane) - 1;
  int taken = 0, equal = 0;      // before these rounds
  constexpr int kRounds = kHeldKeys / kSelectThreads;
  for (int i0 = 0; i0 < n; i0 += kHeldKeys) {
    unsigned long long above_of[kRounds], same_of[kRounds];
#pragma unroll
    for (int x = 0; x < kRounds; ++x) {
      const int i = i0 + x * kSelectThreads + threadIdx.x;
      const uint32_t k = i < n ? key(i) : 0;
      above_of[x] = __ballot(i < n && k >= c.cut);
      same_of[x] = __ballot(i < n && c.ties > 0 && (uint64_t)k + 1 == c.cut);
      if (lane == 0) lds.totals[0][x][wave] = __popcll(above_of[x]), lds.totals[1][x][wave] = __popcll(same_of[x]);
    }
    __syncthreads();
    if (wave < 2) {      // sums of what is before each round and wave
      constexpr int kAll = kRounds * kSelectWaves, kEach = kAll / 64;
      int* const t = &lds.totals[wave][0][0] + kEach * lane;
      int sum = 0, mine[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) mine[i] = t[i], sum += mine[i];
      int before = scan_up(sum) - sum;
      if (lane == 63) lds.found[wave] = before + sum;
#pragma unroll
      for (int i = 0; i < kEach; ++i) t[i] = before, before += mine[i];
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kRounds; ++x) {
      const bool above = (above_of[x] >> lane) & 1, same = (same_of[x] >> lane) & 1;
      const int ties = equal + lds.totals[1][x][wave] + __popcll(same_of[x] & below);
      const int at = taken + lds.totals[0][x][wave] + __popcll(above_of[x] & below) + min(ties, c.ties);
      if (above || (same && ties < c.ties)) put(at, i0 + x * kSelectThreads + threadIdx.x);
    }
    taken += lds.found[0];
    equal += lds.found[1];
    __syncthreads();
  }
}

// The choice of a row and key head, by its scores.  ready(): where they are not needed (all
// pages are taken) this is the whole of it.
struct Chosen {
  int32_t *index, *pages;
  const int32_t* table;

  __device__ __forceinline__ void put(int at, int entry) const { put(at, entry, table[entry]); }
  __device__ __forceinline__ void put(int at, int entry, int page) const {
    index[at] = entry;
    pages[at] = page;
  }
};

// What does not hang on scores; whether that is all.
__device__ __forceinline__ bool choose_without(const SelectArgs& a, const RowPages& r, int row, int h, Chosen& to) {
  const int shift = a.cache.page_shift;
  if (h == 0 && threadIdx.x == 0) {
    const int taken = min(r.pages, a.count);
    a.tokens[row] = r.pages <= 0 ? r.pages : ((taken - 1) << shift) + (r.token & ((1 << shift) - 1)) + 1;
  }
  if (r.pages < 0) return true;
  const int64_t at = ((int64_t)row * a.cache.heads + h) * a.count;
  to = {a.index + at, a.pages + at, a.batch.table + (int64_t)r.b * a.batch.table_stride};
  if (r.pages <= a.count) {
    for (int i = threadIdx.x; i < a.count; i += kSelectThreads) {
      if (i < r.pages) to.put(i, i);
      else to.put(i, -1, -1);
    }
    return true;
  }
  for (int i = threadIdx.x; i < a.first; i += kSelectThreads) to.put(i, i);
  const int end = r.pages - a.recent;
  for (int i = threadIdx.x; i < a.recent; i += kSelectThreads) to.put(a.count - a.recent + i, end + i);
  return a.count == a.first + a.recent;
}

// One workgroup for each row and key head: scores and choice.
template <int D>
__global__ __launch_bounds__(kSelectThreads) void kv_choose_kernel(SelectArgs a) {
  __shared__ QueryCodes<D> codes;
  __shared__ SelectLds lds;
  __shared__ uint32_t keys[kHeldKeys];
  __shared__ typename Scorer<D>::Turn turns[kSelectWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = (int)(blockIdx.x % a.cache.heads), row = (int)(blockIdx.x / a.cache.heads);
  QueryLane<D> query;
  query.load(a, row, h * a.group + min(wave, a.group - 1));
  const RowPages r = row_pages(a, row);
  Chosen to;
  if (choose_without(a, r, row, h, to)) return;
  const int first = a.first, end = r.pages - a.recent, n = end - first;
  for (int a0 = 0; a0 < a.group; a0 += kColumns) {
    const int heads = min(a.group - a0, kColumns);
    if (a0 > 0) query.load(a, row, h * a.group + a0 + min(wave, heads - 1));
    if (wave < heads) query_codes<D>(query, wave, codes);
    __syncthreads();
    score_pages<D, kSelectWaves>(a, codes, heads, h, to.table, first, end, first & ~15, end, turns, [&](int j, uint32_t key) {
      keys[j - first] = a0 == 0 ? key : max(keys[j - first], key);
    });
    __syncthreads();
  }
  const auto key = [&](int i) { return keys[i]; };
  const Cut c = find_cut(lds, n, a.count - a.first - a.recent, key);
  put_taken(lds, n, c, key, [&](int at, int i) { to.put(first + at, first + i); });
}

// The same in two launches, for few rows of long sequences: the scores, a workgroup for
// `each` pages, and the choice.
constexpr int kScoreWaves = 4, kScorePages = 1024;

template <int D>
__global__ __launch_bounds__(64 * kScoreWaves) void kv_page_scores_kernel(SelectArgs a, int chunks, int each) {
  __shared__ QueryCodes<D> codes;
  __shared__ uint32_t keys[kScorePages];
  __shared__ typename Scorer<D>::Turn turns[kScoreWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = blockIdx.x;
  const int h = id % a.cache.heads;
  id /= a.cache.heads;
  const int row = id / chunks, chunk = id % chunks;
  constexpr int kMine = kColumns / kScoreWaves;
  QueryLane<D> query[kMine];
  const auto load = [&](int a0) {
#pragma unroll
    for (int x = 0; x < kMine; ++x) query[x].load(a, row, h * a.group + min(a0 + x * kScoreWaves + wave, a.group - 1));
  };
  load(0);
  const RowPages r = row_pages(a, row);
  if (r.pages <= a.count) return;                                    // (all of them are taken)
  const int first = a.first, end = r.pages - a.recent;
  const int j0 = chunk * each, j1 = min(end, j0 + each);
  if (j0 >= j1) return;
  const int32_t* const table = a.batch.table + (int64_t)r.b * a.batch.table_stride;
  for (int a0 = 0; a0 < a.group; a0 += kColumns) {
    const int heads = min(a.group - a0, kColumns);
    if (a0 > 0) load(a0);
#pragma unroll
    for (int x = 0; x < kMine; ++x)
      if (x * kScoreWaves + wave < heads) query_codes<D>(query[x], x * kScoreWaves + wave, codes);
    __syncthreads();
    score_pages<D, kScoreWaves>(a, codes, heads, h, table, first, end, j0, j1, turns, [&](int j, uint32_t key) {
      keys[j - j0] = a0 == 0 ? key : max(keys[j - j0], key);
    });
    __syncthreads();
  }
  uint32_t* const scores = a.scores + ((int64_t)row * a.cache.heads + h) * a.max_pages;
  for (int j = max(first, j0) + threadIdx.x; j < j1; j += 64 * kScoreWaves) scores[j] = keys[j - j0];
}

template <bool kHeld>
__global__ __launch_bounds__(kSelectThreads) void kv_select_kernel(SelectArgs a) {
  __shared__ SelectLds lds;
  __shared__ uint32_t keys[kHeld ? kHeldKeys : 1];
  const int h = (int)(blockIdx.x % a.cache.heads), row = (int)(blockIdx.x / a.cache.heads);
  const RowPages r = row_pages(a, row);
  Chosen to;
  if (choose_without(a, r, row, h, to)) return;
  const int first = a.first, n = r.pages - a.recent - first;
  const uint32_t* const scores = a.scores + ((int64_t)row * a.cache.heads + h) * a.max_pages + first;
  if (kHeld) {
    for (int i = threadIdx.x; i < n; i += kSelectThreads) keys[i] = scores[i];      // (read by the thread that writes it)
  }
  const auto key = [&](int i) { return kHeld ? keys[i] : scores[i]; };
  const Cut c = find_cut(lds, n, a.count - a.first - a.recent, key);
  put_taken(lds, n, c, key, [&](int at, int i) { to.put(first + at, first + i); });
}

namespace {

// Pages of a workgroup that only scores: so that there are up to eight for each compute unit.
// (By the table's width: 32 rows of 2000 tokens, 8 key heads, take 9.6 us with 8192 pages, 14.2 with
// 8193, in two launches, and 27.2 with 65536.)
int score_each(const SelectArgs& a) {
  const int64_t work = (int64_t)a.batch.rows * a.cache.heads * ((a.max_pages + 63) / 64);      // of 64 pages
  const int64_t n = (work + 2047) / 2048;
  return (int)(n < 1 ? 1 : n < kScorePages / 64 ? n : kScorePages / 64) * 64;
}

// One launch or two: one where there is a row and key head for each compute unit, or
// little for one to do.  In one and in two (us; rows x key heads, largest table):
//   8, 126   7.8  9.2     26, 627 (heads of 256)   14.6 10.8     32, 1001   12.7 11.3
//   8, 2049 16.9 11.2     64, 2001 (64)            13.8 14.4     128, 1876  18.2 17.5
//   256, 2049 22.9 25.9   504, 501                 20.2 22.2     496, 126   16.0 15.2
// (A unit holds one workgroup of the one launch, so 257 and more take a second round: 264 of 2049
// 36 us, of 4000 55, where 248 take 27 and 38 in two.)
bool choose_at_once(const SelectArgs& a) {
  return a.max_pages <= 256 || (a.max_pages <= kHeldKeys && (int64_t)a.batch.rows * a.cache.heads >= 256);
}

// Whether a launch of its own scores pages: not where all are taken.
bool scores_apart(const SelectArgs& a) {
  return !choose_at_once(a) && a.max_pages > a.count && a.count > a.first + a.recent;
}

template <int D>
hipError_t launch_scores(const SelectArgs& a, hipStream_t stream) {
  const int each = score_each(a), chunks = (a.max_pages + each - 1) / each;
  kv_page_scores_kernel<D><<<dim3((unsigned)((int64_t)a.batch.rows * a.cache.heads * chunks)), 64 * kScoreWaves, 0, stream>>>(
      a, chunks, each);
  return hipGetLastError();
}

}  // namespace

size_t kv_select_workspace_bytes(const SelectArgs& a) {
  return choose_at_once(a) ? 0 : (size_t)((int64_t)a.batch.rows * a.cache.heads * a.max_pages) * sizeof(uint32_t);
}

bool select_fits(const SelectArgs& a) {
  const int64_t work = (int64_t)a.batch.rows * a.cache.heads;
  if (!one_grid(work, kSelectThreads)) return false;
  const int each = score_each(a);
  return !scores_apart(a) || one_grid(work * ((a.max_pages + each - 1) / each), 64 * kScoreWaves);
}

hipError_t launch_kv_select(const SelectArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)a.batch.rows * a.cache.heads));
  if (choose_at_once(a)) {
    if (a.cache.dim == 64) kv_choose_kernel<64><<<grid, kSelectThreads, 0, stream>>>(a);
    else if (a.cache.dim == 128) kv_choose_kernel<128><<<grid, kSelectThreads, 0, stream>>>(a);
    else kv_choose_kernel<256><<<grid, kSelectThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  if (scores_apart(a)) {
    const hipError_t e = a.cache.dim == 64    ? launch_scores<64>(a, stream)
                         : a.cache.dim == 128 ? launch_scores<128>(a, stream)
                                              : launch_scores<256>(a, stream);
    if (e != hipSuccess) return e;
  }
  if (a.max_pages <= kHeldKeys) kv_select_kernel<true><<<grid, kSelectThreads, 0, stream>>>(a);
  else kv_select_kernel<false><<<grid, kSelectThreads, 0, stream>>>(a);
  return hipGetLastError();
}

// Pages that a step may complete: for sequence b, at most those that its rows'
// numbers reach into.
int64_t bounds_items(const KvBatchArgs& b, int page_shift) {
  return b.cu_rows == nullptr ? b.seqs : (b.rows >> page_shift) + (int64_t)b.seqs;
}

bool bounds_fit(const BoundsArgs& a) {
  return one_grid((bounds_items(a.batch, a.cache.page_shift) * a.cache.heads + 3) / 4, 256);
}

hipError_t launch_kv_page_bounds(const BoundsArgs& a, hipStream_t stream) {
  const int64_t items = bounds_items(a.batch, a.cache.page_shift);
  const dim3 grid((unsigned)((items * a.cache.heads + 3) / 4));
  if (a.cache.dim == 64)
    kv_page_bounds_kernel<64><<<grid, 256, 0, stream>>>(a, (int)items);
  else if (a.cache.dim == 128)
    kv_page_bounds_kernel<128><<<grid, 256, 0, stream>>>(a, (int)items);
  else
    kv_page_bounds_kernel<256><<<grid, 256, 0, stream>>>(a, (int)items);
  return hipGetLastError();
}

}  // namespace nvfp4
