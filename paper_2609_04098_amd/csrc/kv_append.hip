// Append of keys and values to the paged E4M3 cache, keys normed and rotated on
// the way, for gfx950 (layout: nvfp4_attention.h).
//
// Many rows: one workgroup for each touched page and some of the heads, one head's
// keys or values after the other.  It holds their new tokens (8 or 16 elements
// a lane, so 256 to 1024 threads by the page's size) in registers between the
// maximum and the rounding, with the next ones' loads in flight, so the input is
// read once, no workgroup waits for another and the result does not depend on
// any order.  The tokens' sines and cosines are computed once for all heads; their
// table bounds a compute unit to 16 waves.  Codes go through LDS into the
// cache's order and leave it in 16-byte pieces.
// Bound by the issue of vector instructions, 115 for 8 keys and 45 for 8 values a
// lane: 16000 tokens of 8 heads of 128 take 28 us, 18 of them issue, where the bytes
// would take 19.  (Pages of 16384 elements with 64 elements a lane, four waves to a
// compute unit: 74 us; with 16 a lane 31.)
// Few rows (under 5 for a sequence): four waves for each touched page, keys or
// values, and as many heads as a wave has lanes for (512 / D), a token at a time
// each; the codes are stored from registers.  (The rule and both sides' times:
// attention_plan.h.)
//
// Keys are computed in binary64: an 8-bit rounding turns the last bit of a
// binary32 value that is next to a border into a step of 6 to 12 %, and binary64
// products issue at the rate of binary32 ones here.  A value reaches the rounding
// as a binary32 number whose rounding to E4M3 is that of the value itself
// (values()); a power-of-two scale does not change that.  (In binary32, with the
// codes of the value less and plus its error compared and waves computed again
// where they differ, the same took 123 us.  With the partners of the rotation
// fetched by lane moves instead of LDS shuffles, 29.6 us.)
#include "attention_device.h"
#include "attention_plan.h"

namespace nvfp4 {

constexpr float kLargest = 3.40282347e38f;

// The binary32 number next to d towards zero, with its last bit set unless it
// is d itself: rounds to E4M3 as d does, also after a division by a power of two.
__device__ __forceinline__ float sticky(double d) {
  const float f = (float)d;
  const double back = (double)f;
  uint32_t b = __float_as_uint(f);
  if (back != d) b = (fabs(back) > fabs(d) ? b - 1 : b) | 1u;
  return __uint_as_float(b);
}

// The smallest power of two s >= 2^-100 with a <= 448 s (448 = 1.75 * 2^8).
__device__ __forceinline__ float page_scale(float a) {
  const uint32_t b = __float_as_uint(a);
  const int k = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(k, -100) + 127) << 23);
}

__device__ __forceinline__ double shfl_f64(double v, int l) {
  const int lo = __shfl(__double2loint(v), l), hi = __shfl(__double2hiint(v), l);
  return __hiloint2double(hi, lo);
}

// Another lane's value within the row of 16 (all lanes active): from lane ^ 1,
// ^ 2, ^ 7, ^ 15 for step 1, 2, 4, 8.  After the steps before, whose sums or
// maxima groups of that many lanes share, ^ 7 and ^ 15 are as good as ^ 4 and ^ 8.
template <int kStep>
__device__ __forceinline__ int of_other(int v) {
  constexpr int kHow = kStep == 1 ? 0xB1 : kStep == 2 ? 0x4E : kStep == 4 ? 0x141 : 0x140;
  return __builtin_amdgcn_update_dpp(0, v, kHow, 0xF, 0xF, true);
}

template <int kStep>
__device__ __forceinline__ double of_other(double v) {
  return __hiloint2double(of_other<kStep>(__double2hiint(v)), of_other<kStep>(__double2loint(v)));
}

// The sum over the kLanes (8, 16 or 32) lanes that hold a token.
template <int kLanes>
__device__ __forceinline__ double sum_over(double v) {
  v += of_other<1>(v);
  v += of_other<2>(v);
  v += of_other<4>(v);
  if (kLanes >= 16) v += of_other<8>(v);
  if (kLanes >= 32) {
    const auto lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    v = __hiloint2double((int)hi[0], (int)lo[0]) + __hiloint2double((int)hi[1], (int)lo[1]);
  }
  return v;
}

// The maximum over the wave.
__device__ __forceinline__ float wave_max_of(float v) {
  v = fmaxf(v, __int_as_float(of_other<1>(__float_as_int(v))));
  v = fmaxf(v, __int_as_float(of_other<2>(__float_as_int(v))));
  v = fmaxf(v, __int_as_float(of_other<4>(__float_as_int(v))));
  v = fmaxf(v, __int_as_float(of_other<8>(__float_as_int(v))));
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Four codes times the ratio of the old scale to the new one.
__device__ __forceinline__ uint32_t rescaled(uint32_t codes, float ratio) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return e4m3_codes(lo.x * ratio, lo.y * ratio, hi.x * ratio, hi.y * ratio);
}

// What a lane does to its 8 elements e0 .. e0 + 7 of a head held by D / 8 lanes.
struct Treatment {
  bool norm, rotate;             // keys only
  bool turned;                   // these elements are among the rotated ones
  bool interleaved;
  int half, e0, partner;         // the lane that holds the other elements of the pairs
  uint32_t flip;                 // split halves: sign bit where the partner counts negative
  double gamma[8];
  float eps;
};

template <int D>
__device__ __forceinline__ Treatment treatment(const AppendArgs& a, int kind) {
  Treatment t;
  const int lane = threadIdx.x & 63;
  t.half = a.rope.rot / 2;
  t.e0 = (lane % (D / 8)) * 8;
  t.norm = kind == 0 && a.gamma != nullptr;
  t.rotate = kind == 0 && t.half > 0;
  t.turned = t.rotate && t.e0 < a.rope.rot;
  t.interleaved = a.rope.interleaved;
  t.partner = lane;
  if (t.turned && !t.interleaved) t.partner = lane + (t.e0 < t.half ? t.half / 8 : -(t.half / 8));
  t.flip = t.e0 < t.half ? 0x80000000u : 0u;
  uint4 gamma = make_uint4(0, 0, 0, 0);
  if (t.norm) gamma = *reinterpret_cast<const uint4*>(a.gamma + t.e0);
  const uint32_t g[4] = {gamma.x, gamma.y, gamma.z, gamma.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) t.gamma[2 * j] = (double)bf16_low(g[j]), t.gamma[2 * j + 1] = (double)bf16_high(g[j]);
  t.eps = a.eps;
  return t;
}

// Place of angle f in a token's table: neighbouring lanes, which want f and f + 8,
// read neighbouring places.
__device__ __forceinline__ int turn_at(int half, int f) { return (f & 7) * (half >> 3) + (f >> 3); }

__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 1 / sqrt(x), to a few last bits: v_rsq_f64 and two Newton steps.
__device__ __forceinline__ double reciprocal_root(double x) {
  double r = __builtin_amdgcn_rsq(x);
  const double h = -0.5 * x;
  r *= fma(h * r, r, 1.5);
  r *= fma(h * r, r, 1.5);
  return r;
}

// The lane's 8 values, ready for rounding.  turn: cosines and sines of the
// token's angles.  All lanes of the wave call it.
// The binary32 number next to a value rounds to E4M3 as the value itself does,
// and is over 448 scales where it is, unless it is a border itself, halfway
// between two codes or 448 scales: then its last 19 bits are zero (5 significant
// bits; scales are powers of two), and the wave takes the sticky ones.
template <int D, bool kDynamic>
__device__ __forceinline__ void values(const Treatment& t, uint4 in, const double2* turn, float (&v)[8]) {
  const uint32_t d[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) v[2 * j] = bf16_low(d[j]), v[2 * j + 1] = bf16_high(d[j]);
  if (!t.norm && !t.rotate) return;
  double w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = (double)v[j];
  if (t.norm) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fma(w[j], w[j], sum);
    const double r = reciprocal_root(sum_over<D / 8>(sum) * (1.0 / D) + (double)t.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] *= r * t.gamma[j];
  }
  if (t.rotate && t.interleaved) {
    if (t.turned) {
      const double2* at = turn + turn_at(t.half, t.e0 / 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const double2 cs = at[j * (t.half >> 3)];
        const double x = w[2 * j], y = w[2 * j + 1];
        w[2 * j] = fma(x, cs.x, -(y * cs.y));
        w[2 * j + 1] = fma(y, cs.x, x * cs.y);
      }
    }
  } else if (t.rotate) {
    double p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = shfl_f64(w[j], t.partner);
    if (t.turned) {
      const double2* at = turn + turn_at(t.half, t.e0 < t.half ? t.e0 : t.e0 - t.half);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double2 cs = at[j * (t.half >> 3)];
        const double other = __hiloint2double(__double2hiint(p[j]) ^ (int)t.flip, __double2loint(p[j]));
        w[j] = fma(w[j], cs.x, other * cs.y);
      }
    }
  }
  uint32_t border = ~0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = (float)w[j];
    border = min(border, __float_as_uint(v[j]) & 0x7FFFFu);
  }
  if (!kDynamic || __any(border == 0)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = sticky(w[j]);
  }
}

// Codes of 8 values over the scale.  In dynamic mode none is over 448 scales and
// 1 / scale is exact; in static mode a quotient over 448 is cut, and rounded
// once.  Values that are not finite give NaN.
template <bool kDynamic>
__device__ __forceinline__ uint2 eight_codes(const float (&v)[8], float scale, float inverse) {
  float q[8];
  if (kDynamic) {
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = v[j] * inverse;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = sticky((double)v[j] / (double)scale);
      q[j] = fabsf(v[j]) <= kLargest ? __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f) : __uint_as_float(0x7FC00000u);
    }
  }
  return make_uint2(e4m3_codes(q[0], q[1], q[2], q[3]), e4m3_codes(q[4], q[5], q[6], q[7]));
}

// The largest |v| of 8 values (all: without those that are not finite).
__device__ __forceinline__ float largest(const float (&v)[8], float top, bool all) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float m = fabsf(v[j]);
    top = fmaxf(top, all || m <= kLargest ? m : 0.0f);
  }
  return top;
}

// The page that a workgroup or wave writes to, and which of the step's tokens.
struct Touch {
  int page;
  int n, slot0, row0, token0;      // tokens, first slot, first row, first token's number
};

// Item of the step: sequence b's pages have the numbers from
// cu_rows[b] / page_size + 2 b on (n rows reach (n - 1) / page_size + 2 pages).
__device__ __forceinline__ bool find_touch(const AppendArgs& a, int item, Touch& t) {
  const int shift = a.cache.page_shift;
  int b, ordinal;
  const SeqRows s =
      find_rows(a.batch, item, 1, b, ordinal, [&](int row, int x) { return (row >> shift) + 2 * x; });
  const int begin = max(s.first, 0), entry = (begin >> shift) + ordinal;
  if (ordinal < 0 || entry >= (a.batch.max_tokens >> shift)) return false;
  const int t0 = max(begin, entry << shift), t1 = min(s.len, (entry + 1) << shift);
  if (t0 >= t1) return false;
  t.page = a.batch.table[(int64_t)b * a.batch.table_stride + entry];
  t.n = t1 - t0;
  t.slot0 = t0 - (entry << shift);
  t.row0 = s.row + (t0 - s.first);
  t.token0 = t0;
  return t.page >= 0 && t.page < a.cache.num_pages;
}

__device__ __forceinline__ int position(const AppendArgs& a, const Touch& t, int i) {
  return a.rope.positions != nullptr ? a.rope.positions[t.row0 + i] : t.token0 + i;
}

// Held tokens (slots below slot0) of one page and head, brought to a grown
// scale: pieces start, start + step, ...
template <int D>
__device__ __forceinline__ void bring_along(uint8_t* out, int kind, int slot0, float ratio, int start, int step) {
  const int pieces = ((slot0 + 15) / 16) * D;
  for (int x = start; x < pieces; x += step) {
    const int group = x / D, in_group = x % D;
    uint4* at = reinterpret_cast<uint4*>(out) + x;
    // Of a piece of keys, one token; of values, four, held ones first.
    const int held = slot0 - (kind == 0 ? group * 16 + (in_group & 15) : group * 16 + ((in_group >> 4) & 3) * 4);
    if (held <= 0) continue;
    const uint32_t keep = kind == 0 || held >= 4 ? 0u : 0xFFFFFFFFu << (8 * held);
    const uint4 c = *at;
    *at = make_uint4((c.x & keep) | (rescaled(c.x, ratio) & ~keep), (c.y & keep) | (rescaled(c.y, ratio) & ~keep),
                     (c.z & keep) | (rescaled(c.z, ratio) & ~keep), (c.w & keep) | (rescaled(c.w, ratio) & ~keep));
  }
}

// A lane's 8 codes of the token in slot t into a page and head's bytes.
template <int D>
__device__ __forceinline__ void put_codes(uint8_t* out, int kind, int t, int e0, uint2 c) {
  const int base = (t / 16) * 16 * D, u = t % 16;
  if (kind == 0) {
    *reinterpret_cast<uint2*>(out + base + (e0 / 16) * 256 + u * 16 + (e0 & 8)) = c;
  } else {
    uint8_t* to = out + base + (e0 / 64) * 1024 + ((u / 4) * 16 + (e0 & 8)) * 16 + (e0 / 16 % 4) * 4 + u % 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j * 16] = (uint8_t)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
  }
}

// Codes of values, four tokens to a 32-bit word as the cache has them, from lanes
// that hold 8 elements of one token each.
//   D <= 128: bits 4 and 5 of the lane are the token's place in the four.  The lane
//   gets elements first, first + 1 of its 8, first = 4 (lane / 32) + 2 (lane / 16 % 2).
__device__ __forceinline__ uint2 fours(uint2 c) {
  const auto a = __builtin_amdgcn_permlane32_swap(c.x, c.y, false, false);      // tokens 0, 1 and 2, 3
  const uint32_t lo = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), hi = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
  const auto b = __builtin_amdgcn_permlane16_swap(lo, hi, false, false);        // 0 2 0 2 and 1 3 1 3
  return make_uint2(__builtin_amdgcn_perm(b[1], b[0], 0x05010400u), __builtin_amdgcn_perm(b[1], b[0], 0x07030602u));
}

//   D = 256: bit 5 is the place's low bit, and c0, c1 are two tokens.  The lane
//   gets elements first .. first + 3, first = 4 (lane / 32).
__device__ __forceinline__ uint4 fours(uint2 c0, uint2 c1) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_amdgcn_perm(c1.x, c0.x, 0x05010400u),
                                                  __builtin_amdgcn_perm(c1.y, c0.y, 0x05010400u), false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(__builtin_amdgcn_perm(c1.x, c0.x, 0x07030602u),
                                                  __builtin_amdgcn_perm(c1.y, c0.y, 0x07030602u), false, false);
  return make_uint4(__builtin_amdgcn_perm(a[1], a[0], 0x05010400u), __builtin_amdgcn_perm(a[1], a[0], 0x07030602u),
                    __builtin_amdgcn_perm(b[1], b[0], 0x05010400u), __builtin_amdgcn_perm(b[1], b[0], 0x07030602u));
}

// Place of a 16-byte piece of keys in LDS: the pieces of a token, 256 bytes apart
// in the cache's order, in different banks.
__device__ __forceinline__ int key_piece(int x) { return x ^ ((x >> 4) & 15); }

// Many rows.  kPasses * kThreads * 8 / D slots at most; heads_each heads a workgroup.
template <int D, int kThreads, int kPasses, bool kDynamic>
__global__ __launch_bounds__(kThreads, 4) void kv_append_pages_kernel(AppendArgs a, int heads_each) {
  constexpr int kLanes = D / 8, kTokens = kThreads / kLanes;        // of one pass
  __shared__ double2 turn[kPasses * kTokens][D / 2];
  __shared__ uint8_t __attribute__((aligned(16))) codes[kPasses * kTokens * D];
  __shared__ float wave_max[kThreads / 64];

  const int parts = (a.cache.heads + heads_each - 1) / heads_each;
  Touch t;
  if (!find_touch(a, (int)blockIdx.x / parts, t)) return;
  const int h0 = (int)blockIdx.x % parts * heads_each, h1 = min(h0 + heads_each, a.cache.heads);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Treatment for_keys = treatment<D>(a, 0);
  const int e0 = for_keys.e0, last = t.slot0 + t.n;
  // The slot of this lane's token in pass p, so that the four tokens of a word of
  // values are in lanes (or passes) that fours() joins; and whether the wave has some.
  const auto slot = [&](int p) __attribute__((always_inline)) {
    const int g = lane / kLanes;
    return D == 256 ? p / 2 * 2 * kTokens + wave * 4 + p % 2 * 2 + g
                    : p * kTokens + wave * (64 / kLanes) + (D == 64 ? (g & 1) * 4 + (g >> 1) : g);
  };
  const auto holds = [&](int p) __attribute__((always_inline)) {
    constexpr int kSpan = D == 256 ? 4 : 64 / kLanes;
    const int s0 = (D == 256 ? p / 2 * 2 : p) * kTokens + wave * kSpan;
    return s0 < last && s0 + kSpan > t.slot0;
  };

  uint4 in[kPasses];
  const auto load = [&](int h, int kind) __attribute__((always_inline)) {
    const int64_t ld = kind ? a.ld[1] : a.ld[0];
    const uint16_t* x = (kind ? a.x[1] : a.x[0]) + (int64_t)t.row0 * ld + (int64_t)h * D + e0;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int i = slot(p) - t.slot0;
      in[p] = make_uint4(0, 0, 0, 0);
      if (i >= 0 && i < t.n) in[p] = *reinterpret_cast<const uint4*>(x + i * ld);
    }
  };
  load(h0, 0);
  if (for_keys.rotate) {
    // A thread takes one angle of 8 tokens; where a token's position is the last
    // one's and 1, from that one's sine and cosine (4 operations instead of 50).
    const int runs = (t.n + 7) / 8;
    for (int x = threadIdx.x; x < runs * for_keys.half; x += kThreads) {
      const int run = x / for_keys.half, f = x - run * for_keys.half;
      const float freq = a.rope.inv_freq[f];
      double s, c, s1, c1;
      sin_cos<double>(1, freq, s1, c1);
      uint32_t before = 0;
      for (int i = 8 * run; i < min(8 * run + 8, t.n); ++i) {
        const int pos = position(a, t, i);
        if (i % 8 != 0 && (uint32_t)pos == before + 1) {
          const double c0 = c;
          c = fma(c0, c1, -(s * s1));
          s = fma(s, c1, c0 * s1);
        } else {
          sin_cos<double>(pos, freq, s, c);
        }
        before = (uint32_t)pos;
        turn[i][turn_at(for_keys.half, f)] = make_double2(c, s);
      }
    }
    __syncthreads();
  }

  const auto one = [&](int h, int kind, bool more, int next_h, int next_kind) __attribute__((always_inline)) {
    float v[kPasses][8], top = 0.0f;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      if (!holds(p)) continue;
      if (kind == 0) {
        values<D, kDynamic>(for_keys, in[p], turn[min(max(slot(p) - t.slot0, 0), t.n - 1)], v[p]);
      } else {
        const uint32_t d[4] = {in[p].x, in[p].y, in[p].z, in[p].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[p][2 * j] = bf16_low(d[j]), v[p][2 * j + 1] = bf16_high(d[j]);
      }
      top = largest(v[p], top, true);      // (0 where there is no token)
      __builtin_amdgcn_sched_barrier(0);   // (one pass's binary64 values at a time: registers)
    }
    if (more) load(next_h, next_kind);
    float* scale_at = (kind ? a.cache.scale[1] : a.cache.scale[0]) + (int64_t)t.page * a.cache.scale_stride + h;
    uint8_t* out = (kind ? a.cache.kv[1] : a.cache.kv[0]) +
                   (int64_t)t.page * (kind ? a.cache.page_stride[1] : a.cache.page_stride[0]) +
                   (int64_t)h * a.cache.page_size * D;
    const float held = kDynamic && t.slot0 == 0 ? 0.0f : *scale_at;
    if (kDynamic && __any(!(top <= kLargest))) {      // without what is not finite
      top = 0.0f;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        if (holds(p)) top = largest(v[p], top, false);
      }
    }
    top = wave_max_of(top);
    if (lane == 0) wave_max[wave] = top;
    __syncthreads();      // (the last head's codes have left LDS, too)
    float scale = held;
    if (kDynamic) {
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) top = fmaxf(top, wave_max[w]);
      scale = fmaxf(held, page_scale(top));
      if (scale > held && t.slot0 > 0) bring_along<D>(out, kind, t.slot0, held / scale, threadIdx.x, kThreads);
    }
    const float inverse = 1.0f / scale;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      if (!holds(p) || (D == 256 && kind == 1 && p % 2 == 1)) continue;
      const int s = slot(p);
      if (kind == 0) {
        uint8_t* to = codes + 16 * key_piece(s / 16 * D + e0 / 16 * 16 + s % 16) + (e0 & 8);
        *reinterpret_cast<uint2*>(to) = eight_codes<kDynamic>(v[p], scale, inverse);
      } else {
        uint8_t* to = codes + s / 16 * 16 * D + e0 / 64 * 1024 + (s % 16 / 4 * 16 + (e0 & 8)) * 16 + e0 / 16 % 4 * 4;
        if constexpr (D == 256) {
          const uint4 c = fours(eight_codes<kDynamic>(v[p], scale, inverse), eight_codes<kDynamic>(v[p + 1], scale, inverse));
          uint8_t* at = to + lane / 32 * 64;
          *reinterpret_cast<uint32_t*>(at) = c.x;
          *reinterpret_cast<uint32_t*>(at + 16) = c.y;
          *reinterpret_cast<uint32_t*>(at + 32) = c.z;
          *reinterpret_cast<uint32_t*>(at + 48) = c.w;
        } else {
          const uint2 c = fours(eight_codes<kDynamic>(v[p], scale, inverse));
          uint8_t* at = to + lane / 32 * 64 + lane / 16 % 2 * 32;
          *reinterpret_cast<uint32_t*>(at) = c.x;
          *reinterpret_cast<uint32_t*>(at + 16) = c.y;
        }
      }
    }
    __syncthreads();      // (the held codes are written, too)
    for (int y = (t.slot0 / 16) * D + threadIdx.x; y < ((last + 15) / 16) * D; y += kThreads) {
      const int group = y / D, in_group = y % D;
      const uint4 c = reinterpret_cast<const uint4*>(codes)[kind == 0 ? key_piece(y) : y];
      uint4* at = reinterpret_cast<uint4*>(out) + y;
      if (kind == 0) {
        const int s = group * 16 + (in_group & 15);
        if (s >= t.slot0 && s < last) *at = c;
      } else {
        const int s = group * 16 + ((in_group >> 4) & 3) * 4;
        if (s >= t.slot0 && s + 4 <= last) {
          *at = c;
        } else {
          const uint32_t word[4] = {c.x, c.y, c.z, c.w};
          uint8_t* bytes = reinterpret_cast<uint8_t*>(at);
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (s + u >= t.slot0 && s + u < last)
#pragma unroll
              for (int j = 0; j < 4; ++j) bytes[j * 4 + u] = (uint8_t)(word[j] >> (8 * u));
        }
      }
    }
    if (kDynamic && threadIdx.x == 0) *scale_at = scale;
  };
  for (int h = h0; h < h1; ++h) {
    one(h, 0, true, h, 1);
    one(h, 1, h + 1 < h1, h + 1, 0);
  }
}

// Few rows: a workgroup for a page, keys or values, and 512 / D heads; a wave's lanes
// hold one token of each head at a time, and its four waves take turns with the
// tokens (a page may have all that a sequence among many short ones has).
template <int D, bool kDynamic>
__global__ __launch_bounds__(256) void kv_append_tokens_kernel(AppendArgs a) {
  constexpr int kLanes = D / 8, kHeads = 64 / kLanes, kWaves = 4;
  __shared__ double2 turns[kWaves][D / 2];
  __shared__ float tops[kWaves][64];
  const int groups = (a.cache.heads + kHeads - 1) / kHeads;
  const int kind = blockIdx.x & 1, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h0 = (int)(blockIdx.x >> 1) % groups * kHeads;
  Touch t;
  if (!find_touch(a, (int)(blockIdx.x >> 1) / groups, t)) return;
  const int waves = min(t.n, kWaves);
  if (wave >= waves) return;
  double2* turn = turns[wave];
  const Treatment how = treatment<D>(a, kind);
  const bool live = h0 + lane / kLanes < a.cache.heads;
  const int h = min(h0 + lane / kLanes, a.cache.heads - 1);
  const int64_t ld = kind ? a.ld[1] : a.ld[0];
  const uint16_t* x = (kind ? a.x[1] : a.x[0]) + (int64_t)t.row0 * ld + (int64_t)h * D + how.e0;
  const auto load = [&](int i) { return *reinterpret_cast<const uint4*>(x + i * ld); };
  const auto treated = [&](int i, float(&v)[8]) __attribute__((always_inline)) {
    const uint4 in = load(i);
    if (how.rotate) {
      wave_lds_fence();
      const int pos = position(a, t, i);
      for (int f = lane; f < how.half; f += 64) {
        double s, c;
        sin_cos<double>(pos, a.rope.inv_freq[f], s, c);
        turn[turn_at(how.half, f)] = make_double2(c, s);
      }
      wave_lds_fence();
    }
    values<D, kDynamic>(how, in, turn, v);
  };

  float* scale_at = (kind ? a.cache.scale[1] : a.cache.scale[0]) + (int64_t)t.page * a.cache.scale_stride + h;
  const float held = kDynamic && t.slot0 == 0 ? 0.0f : *scale_at;
  const int last = wave + (t.n - 1 - wave) / waves * waves;      // of this wave's tokens
  float v[8], scale = held;
  if (kDynamic) {
    float top = 0.0f;
    for (int i = wave; i < t.n; i += waves) {
      treated(i, v);
      top = largest(v, top, false);
    }
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (waves > 1) {
      tops[wave][lane] = top;
      __syncthreads();
      for (int w = 0; w < waves; ++w) top = fmaxf(top, tops[w][lane]);
    }
    scale = fmaxf(held, page_scale(top));
  }
  uint8_t* out = (kind ? a.cache.kv[1] : a.cache.kv[0]) +
                 (int64_t)t.page * (kind ? a.cache.page_stride[1] : a.cache.page_stride[0]) +
                 (int64_t)h * a.cache.page_size * D;
  if (live && scale > held && t.slot0 > 0)
    bring_along<D>(out, kind, t.slot0, held / scale, wave * kLanes + lane % kLanes, waves * kLanes);
  __syncthreads();      // (the held codes of pieces that new values share are written)
  const float inverse = 1.0f / scale;
  for (int i = last; i >= 0; i -= waves) {      // (the last one's values are at hand)
    if (!kDynamic || i != last) treated(i, v);
    const uint2 c = eight_codes<kDynamic>(v, scale, inverse);
    if (live) put_codes<D>(out, kind, t.slot0 + i, how.e0, c);
  }
  if (kDynamic && live && wave == 0 && lane % kLanes == 0) *scale_at = scale;
}

template <int D, bool kDynamic>
static hipError_t launch(const AppendArgs& a, const AppendPlan& p, hipStream_t stream) {
  const dim3 grid((unsigned)p.workgroups);
  const int elements = a.cache.page_size * D;
  if (p.tokens) {
    kv_append_tokens_kernel<D, kDynamic><<<grid, 256, 0, stream>>>(a);
  } else if (elements <= 2048) {
    if constexpr (D <= 128) kv_append_pages_kernel<D, 256, 1, kDynamic><<<grid, 256, 0, stream>>>(a, p.each);
  } else if (elements <= 4096) {
    kv_append_pages_kernel<D, 256, 2, kDynamic><<<grid, 256, 0, stream>>>(a, p.each);
  } else if (elements <= 8192) {
    kv_append_pages_kernel<D, 512, 2, kDynamic><<<grid, 512, 0, stream>>>(a, p.each);
  } else {
    if constexpr (D >= 128) kv_append_pages_kernel<D, 1024, 2, kDynamic><<<grid, 1024, 0, stream>>>(a, p.each);
  }
  return hipGetLastError();
}

template <bool kDynamic>
static hipError_t launch_mode(const AppendArgs& a, const AppendPlan& p, hipStream_t stream) {
  return a.cache.dim == 64    ? launch<64, kDynamic>(a, p, stream)
         : a.cache.dim == 128 ? launch<128, kDynamic>(a, p, stream)
                              : launch<256, kDynamic>(a, p, stream);
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream) {
  const AppendPlan p = append_plan(a.cache, a.batch);
  return a.dynamic ? launch_mode<true>(a, p, stream) : launch_mode<false>(a, p, stream);
}

}  // namespace nvfp4
