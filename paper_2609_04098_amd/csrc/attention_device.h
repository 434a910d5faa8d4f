// Device helpers of the attention kernels: bf16 and E4M3 conversions, the
// rotation's sines and cosines, and the place of a step's rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention_launch.h"

namespace nvfp4 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_low(uint32_t d) { return __uint_as_float(d << 16); }
__device__ __forceinline__ float bf16_high(uint32_t d) { return __uint_as_float(d & 0xFFFF0000u); }

// Two values rounded to nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)lo, (__bf16)hi});
}

// sin and cos of the angle pos * inv_freq.  Whole turns and quarters are taken
// off in binary64, where a position of 2^24 leaves 2^-29 turns' accuracy; the
// rest, |x| <= pi / 4, goes through the Taylor series in T (float: to 1e-8,
// double: to 5e-13).
template <typename T>
__device__ __forceinline__ void sin_cos(int pos, float inv_freq, T& sine, T& cosine) {
  double t = (double)pos * (double)inv_freq * 0.15915494309189535;      // turns
  t -= rint(t);
  const double q = rint(4.0 * t);
  const T x = (T)((t - 0.25 * q) * 6.283185307179586);
  const T z = x * x;
  T s, c;
  if (sizeof(T) == 8) {
    s = fma(z, (T)(1.0 / 6227020800.0), (T)(-1.0 / 39916800.0));
    s = fma(z, s, (T)(1.0 / 362880.0));
    s = fma(z, s, (T)(-1.0 / 5040.0));
    c = fma(z, (T)(1.0 / 479001600.0), (T)(-1.0 / 3628800.0));
    c = fma(z, c, (T)(1.0 / 40320.0));
  } else {
    s = fma(z, (T)(1.0 / 362880.0), (T)(-1.0 / 5040.0));
    c = fma(z, (T)(-1.0 / 3628800.0), (T)(1.0 / 40320.0));
  }
  s = fma(z, s, (T)(1.0 / 120.0));
  s = fma(z, s, (T)(-1.0 / 6.0));
  s = fma(x * z, s, x);
  c = fma(z, c, (T)(-1.0 / 720.0));
  c = fma(z, c, (T)(1.0 / 24.0));
  c = fma(z, c, (T)-0.5);
  c = fma(z, c, (T)1);
  const int n = (int)q & 3;
  const T a = (n & 1) ? c : s, b = (n & 1) ? s : c;
  sine = (n & 2) ? -a : a;
  cosine = ((n + 1) & 2) ? -b : b;
}

// The nearest E4M3 codes (ties to even) of four values of at most 448; NaN
// gives 0x7F.
__device__ __forceinline__ uint32_t e4m3_codes(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

// Rows [row, row + rows) of a sequence and the tokens that they are: row + i is
// token first + i (which may be below 0).  Bounded by the tensors whatever
// cu_rows and kv_len hold.
struct SeqRows {
  int row, rows, first, len;
};

__device__ __forceinline__ SeqRows seq_rows(const KvBatchArgs& a, int row0, int row1, int len) {
  SeqRows s;
  s.row = min(max(row0, 0), a.rows);
  s.rows = min(max(row1, s.row), a.rows) - s.row;
  s.first = max(len, 0) - s.rows;              // a length above the table's keeps its tokens' numbers
  s.len = min(max(len, 0), a.max_tokens);
  return s;
}

__device__ __forceinline__ int row_bound(const KvBatchArgs& a, int b) { return min(max(a.cu_rows[b], 0), a.rows); }

// The last of n entries (n >= 1) whose key is at most `value` (the first if
// none is), and its key.  Keys do not decrease.  A wave looks at 64 entries at
// a time, so that up to 64 entries cost one load's latency and up to 4096 two;
// all 64 lanes call it with the same arguments.
template <typename Key>
__device__ __forceinline__ int last_at_most(int n, int value, int& entry, Key key) {
  const int lane = threadIdx.x & 63;
  int stride = 1, lo = 0;
  while (stride * 64 < n) stride *= 64;
  int found = 0;
  for (; stride > 0; stride /= 64) {
    const int at = lo + lane * stride;
    const int k = key(min(at, n - 1));
    const unsigned long long hit = __ballot(at < n && k <= value);
    const int i = hit == 0 ? 0 : 63 - __builtin_clzll(hit);
    found = __builtin_amdgcn_readlane(k, i);
    lo += i * stride;
  }
  entry = __builtin_amdgcn_readfirstlane(min(lo, n - 1));
  return found;
}

// The sequence b of work item `item` and its rows: the last one whose first item,
// first_item(first row, b), is at most `item`; ordinal: which of its items this
// is.  (Without cu_rows, sequence item / each.)  For up to 64 sequences all that
// there is to know of them comes in one load's latency.
template <typename First>
__device__ __forceinline__ SeqRows find_rows(const KvBatchArgs& a, int item, int each, int& b, int& ordinal,
                                             First first_item) {
  if (a.cu_rows == nullptr) {
    b = item / each;
    ordinal = item - b * each;
    return seq_rows(a, b, b + 1, a.kv_len[b]);
  }
  if (a.seqs <= 64) {
    const int lane = threadIdx.x & 63, at = min(lane, a.seqs - 1);
    const int row0 = a.cu_rows[at], row1 = a.cu_rows[at + 1], len = a.kv_len[at];
    const int k = first_item(min(max(row0, 0), a.rows), at);
    const unsigned long long hit = __ballot(lane < a.seqs && k <= item);
    b = hit == 0 ? 0 : 63 - __builtin_clzll(hit);
    ordinal = item - __builtin_amdgcn_readlane(k, b);
    return seq_rows(a, __builtin_amdgcn_readlane(row0, b), __builtin_amdgcn_readlane(row1, b),
                    __builtin_amdgcn_readlane(len, b));
  }
  ordinal = item - last_at_most(a.seqs, item, b, [&](int x) { return first_item(row_bound(a, x), x); });
  return seq_rows(a, a.cu_rows[b], a.cu_rows[b + 1], a.kv_len[b]);
}

}  // namespace nvfp4
