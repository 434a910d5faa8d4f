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
// rows; else by launches and the selection's passes over a row's scores.
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

template <int kHow, bool kMax>
__device__ __forceinline__ f16x2 fold(f16x2 v) {
  const f16x2 o = __builtin_bit_cast(f16x2, row_other<kHow>(__builtin_bit_cast(uint32_t, v)));
  return kMax ? max2(v, o) : min2(v, o);
}

template <bool kMax>
__device__ __forceinline__ f16x2 over_row(f16x2 v) {
  v = fold<0xB1, kMax>(v);
  v = fold<0x4E, kMax>(v);
  v = fold<0x141, kMax>(v);
  return fold<0x140, kMax>(v);
}

// A wave takes one head of one full page.  Pages of sequence b that its new rows
// completed have the numbers from cu_rows[b] / page_size + b on.
template <int D>
__global__ __launch_bounds__(256) void kv_page_bounds_kernel(BoundsArgs a, int items) {
  __shared__ _Float16 found[4][2][D];
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
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f16x2 top = over_row<true>(hi[c][i]), low = over_row<false>(lo[c][i]);
      if ((lane & 15) == 0) {
        *reinterpret_cast<f16x2*>(&found[wave][0][64 * c + 16 * (lane >> 4) + 2 * i]) = top;
        *reinterpret_cast<f16x2*>(&found[wave][1][64 * c + 16 * (lane >> 4) + 2 * i]) = low;
      }
    }
  // (One wave's LDS, in the order of its accesses.)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  constexpr int kEach = 2 * D / 64;      // elements of hi, then of lo
  float v[kEach], top = 0.0f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = (float)(&found[wave][0][0])[lane * kEach + i];
    top = fmaxf(top, fabsf(v[i]));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  const float over = top > 0.0f ? top : 1.0f;
  uint32_t packed[(kEach + 3) / 4] = {};
#pragma unroll
  for (int i = 0; i < kEach; ++i) packed[i / 4] |= ((uint32_t)(int)rintf(v[i] * 127.0f / over) & 255u) << (8 * (i % 4));
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

// Whole numbers that order as the scores do (no NaN; -0 is 0).
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kScorePages = 256;         // pages of a workgroup

template <int D>
__global__ __launch_bounds__(256) void kv_page_scores_kernel(SelectArgs a, int chunks) {
  constexpr int kSteps = D / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  int id = blockIdx.x;
  const int h = id % a.cache.heads;
  id /= a.cache.heads;
  const int row = id / chunks, chunk = id % chunks;
  const RowPages r = row_pages(a, row);
  if (r.pages <= a.count) return;                                    // (all of them are taken)
  const int first = a.first, end = r.pages - a.recent;
  const int from = chunk * kScorePages + wave * 16;
  if ((int64_t)chunk * kScorePages >= end) return;
  uint32_t* const scores = a.scores + ((int64_t)row * a.cache.heads + h) * a.max_pages;
  float best[kScorePages / 64][4];
#pragma unroll
  for (int x = 0; x < kScorePages / 64; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) best[x][e] = -INFINITY;
  int pages[kScorePages / 64];
#pragma unroll
  for (int x = 0; x < kScorePages / 64; ++x) {
    const int j = from + 64 * x + col;
    int p = -1;
    if (j >= first && j < end) p = a.batch.table[(int64_t)r.b * a.batch.table_stride + j];
    pages[x] = p >= 0 && p < a.cache.num_pages ? p : -1;
  }
  for (int a0 = 0; a0 < a.group; a0 += 16) {
    // Query head h * group + a0 + col in 8 bits; elements 64 s + 16 quarter .. + 15.
    const uint16_t* src = a.q + (int64_t)row * a.ldq + (int64_t)(h * a.group + min(a0 + col, a.group - 1)) * D + quarter * 16;
    float v[kSteps][16], top = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const u32x4 w0 = *reinterpret_cast<const u32x4*>(src + 64 * s), w1 = *reinterpret_cast<const u32x4*>(src + 64 * s + 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[s][2 * i] = bf16_low(w0[i]), v[s][2 * i + 1] = bf16_high(w0[i]);
        v[s][8 + 2 * i] = bf16_low(w1[i]), v[s][9 + 2 * i] = bf16_high(w1[i]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[s][i]));
    }
    top = over_quarters_max(top);
    const float over = top > 0.0f ? top : 1.0f, unit = top / 127.0f;
    i32x4 above[kSteps], below[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t up = 0, down = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int n = (int)rintf(v[s][4 * i + e] * 127.0f / over);
          up |= ((uint32_t)max(n, 0) & 255u) << (8 * e);
          down |= ((uint32_t)min(n, 0) & 255u) << (8 * e);
        }
        above[s][i] = (int)up, below[s][i] = (int)down;
      }
#pragma unroll
    for (int x = 0; x < kScorePages / 64; ++x) {
      const int8_t* at = a.bounds.codes + (int64_t)max(pages[x], 0) * a.bounds.page_stride + (int64_t)h * 2 * D + quarter * 16;
      i32x4 sum = (i32x4){0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const i32x4 hi = *reinterpret_cast<const i32x4*>(at + 64 * s), lo = *reinterpret_cast<const i32x4*>(at + D + 64 * s);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi, above[s], sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(lo, below[s], sum, 0, 0, 0);
      }
      // Pages 4 quarter + e, query head col.
#pragma unroll
      for (int e = 0; e < 4; ++e) best[x][e] = fmaxf(best[x][e], (float)sum[e] * unit);
    }
  }
#pragma unroll
  for (int x = 0; x < kScorePages / 64; ++x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float m = best[x][e];
      m = fmaxf(m, __uint_as_float(row_other<0xB1>(__float_as_uint(m))));
      m = fmaxf(m, __uint_as_float(row_other<0x4E>(__float_as_uint(m))));
      m = fmaxf(m, __uint_as_float(row_other<0x141>(__float_as_uint(m))));
      best[x][e] = fmaxf(m, __uint_as_float(row_other<0x140>(__float_as_uint(m))));
    }
    // Lane col of a quarter writes page 4 quarter + col.
    const int mine = 4 * quarter + (col & 3), j = from + 64 * x + mine;
    const float m = (col & 2) ? ((col & 1) ? best[x][3] : best[x][2]) : ((col & 1) ? best[x][1] : best[x][0]);
    const int page = __shfl(pages[x], mine);
    if (col < 4 && j >= first && j < end) {
      const float step = page < 0 ? 0.0f : a.bounds.step[(int64_t)page * a.bounds.step_stride + h];
      scores[j] = page < 0 ? 0u : key_of(m * step);                   // (a page that is not in the cache: the last choice)
    }
  }
}

// ---------------------------------------------------------------- selection

// One workgroup for each row and key head: the want largest keys of scores[first ..
// end), the lowest pages first among equals.  The want-th largest key is found 8 bits at
// a time from the counts of each value of them; then the pages are written in order.
constexpr int kSelectThreads = 512, kSelectWaves = kSelectThreads / 64;

__global__ __launch_bounds__(kSelectThreads) void kv_select_kernel(SelectArgs a) {
  __shared__ int counts[256];
  __shared__ int totals[2][kSelectWaves];
  __shared__ int found[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int h = (int)(blockIdx.x % a.cache.heads), row = (int)(blockIdx.x / a.cache.heads);
  const RowPages r = row_pages(a, row);
  const int shift = a.cache.page_shift;
  if (h == 0 && threadIdx.x == 0) {
    const int taken = min(r.pages, a.count);
    a.tokens[row] = r.pages <= 0 ? r.pages : ((taken - 1) << shift) + (r.token & ((1 << shift) - 1)) + 1;
  }
  if (r.pages < 0) return;
  const int64_t to = ((int64_t)row * a.cache.heads + h) * a.count;
  const int32_t* const table = a.batch.table + (int64_t)r.b * a.batch.table_stride;
  const auto put = [&](int at, int entry) {
    a.index[to + at] = entry;
    a.pages[to + at] = table[entry];
  };
  if (r.pages <= a.count) {
    for (int i = threadIdx.x; i < a.count; i += kSelectThreads) {
      if (i < r.pages) put(i, i);
      else a.index[to + i] = -1, a.pages[to + i] = -1;
    }
    return;
  }
  for (int i = threadIdx.x; i < a.first; i += kSelectThreads) put(i, i);
  const int first = a.first, end = r.pages - a.recent;
  for (int i = threadIdx.x; i < a.recent; i += kSelectThreads) put(a.count - a.recent + i, end + i);
  int want = a.count - a.first - a.recent;
  if (want == 0) return;
  const uint32_t* const scores = a.scores + ((int64_t)row * a.cache.heads + h) * a.max_pages;
  uint32_t prefix = 0;
  int left = want;                                       // of those with this prefix
  for (int bit = 24; bit >= 0; bit -= 8) {
    for (int i = threadIdx.x; i < 256; i += kSelectThreads) counts[i] = 0;
    __syncthreads();
    for (int j = first + threadIdx.x; j < end; j += kSelectThreads) {
      const uint32_t k = scores[j];
      if (bit == 24 || (k >> (bit + 8)) == prefix) atomicAdd(&counts[(k >> bit) & 255], 1);      // (whole numbers: any order)
    }
    __syncthreads();
    if (wave == 0) {      // the largest value with at least `left` keys at or above it
      int mine[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += mine[i] = counts[255 - 4 * lane - i];
      int up = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int other = __shfl_up(up, d);
        if (lane >= d) up += other;
      }
      int above = up - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < left && above + mine[i] >= left) found[0] = 255 - 4 * lane - i, found[1] = left - above;
        above += mine[i];
      }
    }
    __syncthreads();
    prefix = (prefix << 8) | (uint32_t)found[0];
    left = found[1];
  }
  // prefix: the want-th largest key; `left` of the pages with it, the lowest, are taken.
  int taken = 0, equal = 0;                              // before this round of pages
  for (int j0 = first; j0 < end && taken + min(equal, left) < want; j0 += kSelectThreads) {
    const int j = j0 + threadIdx.x;
    const uint32_t k = j < end ? scores[j] : 0;
    const bool above = j < end && k > prefix, same = j < end && k == prefix;
    const unsigned long long above_of = __ballot(above), same_of = __ballot(same), below = (1ull << lane) - 1;
    if (lane == 0) totals[0][wave] = __popcll(above_of), totals[1][wave] = __popcll(same_of);
    __syncthreads();
    int before = taken, same_before = equal;
    for (int w = 0; w < kSelectWaves; ++w) {
      if (w < wave) before += totals[0][w], same_before += totals[1][w];
      taken += totals[0][w];
      equal += totals[1][w];
    }
    before += __popcll(above_of & below);
    same_before += __popcll(same_of & below);
    if (above || (same && same_before < left)) put(a.first + before + min(same_before, left), j);
    __syncthreads();
  }
}

size_t kv_select_workspace_bytes(int64_t rows, int64_t heads, int64_t max_pages) {
  return (size_t)(rows * heads * max_pages) * sizeof(uint32_t);
}

bool select_fits(const SelectArgs& a) {
  const int64_t chunks = (a.batch.max_tokens / a.cache.page_size + kScorePages - 1) / kScorePages;
  const int64_t each = (int64_t)a.batch.rows * a.cache.heads;
  return one_grid(each * (chunks > 0 ? chunks : 1), 256) && one_grid(each, kSelectThreads);
}

hipError_t launch_kv_select(const SelectArgs& a, hipStream_t stream) {
  const int chunks = (a.max_pages + kScorePages - 1) / kScorePages;
  const int64_t each = (int64_t)a.batch.rows * a.cache.heads;
  if (a.max_pages > a.count && a.count > a.first + a.recent) {
    const dim3 grid((unsigned)(each * chunks));
    if (a.cache.dim == 64)
      kv_page_scores_kernel<64><<<grid, 256, 0, stream>>>(a, chunks);
    else if (a.cache.dim == 128)
      kv_page_scores_kernel<128><<<grid, 256, 0, stream>>>(a, chunks);
    else
      kv_page_scores_kernel<256><<<grid, 256, 0, stream>>>(a, chunks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  kv_select_kernel<<<dim3((unsigned)each), kSelectThreads, 0, stream>>>(a);
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
