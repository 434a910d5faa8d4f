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
#include "kv_attention_rows.h"

namespace nvfp4 {

template <int D, int kTiles, int kWaves, bool kSplit>
__global__ __launch_bounds__(kWaves * 64, rows_waves(D, kTiles, kWaves, kSplit)) void kv_attention_rows_kernel(AttentionArgs a) {
  attention_rows<D, kTiles, kWaves, kSplit>(a);
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
