// Attention of a batch whose sequences share prefixes, over the paged E4M3 cache
// (definition: nvfp4_paging.h), for gfx950.
//
// Two passes of the attention's kernels and a join: the rows of all of a group's
// sequences over its prefix, which is read once for all of them, and each sequence's
// rows over its own tokens.  Both keep (maximum, sum, unscaled y) of every row in
// 32 bits, and the join takes them together as it does the pieces of one sequence:
//   m = max m_i,  y = sum_i 2^(m_i - m) y_i / sum_i 2^(m_i - m) l_i.
#include "attention_plan.h"
#include "kv_attention_rows.h"
#include "kv_attention_wide.h"
#include "kv_shared_device.h"

namespace nvfp4 {

template <int D, int kTiles>
__global__ __launch_bounds__(256, rows_waves(D, kTiles, 4, true)) void kv_attention_prefix_rows_kernel(PrefixArgs a) {
  attention_rows<D, kTiles, 4, true>(a);
}

template <int D>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void kv_attention_prefix_tile_kernel(PrefixArgs a, int tiles) {
  attention_tile<D, true>(a, tiles);
}

template <int D, int kTiles, int kWaves>
__global__ __launch_bounds__(kWaves * 64, rows_waves(D, kTiles, kWaves, true)) void kv_attention_own_rows_kernel(OwnArgs a) {
  attention_rows<D, kTiles, kWaves, true>(a);
}

template <int D>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void kv_attention_own_tile_kernel(OwnArgs a, int tiles) {
  attention_tile<D, true>(a, tiles);
}

// A wave takes a packed row, four pieces' loads in flight: those of its group's
// prefix, then its own.
template <int D, int kTiles>
__global__ __launch_bounds__(256) void kv_attention_shared_join_kernel(SharedArgs a, PrefixPieces of) {
  constexpr int kRows = 16 * kTiles, kEach = D / 64, kAhead = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = (int)(blockIdx.x % (kRows / 4)) * 4 + wave;
  const int h = (int)(blockIdx.x / (kRows / 4)) % a.cache.heads;
  const int number = (int)(blockIdx.x / (kRows / 4)) / a.cache.heads;
  Tile t;
  int g, prefix;
  if (!find_own_tile<kRows>(a, number, t, g, prefix) || row >= t.n) return;
  const int r = t.r0 + row;                                            // of the sequence
  const int own = pieces_of(a, t);
  const int before = prefix > 0 ? min((prefix - 1) / of.chunk, of.splits - 1) + 1 : 0;
  const float2* stats[2];
  const float* part[2];
  int stride[2] = {1, kRows};
  stats[0] = nullptr, part[0] = nullptr;
  if (before > 0) {
    const int row0 = start_row(a.batch, group_start(a, g)), rows = 16 * of.tiles;
    const int packed = (t.row0 - row0) * a.group + r;
    const int64_t tile = (int64_t)row0 * a.group / rows + g + packed / rows;
    const int64_t first = (tile * a.cache.heads + h) * of.splits * rows + packed % rows;
    const int64_t all = ((int64_t)a.batch.rows * a.group / rows + a.groups) * a.cache.heads * of.splits * rows;
    stats[0] = reinterpret_cast<const float2*>(of.part) + first;
    part[0] = of.part + 2 * all + first * D + lane * kEach;
    stride[0] = rows;
  }
  const int64_t first = ((int64_t)number * a.cache.heads + h) * a.splits * kRows + row;
  stats[1] = reinterpret_cast<const float2*>(a.part) + first;
  part[1] = a.part + part_tiles(a, kRows) * a.cache.heads * a.splits * (2 * kRows) + first * D + lane * kEach;

  float m = kNone, l = 0.0f, y[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) y[i] = 0.0f;
  for (int p = 0; p < before + own; p += kAhead) {
    float2 st[kAhead];
    float v[kAhead][kEach];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int which = p + u < before ? 0 : 1;
      const int64_t at = (int64_t)(p + u - (which ? before : 0)) * stride[which];
      st[u] = make_float2(kNone, 0.0f);
#pragma unroll
      for (int i = 0; i < kEach; ++i) v[u][i] = 0.0f;
      if (p + u < before + own) {
        st[u] = stats[which][at];
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[u][i] = part[which][at * D + i];
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
      const float w = __builtin_amdgcn_exp2f(st[u].x - base);
      l = fmaf(st[u].y, w, l);
#pragma unroll
      for (int i = 0; i < kEach; ++i) y[i] = fmaf(v[u][i], w, y[i]);
    }
  }
  const int head = h * a.group + r % a.group;
  const int64_t token_row = t.row0 + r / a.group;
  uint16_t* to = a.y + token_row * a.ldy + (int64_t)head * D;
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

template <int D>
hipError_t launch_prefix(const PrefixArgs& a, int64_t tiles, hipStream_t stream) {
  const dim3 grid((unsigned)(tiles * a.cache.heads * a.splits));
  if (a.row_tiles == 8)
    kv_attention_prefix_tile_kernel<D><<<grid, 256, 0, stream>>>(a, (int)tiles);
  else if (a.row_tiles == 2)
    kv_attention_prefix_rows_kernel<D, 2><<<grid, 256, 0, stream>>>(a);
  else
    kv_attention_prefix_rows_kernel<D, 1><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_own(const OwnArgs& a, int64_t tiles, hipStream_t stream) {
  const dim3 grid((unsigned)(tiles * a.cache.heads * a.splits));
  if (a.row_tiles == 8)
    kv_attention_own_tile_kernel<D><<<grid, 256, 0, stream>>>(a, (int)tiles);
  else if (a.row_tiles == 2)
    kv_attention_own_rows_kernel<D, 2, 4><<<grid, 256, 0, stream>>>(a);
  else if (a.waves == 8)
    kv_attention_own_rows_kernel<D, 1, 8><<<grid, 512, 0, stream>>>(a);
  else
    kv_attention_own_rows_kernel<D, 1, 4><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_join(const SharedArgs& a, const PrefixPieces& of, int64_t tiles, hipStream_t stream) {
  const dim3 grid((unsigned)(tiles * a.cache.heads * a.row_tiles * 4));
  if (a.row_tiles == 8)
    kv_attention_shared_join_kernel<D, 8><<<grid, 256, 0, stream>>>(a, of);
  else if (a.row_tiles == 2)
    kv_attention_shared_join_kernel<D, 2><<<grid, 256, 0, stream>>>(a, of);
  else
    kv_attention_shared_join_kernel<D, 1><<<grid, 256, 0, stream>>>(a, of);
  return hipGetLastError();
}

template <int D>
hipError_t launch(const SharedArgs& a, const SharedPlan& p, hipStream_t stream) {
  OwnArgs own;
  static_cast<SharedArgs&>(own) = a;
  const int64_t tiles = host_tiles(a.batch, a.group, 16 * a.row_tiles);
  const PrefixPieces of = {p.prefix.tiles, p.prefix.chunk, p.prefix.splits, a.part};
  if (a.groups > 0) {
    PrefixArgs before;
    static_cast<SharedArgs&>(before) = a;
    before.causal = 0;
    before.row_tiles = p.prefix.tiles;
    before.waves = 4;
    before.chunk = p.prefix.chunk;
    before.splits = p.prefix.splits;
    const hipError_t e = launch_prefix<D>(before, host_tiles(prefix_batch(a), a.group, 16 * p.prefix.tiles), stream);
    if (e != hipSuccess) return e;
  }
  own.part = a.part + p.prefix_bytes / sizeof(float);
  hipError_t e = launch_own<D>(own, tiles, stream);
  if (e != hipSuccess) return e;
  return launch_join<D>(own, of, tiles, stream);
}

}  // namespace

hipError_t launch_kv_attention_shared(const SharedArgs& args, const SharedPlan& p, hipStream_t stream) {
  SharedArgs a = args;
  a.row_tiles = p.own.tiles;
  a.waves = p.own.waves;
  a.chunk = p.own.chunk;
  a.splits = p.own.splits;
  return a.cache.dim == 64 ? launch<64>(a, p, stream) : a.cache.dim == 128 ? launch<128>(a, p, stream) : launch<256>(a, p, stream);
}

}  // namespace nvfp4
