// Attention of a batch whose sequences share prefixes, over the paged E4M3 cache
// (definition: nvfp4_paging.h), for gfx950.
//
// Two passes of the attention's kernels, side by side in one launch, and a join: the rows
// of all of a group's sequences over its prefix, which is read once for all of them, and
// each sequence's rows over its own tokens.  Both keep (maximum, sum, unscaled y) of every row in
// 32 bits, and the join takes them together as it does the pieces of one sequence:
//   m = max m_i,  y = sum_i 2^(m_i - m) y_i / sum_i 2^(m_i - m) l_i.
//
// Bound by the conversions and exponentials beside the products, and by what waits between
// them with two waves a SIMD: 64 rows of 40 / 8 heads of 128 behind 32768 tokens take 76.6 us
// (0.56 PFLOP/s; vector units busy 54%, matrix units 25%; 16 rows a workgroup 78.5, 32 77.7, as the
// codes of 32 tokens are converted for more of them at once), the join 7.5, a launch and four
// loads' latencies.  150 rows of 24 / 4 heads of 256 behind 4160: 46.8 (40%, 16%) and 7.1.
#include "attention_plan.h"
#include "kv_attention_rows.h"
#include "kv_attention_wide.h"
#include "kv_shared_device.h"

namespace nvfp4 {

// The rows of a workgroup in either pass, 16 times kPrefix and kOwn: 8, for heads of 256, is
// the form of 128 rows (kv_attention_wide.h).
template <int D, int kForm>
struct PassLds {
  RowsLds<D, kForm, 4> of;
};

template <int D>
struct PassLds<D, 8> {
  TileLds<D> of;
};

constexpr int pass_waves(int dim, int form) { return form == 8 ? 2 : rows_waves(dim, form, 4, false); }
constexpr int fewer(int a, int b) { return a < b ? a : b; }

template <int D, int kForm, typename Args>
__device__ __forceinline__ void pass(const Args& a, int tiles, int h, int number, int piece, void* lds) {
  auto& of = static_cast<PassLds<D, kForm>*>(lds)->of;
  if constexpr (kForm == 8)
    attention_tile<D, true>(a, tiles, h, number, piece, of);
  else
    attention_rows<D, kForm, 4, true>(a, h, number, piece, of);
}

// Both passes in one launch, so that the prefixes' products, which the matrix and vector
// units bound, run beside the own tokens' loads, which memory bounds.  The prefixes' go
// first: few long workgroups, spread evenly while the compute units are empty (mixed with
// the short ones, 3 of 288 came to one unit and none to others: 218 us for 80).
// Workgroups go to the eight dies in turn: a die takes a run of the prefix's work, in
// which the tiles of rows that read the same keys follow each other.
template <int D, int kPrefix, int kOwn>
__global__ __launch_bounds__(256, fewer(pass_waves(D, kPrefix), pass_waves(D, kOwn))) void kv_attention_shared_kernel(
    SharedArgs a, PrefixPieces of, SharedWork w) {
  constexpr size_t kBytes = sizeof(PassLds<D, kPrefix>) > sizeof(PassLds<D, kOwn>) ? sizeof(PassLds<D, kPrefix>)
                                                                                   : sizeof(PassLds<D, kOwn>);
  __shared__ __attribute__((aligned(16))) char lds[kBytes];
  if (blockIdx.x >= 8 * w.prefix_eighth) {
    const unsigned id = blockIdx.x - 8 * w.prefix_eighth;
    OwnArgs o;
    static_cast<SharedArgs&>(o) = a;
    const unsigned rest = id / a.cache.heads, number = rest / a.splits;
    pass<D, kOwn>(o, w.own_tiles, (int)(id % a.cache.heads), (int)number, piece_of((int)(rest % a.splits), (int)number, a.splits), lds);
  } else {
    const unsigned id = (blockIdx.x & 7) * w.prefix_eighth + (blockIdx.x >> 3);
    if (id >= w.prefix) return;
    PrefixArgs p;
    static_cast<SharedArgs&>(p) = a;
    p.causal = 0;
    p.chunk = of.chunk;
    p.splits = of.splits;
    p.part = of.part;
    const unsigned rest = id / w.prefix_tiles;
    pass<D, kPrefix>(p, w.prefix_tiles, (int)(rest / of.splits), (int)(id % w.prefix_tiles), (int)(rest % of.splits), lds);
  }
}

// kShare waves take a query head of a row, each its share of the pieces, kAhead of their loads in
// flight: those of the group's prefix, then its own.
template <int D, int kShare>
__global__ __launch_bounds__(256) void kv_attention_shared_join_kernel(SharedArgs a, PrefixPieces of) {
  constexpr int kEach = D / 64, kAhead = 8;
  __shared__ float sums[kShare > 1 ? 4 : 1][kShare > 1 ? D : 1];
  __shared__ float2 totals[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = wave % kShare;
  const unsigned item = blockIdx.x * (4 / kShare) + wave / kShare;
  const int token_row = __builtin_amdgcn_readfirstlane(item / a.q_heads), head = __builtin_amdgcn_readfirstlane(item % a.q_heads);
  if (token_row >= a.batch.rows) return;
  Tile t;
  int g, group_seq, ordinal;
  const SeqRows s = find_rows(a.batch, token_row, 1, t.b, ordinal, [](int first, int) { return first; });
  if (ordinal < 0 || ordinal >= s.rows) return;                        // behind the last sequence
  const int prefix = shared_prefix(a, t.b, s.first, g, group_seq);
  const int h = head / a.group, r = ordinal * a.group + head % a.group;      // packed row of the sequence
  const float2* stats[2];
  const float* part[2];
  int stride[2];
  // A row of a tile, of `rows`: its first piece, of `splits` of that many tiles' heads.
  const auto of_tile = [&](int which, const float* parts, int64_t tile, int64_t tiles, int row, int rows, int splits) {
    const int64_t first = (tile * a.cache.heads + h) * splits * rows + row;
    stats[which] = reinterpret_cast<const float2*>(parts) + first;
    part[which] = parts + 2 * (tiles * a.cache.heads * splits * rows) + first * D + lane * kEach;
    stride[which] = rows;
  };
  const int row0 = prefix > 0 ? start_row(a.batch, group_seq) : 0;
  // (Offsets that make no sense may put a group's first row behind this one.)
  const int before = prefix > 0 && row0 <= s.row ? min((prefix - 1) / of.chunk, of.splits - 1) + 1 : 0;
  stats[0] = nullptr, part[0] = nullptr, stride[0] = 0;
  if (before > 0) {
    const int rows = 16 * of.tiles, shift = 4 + __builtin_ctz(of.tiles);
    const auto tiles_in = [&](uint32_t x) { return of.tiles == 3 ? x / 48u : x >> shift; };
    const uint32_t packed = (uint32_t)(s.row - row0) * a.group + r, tile = tiles_in(packed);
    of_tile(0, of.part, (int64_t)tiles_in((uint32_t)row0 * a.group) + g + tile,
            prefix_tile_numbers((int64_t)a.batch.rows * a.group, rows, a.groups), (int)(packed - tile * rows), rows, of.splits);
  }
  int own;
  {
    const int shift = 4 + __builtin_ctz(a.row_tiles), rows = 1 << shift, row = r & (rows - 1);
    const int tile = a.batch.cu_rows == nullptr ? t.b * ((a.group + rows - 1) >> shift) : (int)(((int64_t)s.row * a.group) >> shift) + t.b;
    of_tile(1, a.part, tile + (r >> shift), tiles_of(a.batch, a.group, rows), row, rows, a.splits);
    // The tokens of the row's tile, as find_tile() has them.
    const int last = min(s.rows * a.group, r - row + rows) - 1;
    t.end = a.causal ? min(s.len, s.first + last / a.group + 1) : s.len;
    t.begin = min(prefix, max(0, t.end));
    own = pieces_of(a, t);
  }

  float m = kNone, l = 0.0f, y[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) y[i] = 0.0f;
  for (int p = share * kAhead; p < before + own; p += kShare * kAhead) {
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
  if (kShare > 1) {      // (the workgroup has one row and head: all of its waves are here)
    if (lane == 0) totals[wave] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < kEach; ++i) sums[kShare > 1 ? wave : 0][kShare > 1 ? lane * kEach + i : 0] = y[i];
    __syncthreads();
    if (wave != 0) return;
    const float top = fmaxf(fmaxf(totals[0].x, totals[1].x), fmaxf(totals[2].x, totals[3].x)), base = top == kNone ? 0.0f : top;
    m = top;
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) y[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float w = __builtin_amdgcn_exp2f(totals[u].x - base);
      l = fmaf(totals[u].y, w, l);
#pragma unroll
      for (int i = 0; i < kEach; ++i) y[i] = fmaf(sums[kShare > 1 ? u : 0][kShare > 1 ? lane * kEach + i : 0], w, y[i]);
    }
  }
  uint16_t* to = a.y + (int64_t)token_row * a.ldy + (int64_t)head * D;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (D == 64)
    to[lane] = __builtin_bit_cast(uint16_t, (__bf16)(y[0] * inv));
  else
#pragma unroll
    for (int i = 0; i + 1 < kEach; i += 2)
      *reinterpret_cast<uint32_t*>(to + lane * kEach + i) = bf16_pair(y[i] * inv, y[i + 1] * inv);
  if (a.lse != nullptr && lane == 0)
    a.lse[(int64_t)token_row * a.q_heads + head] = l == 0.0f ? kNone : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

namespace {

template <int D, int kPrefix, int kOwn>
hipError_t launch_passes(const SharedArgs& a, const PrefixPieces& of, const SharedWork& w, unsigned workgroups, hipStream_t stream) {
  kv_attention_shared_kernel<D, kPrefix, kOwn><<<dim3(workgroups), 256, 0, stream>>>(a, of, w);
  return hipGetLastError();
}

template <int D>
hipError_t launch_join(const SharedArgs& a, const PrefixPieces& of, int join_share, hipStream_t stream) {
  const int64_t items = (int64_t)a.batch.rows * a.q_heads;
  if (join_share == 4)
    kv_attention_shared_join_kernel<D, 4><<<dim3((unsigned)items), 256, 0, stream>>>(a, of);
  else
    kv_attention_shared_join_kernel<D, 1><<<dim3((unsigned)((items + 3) / 4)), 256, 0, stream>>>(a, of);
  return hipGetLastError();
}

template <int D>
hipError_t launch(const SharedArgs& a, const SharedPlan& p, hipStream_t stream) {
  const PrefixPieces of = {p.prefix.tiles, p.prefix.chunk, p.prefix.splits, a.part};
  const SharedWork w = shared_work(a, p);
  const unsigned workgroups = (unsigned)shared_workgroups(w);
  SharedArgs own = a;
  own.part = a.part + p.prefix_bytes / sizeof(float);
  constexpr int kMore = D == 64 ? 2 : D == 128 ? 3 : 8, kMoreOwn = D == 256 ? 8 : 2;
  hipError_t e = hipErrorInvalidValue;      // (by the plan, never)
  if (p.own.tiles == kMoreOwn && p.prefix.tiles == kMore) e = launch_passes<D, kMore, kMoreOwn>(own, of, w, workgroups, stream);
  if (p.own.tiles == 1 && p.prefix.tiles == 1) e = launch_passes<D, 1, 1>(own, of, w, workgroups, stream);
  if constexpr (D < 256) {
    if (p.own.tiles == 1 && p.prefix.tiles == kMore) e = launch_passes<D, kMore, 1>(own, of, w, workgroups, stream);
  }
  return e != hipSuccess ? e : launch_join<D>(own, of, p.join_share, stream);
}

}  // namespace

hipError_t launch_kv_attention_shared(const SharedArgs& args, const SharedPlan& p, hipStream_t stream) {
  SharedArgs a = args;
  if (p.apart) {
    a.row_tiles = p.whole.tiles;
    a.waves = p.whole.waves;
    a.chunk = p.whole.chunk;
    a.splits = p.whole.splits;
    return launch_kv_attention(a, a.part, p.bytes, stream);
  }
  a.row_tiles = p.own.tiles;
  a.waves = p.own.waves;
  a.chunk = p.own.chunk;
  a.splits = p.own.splits;
  return a.cache.dim == 64 ? launch<64>(a, p, stream) : a.cache.dim == 128 ? launch<128>(a, p, stream) : launch<256>(a, p, stream);
}

}  // namespace nvfp4
