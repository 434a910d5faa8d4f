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
  attention_rows_kernel<D, kTiles, kWaves, kSplit>(a);
}

template <int D, int kTiles, int kShare>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(AttentionArgs a) {
  attention_join<D, kTiles, kShare>(a);
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
