// Attention of each row over the pages chosen for it (definition: nvfp4_paging.h), for
// gfx950: the attention's kernels, with each row and key head as a sequence of its own
// whose pages stand in the choice and not in a table.  Bound by the chosen pages' bytes where
// there are many rows (32 rows, 8 key heads of 128, 128 pages of 16 each: 24.4 us, 5.5 TB/s), else
// by a launch and the chain choice, codes, join (one row, 64 pages of 64: 6.3 and 3.4 us).
#include "attention_plan.h"
#include "kv_attention_rows.h"
#include "kv_attention_wide.h"
#include "paging_launch.h"

namespace nvfp4 {

template <int kRows>
__device__ __forceinline__ bool find_tile(const SelectedArgs& a, int number, Tile& t) {
  const int each = (a.group + kRows - 1) / kRows, row = __builtin_amdgcn_readfirstlane(number / each);
  const int tokens = a.batch.kv_len[row];
  if (tokens < 0) return false;      // behind the last sequence
  t.b = t.row0 = row;
  t.rows = 1;
  t.first = 0;
  t.r0 = (number - row * each) * kRows;
  t.n = min(kRows, a.group - t.r0);
  t.begin = 0;
  t.end = min(tokens, a.batch.max_tokens);
  return true;
}

__device__ __forceinline__ GroupPages group_pages(const SelectedArgs& a, int b, int h, int64_t token, int begin, int end) {
  GroupPages g;
  g.page = -1;
  g.k_scale = g.v_scale = 0.0f;
  if (token < end && token + 16 > begin) {
    const int p = a.pages[((int64_t)b * a.cache.heads + h) * a.count + (token >> a.cache.page_shift)];
    if (p >= 0 && p < a.cache.num_pages) {
      g.page = p;
      g.k_scale = a.cache.scale[0][(int64_t)p * a.cache.scale_stride + h];
      g.v_scale = a.cache.scale[1][(int64_t)p * a.cache.scale_stride + h];
    }
  }
  return g;
}

template <int D, int kTiles, int kWaves, bool kSplit>
__global__ __launch_bounds__(kWaves * 64, rows_waves(D, kTiles, kWaves, kSplit)) void kv_selected_rows_kernel(SelectedArgs a) {
  attention_rows_kernel<D, kTiles, kWaves, kSplit>(a);
}

template <int D>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void kv_selected_tile_kernel(SelectedArgs a, int tiles) {
  attention_tile_kernel<D, true>(a, tiles);
}

template <int D, int kTiles, int kShare>
__global__ __launch_bounds__(256) void kv_selected_join_kernel(SelectedArgs a) {
  attention_join<D, kTiles, kShare>(a);
}

namespace {

template <int D, int kTiles>
hipError_t launch_join(const SelectedArgs& a, int64_t work, hipStream_t stream) {
  if (a.splits == 1) return hipSuccess;
  if (a.splits > 8)
    kv_selected_join_kernel<D, kTiles, 4><<<dim3((unsigned)(work * 16 * kTiles)), 256, 0, stream>>>(a);
  else
    kv_selected_join_kernel<D, kTiles, 1><<<dim3((unsigned)(work * 4 * kTiles)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch(const SelectedArgs& a, hipStream_t stream) {
  const int64_t tiles = host_tiles(a.batch, a.group, 16 * a.row_tiles), work = tiles * a.cache.heads;
  const dim3 grid((unsigned)(work * a.splits));
  if (a.row_tiles == 8)
    kv_selected_tile_kernel<D><<<grid, 256, 0, stream>>>(a, (int)tiles);
  else if (a.row_tiles == 2)
    kv_selected_rows_kernel<D, 2, 4, true><<<grid, 256, 0, stream>>>(a);
  else if (a.waves == 8)
    kv_selected_rows_kernel<D, 1, 8, false><<<grid, 512, 0, stream>>>(a);
  else if (a.splits > 1)
    kv_selected_rows_kernel<D, 1, 4, true><<<grid, 256, 0, stream>>>(a);
  else
    kv_selected_rows_kernel<D, 1, 4, false><<<grid, 256, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return a.row_tiles == 8   ? launch_join<D, 8>(a, work, stream)
         : a.row_tiles == 2 ? launch_join<D, 2>(a, work, stream)
                            : launch_join<D, 1>(a, work, stream);
}

}  // namespace

hipError_t launch_kv_attention_selected(const SelectedArgs& a, hipStream_t stream) {
  return a.cache.dim == 64 ? launch<64>(a, stream) : a.cache.dim == 128 ? launch<128>(a, stream) : launch<256>(a, stream);
}

}  // namespace nvfp4
