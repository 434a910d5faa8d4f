// Attention of many rows (prompts) over the paged E4M3 cache for gfx950 (layout
// and definition: nvfp4_attention.h).
//
// A workgroup takes 128 packed rows of one sequence and key head, 32 a wave.
// Keys and values go through LDS as they are (E4M3) in tiles of 64 tokens,
// loaded by direct loads one tile ahead and read by all four waves.
//
// Bound by the instructions that a SIMD issues (one in four cycles, vector or
// matrix; an exponential takes two turns), 168 vector and 16 matrix instructions
// for 32 rows, 32 tokens and a head of 128: 8192 tokens, 40 heads of 128, causal,
// take 705 us, 0.97 PFLOP/s, with the vector units busy 74% of the time and the
// matrix units 46%.  So the products are the largest there are:
//   S^T = K Q^T by v_mfma_f32_32x32x16_bf16, Y^T += V^T P^T by
//   v_mfma_f32_32x32x16_f16, on keys and values converted on the way.
// With the products transposed a lane holds the scores of ONE row, for the
// tokens 8 x + 4 h .. + 3 (h = lane / 32, x = 0 .. 3) of 32, and the second
// product wants just these of it: of 16 tokens, its contraction indexes 8 h + e
// and 8 h + 4 + e are the tokens 4 h + e and 8 + 4 h + e.  So P never leaves its
// lane.  (The keys as they are, with Q in two E4M3 parts, by
// v_mfma_scale_f32_32x32x64_f8f6f4 would take 32 conversions of 184 instructions
// off; that instruction drops what is 2^-16 below the largest of 8 products.)
// (At 690 us: 64 tokens a pass, two score tiles in registers and two waves a SIMD, 739;
// keys and values converted once into LDS for the four waves, 857.)
//
// Running maximum, sums and scales: as in kv_attention_device.h.
#include "kv_attention_wide.h"

namespace nvfp4 {

template <int D, bool kSplit>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void kv_attention_tile_kernel(AttentionArgs a, int tiles) {
  attention_tile_kernel<D, kSplit>(a, tiles);
}

template <int D>
static hipError_t launch(const AttentionArgs& a, int64_t tiles, hipStream_t stream) {
  const int64_t work = tiles * a.cache.heads;
  if (a.splits == 1)
    kv_attention_tile_kernel<D, false><<<dim3((unsigned)work), 256, 0, stream>>>(a, (int)tiles);
  else
    kv_attention_tile_kernel<D, true><<<dim3((unsigned)(work * a.splits)), 256, 0, stream>>>(a, (int)tiles);
  return hipGetLastError();
}

hipError_t launch_kv_attention_tile(const AttentionArgs& a, int64_t tiles, hipStream_t stream) {
  return a.cache.dim == 64    ? launch<64>(a, tiles, stream)
         : a.cache.dim == 128 ? launch<128>(a, tiles, stream)
                              : launch<256>(a, tiles, stream);
}

}  // namespace nvfp4
