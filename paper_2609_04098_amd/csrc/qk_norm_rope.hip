// RMSNorm of query and key heads with the rotation of their first elements, in
// one pass, for gfx950.
//
//   y = x * gamma / sqrt(sum x^2 / D + eps), then for the pairs (a, b) of the
//   rotation  (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin)
//
// Bound by HBM (2 D bytes read and written per head).  A lane holds 8 elements
// (one 16-byte load), D / 8 lanes a head, so that a wave works on 512 / D heads
// at a time and the sum of squares is a butterfly over D / 8 lanes.  A wave
// takes several heads of ONE row: the row's sines and cosines (rot / 2 of them,
// one or two a lane) are computed once, go through LDS to the lanes that need
// them and stay in registers for all its heads.  8175 rows of 28 heads of 256:
// 40 us, 5.8 TB/s read and written.
#include "attention_device.h"

namespace nvfp4 {

constexpr int kNormRopeThreads = 256;
constexpr int kInFlight = 4;           // heads of one lane group whose loads are in flight together

template <int D>
__global__ __launch_bounds__(kNormRopeThreads) void qk_norm_rope_kernel(NormRopeArgs a, int chunks, int per_chunk) {
  constexpr int kLanes = D / 8, kHeads = 64 / kLanes;
  __shared__ float2 turn[kNormRopeThreads / 64][D / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t task = (int64_t)blockIdx.x * (kNormRopeThreads / 64) + wave;
  const int64_t row = task / chunks;
  if (row >= a.rows) return;
  const int chunk = (int)(task % chunks);
  const int e0 = (lane % kLanes) * 8, rot = a.rope.rot, half = rot / 2;
  const int heads = a.heads[0] + a.heads[1];

  // This lane's cos and signed sin, and where each element's partner is.
  float c[8], s[8];
  int partner = lane;
#pragma unroll
  for (int j = 0; j < 8; ++j) c[j] = 1.0f, s[j] = 0.0f;
  if (rot > 0) {
    const int pos = a.rope.positions[row];
    for (int i = lane; i < half; i += 64) {
      float si, co;
      sin_cos<float>(pos, a.rope.inv_freq[i], si, co);
      turn[wave][i] = make_float2(co, si);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (e0 < rot) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = e0 + j;
        const bool second = a.rope.interleaved ? (j & 1) : e >= half;
        const float2 t = turn[wave][a.rope.interleaved ? e / 2 : (second ? e - half : e)];
        c[j] = t.x;
        s[j] = second ? t.y : -t.y;
      }
      if (!a.rope.interleaved) partner = lane + (e0 < half ? half / 8 : -(half / 8));
    }
  }
  uint32_t gamma[2][4];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    uint4 g = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);      // ones
    if (a.gamma[w] != nullptr) g = *reinterpret_cast<const uint4*>(a.gamma[w] + e0);
    gamma[w][0] = g.x, gamma[w][1] = g.y, gamma[w][2] = g.z, gamma[w][3] = g.w;
  }

  const int h_end = min(heads, (chunk + 1) * per_chunk * kHeads);
  for (int h0 = chunk * per_chunk * kHeads + lane / kLanes; h0 - lane / kLanes < h_end; h0 += kInFlight * kHeads) {
    uint4 in[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int h = h0 + u * kHeads;
      in[u] = make_uint4(0, 0, 0, 0);
      if (h < h_end) {
        const uint16_t* x = h < a.heads[0] ? a.x[0] + row * a.ldx[0] + (int64_t)h * D
                                           : a.x[1] + row * a.ldx[1] + (int64_t)(h - a.heads[0]) * D;
        in[u] = *reinterpret_cast<const uint4*>(x + e0);
      }
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int h = h0 + u * kHeads;
      const bool key = h >= a.heads[0];
      if (h - lane / kLanes >= h_end) break;           // (the same for the whole wave)
      const uint32_t d[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
      float v[8], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[2 * j] = bf16_low(d[j]), v[2 * j + 1] = bf16_high(d[j]);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
#pragma unroll
      for (int m = 1; m < kLanes; m *= 2) sum += __shfl_xor(sum, m);
      if ((key ? a.gamma[1] : a.gamma[0]) != nullptr) {
        const float r = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t g = key ? gamma[1][j] : gamma[0][j];
          v[2 * j] = v[2 * j] * r * bf16_low(g);
          v[2 * j + 1] = v[2 * j + 1] * r * bf16_high(g);
        }
      }
      if (rot > 0) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = a.rope.interleaved ? v[j ^ 1] : __shfl(v[j], partner);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j], c[j], p[j] * s[j]);
      }
      uint16_t* y = key ? a.y[1] + row * a.ldy[1] + (int64_t)(h - a.heads[0]) * D
                        : a.y[0] + row * a.ldy[0] + (int64_t)h * D;
      if (h < h_end)
        *reinterpret_cast<uint4*>(y + e0) =
            make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
  }
}

// The heads of a row are divided over waves where there are few rows: up to
// 8192 waves (8 per SIMD), each with at least one group of heads.
hipError_t launch_qk_norm_rope(const NormRopeArgs& a, int dim, hipStream_t stream) {
  const int groups = (a.heads[0] + a.heads[1] + 512 / dim - 1) / (512 / dim);
  int chunks = (8192 + a.rows - 1) / a.rows;
  chunks = chunks > groups ? groups : chunks;
  const int per_chunk = (groups + chunks - 1) / chunks;
  chunks = (groups + per_chunk - 1) / per_chunk;
  const int64_t blocks = ((int64_t)a.rows * chunks + kNormRopeThreads / 64 - 1) / (kNormRopeThreads / 64);
  const dim3 grid((unsigned)blocks);
  if (dim == 64)
    qk_norm_rope_kernel<64><<<grid, kNormRopeThreads, 0, stream>>>(a, chunks, per_chunk);
  else if (dim == 128)
    qk_norm_rope_kernel<128><<<grid, kNormRopeThreads, 0, stream>>>(a, chunks, per_chunk);
  else
    qk_norm_rope_kernel<256><<<grid, kNormRopeThreads, 0, stream>>>(a, chunks, per_chunk);
  return hipGetLastError();
}

}  // namespace nvfp4
