// Append of keys and values to the paged E4M3 cache, keys normed and rotated on
// the way, for gfx950 (layout: nvfp4_attention.h).
//
// One workgroup per touched page, head, and keys or values: it holds all its
// new tokens (at most 16384 elements, 64 a lane) in registers between the
// maximum and the rounding, so the input is read once, no workgroup waits for
// another and the result does not depend on any order.  Codes go through LDS
// into the cache's order and leave it in 16-byte pieces.
//
// Keys are computed in binary64: an 8-bit rounding turns the last bit of a
// binary32 value that is next to a border into a step of 6 to 12 %.  The value
// reaches the rounding as the binary32 number with the sticky last bit (cut
// towards zero, last bit set where anything was cut), whose rounding to E4M3 is
// that of the value itself; a power-of-two scale does not change that.
#include "attention_device.h"

namespace nvfp4 {

constexpr int kAppendThreads = 256;

// The binary32 number next to d towards zero, with its last bit set unless it
// is d itself.
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

__device__ __forceinline__ double shfl_xor_f64(double v, int m) {
  const int lo = __shfl_xor(__double2loint(v), m), hi = __shfl_xor(__double2hiint(v), m);
  return __hiloint2double(hi, lo);
}

__device__ __forceinline__ double shfl_f64(double v, int l) {
  const int lo = __shfl(__double2loint(v), l), hi = __shfl(__double2hiint(v), l);
  return __hiloint2double(hi, lo);
}

// Four codes times the ratio of the old scale to the new one.
__device__ __forceinline__ uint32_t rescaled(uint32_t codes, float ratio) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return e4m3_codes(lo.x * ratio, lo.y * ratio, hi.x * ratio, hi.y * ratio);
}

// kPasses * 2048 / D tokens at most.
template <int D, int kPasses>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs a) {
  constexpr int kLanes = D / 8, kTokens = kAppendThreads / kLanes;        // of one pass
  __shared__ union {
    double2 turn[kTokens * D / 2];
    uint8_t codes[kPasses * kTokens * D];
  } lds;
  __shared__ float wave_max[kAppendThreads / 64];

  const int kind = blockIdx.x & 1;                        // 0: keys, 1: values
  const int h = (int)(blockIdx.x >> 1) % a.cache.heads, item = (int)(blockIdx.x >> 1) / a.cache.heads;
  const int shift = a.cache.page_shift, page_size = a.cache.page_size;

  // Sequence and page: sequence b's pages have the numbers from
  // cu_rows[b] / page_size + 2 b on (n rows reach (n - 1) / page_size + 2 pages).
  int b = item, ordinal = 0;
  if (a.batch.cu_rows != nullptr) {
    int lo = 0, hi = a.batch.seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if ((min(max(a.batch.cu_rows[mid], 0), a.batch.rows) >> shift) + 2 * mid <= item)
        lo = mid;
      else
        hi = mid - 1;
    }
    b = lo;
    ordinal = item - ((min(max(a.batch.cu_rows[b], 0), a.batch.rows) >> shift) + 2 * b);
  }
  const SeqRows s = seq_rows(a.batch, b);
  const int begin = max(s.first, 0);
  const int entry = (begin >> shift) + ordinal;
  const int t0 = max(begin, entry << shift), t1 = min(s.len, (entry + 1) << shift);      // tokens
  if (ordinal < 0 || t0 >= t1 || entry >= (a.batch.max_tokens >> shift)) return;
  const int page = a.batch.table[(int64_t)b * a.batch.table_stride + entry];
  if (page < 0 || page >= a.cache.num_pages) return;
  const int n = t1 - t0, slot0 = t0 - (entry << shift);
  const int row0 = s.row + (t0 - s.first);

  const int lane = threadIdx.x & 63, e0 = (threadIdx.x % kLanes) * 8;
  const int rot = a.rope.rot, half = rot / 2;
  const bool norm = kind == 0 && a.gamma != nullptr, rotate = kind == 0 && rot > 0;
  int partner = lane;
  if (rotate && e0 < rot && !a.rope.interleaved) partner = lane + (e0 < half ? half / 8 : -(half / 8));

  float v[kPasses][8];
  float top = 0.0f;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    if (p * kTokens >= n) break;
    const int i = p * kTokens + threadIdx.x / kLanes;
    uint4 in = make_uint4(0, 0, 0, 0);
    if (i < n)
      in = *reinterpret_cast<const uint4*>(a.x[kind] + (int64_t)(row0 + i) * a.ld[kind] + (int64_t)h * D + e0);
    const uint32_t d[4] = {in.x, in.y, in.z, in.w};
    if (!norm && !rotate) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[p][2 * j] = bf16_low(d[j]), v[p][2 * j + 1] = bf16_high(d[j]);
    } else {
      double w[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[2 * j] = (double)bf16_low(d[j]), w[2 * j + 1] = (double)bf16_high(d[j]);
      if (norm) {
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fma(w[j], w[j], sum);
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) sum += shfl_xor_f64(sum, m);
        const double r = 1.0 / sqrt(sum * (1.0 / D) + (double)a.eps);
        const uint4 g4 = *reinterpret_cast<const uint4*>(a.gamma + e0);
        const uint32_t g[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[2 * j] *= r * (double)bf16_low(g[j]);
          w[2 * j + 1] *= r * (double)bf16_high(g[j]);
        }
      }
      if (rotate) {
        const int tokens = min(kTokens, n - p * kTokens);
        __syncthreads();
        for (int x = threadIdx.x; x < tokens * half; x += kAppendThreads) {
          const int t = x / half, f = x % half, at = p * kTokens + t;
          const int pos = a.rope.positions != nullptr ? a.rope.positions[row0 + at] : t0 + at;
          double si, co;
          sin_cos<double>(pos, a.rope.inv_freq[f], si, co);
          lds.turn[x] = make_double2(co, si);
        }
        __syncthreads();
        double q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = a.rope.interleaved ? w[j ^ 1] : shfl_f64(w[j], partner);
        if (e0 < rot && i < n) {
          const double2* t = lds.turn + (threadIdx.x / kLanes) * half;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int e = e0 + j;
            const bool second = a.rope.interleaved ? (j & 1) : e >= half;
            const double2 cs = t[a.rope.interleaved ? e / 2 : (second ? e - half : e)];
            w[j] = fma(w[j], cs.x, second ? q[j] * cs.y : -(q[j] * cs.y));
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[p][j] = sticky(w[j]);
    }
    if (i < n) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float m = fabsf(v[p][j]);
        if (m <= 3.40282347e38f) top = fmaxf(top, m);      // (a value that is not finite has no part in the scale)
      }
    }
  }

  float* scale_at = a.cache.scale[kind] + (int64_t)page * a.cache.scale_stride + h;
  uint8_t* out = a.cache.kv[kind] + (int64_t)page * a.cache.page_stride[kind] + (int64_t)h * page_size * D;
  float scale;
  if (a.dynamic) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) wave_max[threadIdx.x >> 6] = top;
    const float held = slot0 > 0 ? *scale_at : 0.0f;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAppendThreads / 64; ++w) top = fmaxf(top, wave_max[w]);
    scale = fmaxf(held, page_scale(top));
    if (scale > held && slot0 > 0) {
      // The tokens that the page holds, brought to the grown scale.
      const float ratio = held / scale;
      const int pieces = ((slot0 + 15) / 16) * D;
      for (int x = threadIdx.x; x < pieces; x += kAppendThreads) {
        const int group = x / D, in_group = x % D;
        uint4* at = reinterpret_cast<uint4*>(out) + x;
        if (kind == 0) {
          if (group * 16 + (in_group & 15) < slot0) {
            const uint4 c = *at;
            *at = make_uint4(rescaled(c.x, ratio), rescaled(c.y, ratio), rescaled(c.z, ratio), rescaled(c.w, ratio));
          }
        } else {
          const int held_here = slot0 - (group * 16 + ((in_group >> 4) & 3) * 4);        // of the piece's four tokens
          if (held_here > 0) {
            const uint32_t keep = held_here >= 4 ? 0u : 0xFFFFFFFFu << (8 * held_here);
            const uint4 c = *at;
            *at = make_uint4((c.x & keep) | (rescaled(c.x, ratio) & ~keep), (c.y & keep) | (rescaled(c.y, ratio) & ~keep),
                             (c.z & keep) | (rescaled(c.z, ratio) & ~keep), (c.w & keep) | (rescaled(c.w, ratio) & ~keep));
          }
        }
      }
    }
  } else {
    scale = *scale_at;
  }
  const float inverse = 1.0f / scale;      // exact for the powers of two of the dynamic mode

  __syncthreads();      // the rotation's table has been read, the held codes are written
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    if (p * kTokens >= n) break;
    const int i = p * kTokens + threadIdx.x / kLanes;
    if (i < n) {
      const int t = slot0 + i;
      float q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = a.dynamic ? v[p][j] * inverse : v[p][j] / scale;
        q[j] = fabsf(v[p][j]) <= 3.40282347e38f ? __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f) : __uint_as_float(0x7FC00000u);
      }
      const uint32_t c0 = e4m3_codes(q[0], q[1], q[2], q[3]), c1 = e4m3_codes(q[4], q[5], q[6], q[7]);
      const int base = (t / 16) * 16 * D, u = t % 16;
      if (kind == 0) {
        *reinterpret_cast<uint2*>(lds.codes + base + (e0 / 16) * 256 + u * 16 + (e0 & 8)) = make_uint2(c0, c1);
      } else {
        uint8_t* to = lds.codes + base + (e0 / 64) * 1024 + ((u / 4) * 16 + (e0 & 8)) * 16 + (e0 / 16 % 4) * 4 + u % 4;
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j * 16] = (uint8_t)((j < 4 ? c0 : c1) >> (8 * (j & 3)));
      }
    }
  }
  __syncthreads();
  const int last = slot0 + n;
  for (int x = (slot0 / 16) * D + threadIdx.x; x < ((last + 15) / 16) * D; x += kAppendThreads) {
    const int group = x / D, in_group = x % D;
    const uint4 c = reinterpret_cast<const uint4*>(lds.codes)[x];
    uint4* at = reinterpret_cast<uint4*>(out) + x;
    if (kind == 0) {
      const int t = group * 16 + (in_group & 15);
      if (t >= slot0 && t < last) *at = c;
    } else {
      const int t = group * 16 + ((in_group >> 4) & 3) * 4;
      if (t >= slot0 && t + 4 <= last) {
        *at = c;
      } else {
        const uint32_t word[4] = {c.x, c.y, c.z, c.w};
        uint8_t* bytes = reinterpret_cast<uint8_t*>(at);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (t + u >= slot0 && t + u < last)
#pragma unroll
            for (int j = 0; j < 4; ++j) bytes[j * 4 + u] = (uint8_t)(word[j] >> (8 * u));
      }
    }
  }
  if (a.dynamic && threadIdx.x == 0) *scale_at = scale;
}

template <int D>
hipError_t launch_append(const AppendArgs& a, int64_t blocks, hipStream_t stream) {
  const dim3 grid((unsigned)blocks);
  const int elements = a.cache.page_size * D;
  if (elements <= 2048)
    kv_append_kernel<D, 1><<<grid, kAppendThreads, 0, stream>>>(a);
  else if (elements <= 4096)
    kv_append_kernel<D, 2><<<grid, kAppendThreads, 0, stream>>>(a);
  else if (elements <= 8192)
    kv_append_kernel<D, 4><<<grid, kAppendThreads, 0, stream>>>(a);
  else
    kv_append_kernel<D, 8><<<grid, kAppendThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream) {
  const int64_t items = a.batch.cu_rows == nullptr ? a.batch.seqs
                                                   : (a.batch.rows >> a.cache.page_shift) + 2 * (int64_t)a.batch.seqs;
  const int64_t blocks = items * a.cache.heads * 2;
  if (blocks >= (int64_t)1 << 31) return hipErrorInvalidValue;
  return a.cache.dim == 64    ? launch_append<64>(a, blocks, stream)
         : a.cache.dim == 128 ? launch_append<128>(a, blocks, stream)
                              : launch_append<256>(a, blocks, stream);
}

}  // namespace nvfp4
