// Launchers of the attention kernels (called by attention_api.cpp after
// argument validation) and the parameters they pass by value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nvfp4 {

// The rotation of a head's first rot elements (rot 0: none).
struct RopeArgs {
  const int32_t* positions;
  const float* inv_freq;
  int rot;
  int interleaved;
};

struct NormRopeArgs {
  const uint16_t* x[2];        // queries, keys
  uint16_t* y[2];
  const uint16_t* gamma[2];
  int64_t ldx[2], ldy[2];
  int heads[2];
  int rows;
  float eps;
  RopeArgs rope;
};

struct KvCacheArgs {
  uint8_t* kv[2];              // keys, values
  float* scale[2];
  int64_t page_stride[2];
  int64_t scale_stride;
  int num_pages, page_size, page_shift, heads, dim;
};

struct KvBatchArgs {
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* cu_rows;      // null: one row for each sequence
  int64_t table_stride;
  int max_tokens;              // max_pages * page_size
  int seqs, rows;
  int max_kv_len;
};

struct AppendArgs {
  KvCacheArgs cache;
  KvBatchArgs batch;
  const uint16_t* x[2];
  int64_t ld[2];
  const uint16_t* gamma;
  float eps;
  RopeArgs rope;
  int dynamic;
};

struct AttentionArgs {
  static constexpr bool kParts = false;      // a piece that is all its rows see writes their results
  KvCacheArgs cache;
  KvBatchArgs batch;
  const uint16_t* q;
  uint16_t* y;
  float* lse;
  int64_t ldq, ldy;
  int q_heads, group;          // group = q_heads / kv_heads
  float scale;                 // softmax_scale * log2(e)
  int causal, window;
  int row_tiles, waves;        // of a workgroup, and
  int chunk, splits;           // tokens of one piece of a sequence, pieces (attention_plan.h)
  float* part;                 // partial results (launcher)
};

hipError_t launch_qk_norm_rope(const NormRopeArgs& a, int dim, hipStream_t stream);
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream);
// The attention of many rows in tiles of 128 packed rows (kv_attention_tile.hip;
// called by launch_kv_attention, which joins the pieces).
hipError_t launch_kv_attention_tile(const AttentionArgs& a, int64_t tiles, hipStream_t stream);
hipError_t launch_kv_attention(const AttentionArgs& a, void* workspace, size_t workspace_bytes, hipStream_t stream);

// attention_api.cpp and api.cpp share the device check and the record of the
// last HIP error (api.cpp).
int check_device();
int fail_hip(hipError_t e);

}  // namespace nvfp4
