// Launchers of the kernels behind nvfp4_paging.h (called by paging_api.cpp after
// argument validation) and the parameters they pass by value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention_launch.h"

namespace nvfp4 {

struct TablesArgs {
  int32_t* table;
  int32_t* kv_len;
  int32_t* free_pages;
  int32_t* free_count;
  const int32_t* new_rows;
  const int32_t* drop;         // may be null, and so
  const int32_t* kept;
  int32_t* cu_rows;
  int32_t* positions;          // these two
  int64_t* slots;
  int64_t table_stride;
  int max_pages, seqs, num_pages, page_shift, rows;
  int32_t* plan;               // workspace: step_tables.hip
};

size_t step_tables_workspace_bytes(int64_t seqs);
hipError_t launch_step_tables(const TablesArgs& a, hipStream_t stream);

}  // namespace nvfp4
