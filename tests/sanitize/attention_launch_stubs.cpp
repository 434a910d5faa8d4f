// Host-only stand-ins for the attention launchers (csrc/attention_launch.h),
// so that the validation layer (csrc/attention_api.cpp) can be built for the
// CPU with sanitizers.  Without a device, every call that passes validation
// stops at the device check, so none is reached.
#include "attention_launch.h"

namespace nvfp4 {

hipError_t launch_qk_norm_rope(const NormRopeArgs&, int, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv_append(const AppendArgs&, hipStream_t) { return hipErrorNoDevice; }
size_t kv_attention_workspace_bytes(const KvCacheArgs&, const KvBatchArgs& b, int) {
  return b.max_kv_len > 1024 ? 4096 : 0;
}
hipError_t launch_kv_attention(const AttentionArgs&, void*, size_t, hipStream_t) { return hipErrorNoDevice; }

}  // namespace nvfp4
