// Launchers of the cache and attention kernels; each returns the launch status.
#pragma once

#include <hip/hip_runtime.h>

#include "params.h"

namespace fluid {

hipError_t launch_kv_io(const KvIoParams& p, int dtype, int head_dim, bool write, hipStream_t s);
hipError_t launch_kv_attention(const AttnParams& p, int dtype, int head_dim, hipStream_t s);
hipError_t launch_attention_bf16(const AttnParams& p, int head_dim, hipStream_t s);
hipError_t launch_attention_f32(const AttnParams& p, int head_dim, hipStream_t s);
hipError_t launch_attention(const AttnParams& p, int dtype, int head_dim, hipStream_t s);

// Joins the shares of split rows (splits > 1), after either of the above.
hipError_t launch_attention_join(const AttnParams& p, int dtype, int head_dim, hipStream_t s);

}  // namespace fluid
