// What the entry points call once arguments are checked: kernels in the GPU
// library, FLUID_E_UNSUPPORTED in the host-only one.
#pragma once

#include "params.h"

namespace fluid {

void run_kv_io(const KvIoParams& p, int dtype, int head_dim, bool write, void* stream);
void run_kv_attention(const AttnParams& p, int dtype, int head_dim, void* stream);
void run_attention(const AttnParams& p, int dtype, int head_dim, void* stream);

}  // namespace fluid
