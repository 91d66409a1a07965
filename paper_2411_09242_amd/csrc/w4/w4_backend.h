// What the entry points call once arguments are checked: kernels in the GPU
// library, FLUID_E_UNSUPPORTED in the host-only one.
#pragma once

#include "params.h"

namespace fluid {

void run_w4_pack(const W4Params& p, int dtype, void* stream);
void run_w4_read(const W4Params& p, int dtype, void* stream);
void run_w4_matmul(const W4Params& p, int dtype, void* stream);

}  // namespace fluid
