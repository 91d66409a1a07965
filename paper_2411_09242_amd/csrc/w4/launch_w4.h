// Launchers of the 4-bit matrix kernels; each returns the launch status.
#pragma once

#include <hip/hip_runtime.h>

#include "params.h"

namespace fluid {

hipError_t launch_w4_pack(const W4Params& p, int dtype, hipStream_t s);
hipError_t launch_w4_read(const W4Params& p, int dtype, hipStream_t s);
hipError_t launch_w4_few(const W4Params& p, int dtype, hipStream_t s);
hipError_t launch_w4_rows(const W4Params& p, int dtype, hipStream_t s);

}  // namespace fluid
