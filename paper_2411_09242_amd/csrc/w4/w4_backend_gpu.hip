// GPU library: kernels on the caller's stream.
#include "../host/common.h"
#include "launch_w4.h"
#include "w4_backend.h"

namespace fluid {

namespace {
void check(hipError_t e, const char* what) {
  if (e != hipSuccess) fail(FLUID_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}
}  // namespace

void run_w4_pack(const W4Params& p, int dtype, void* stream) {
  check(launch_w4_pack(p, dtype, (hipStream_t)stream), "fluid_w4_pack");
}
void run_w4_read(const W4Params& p, int dtype, void* stream) {
  check(launch_w4_read(p, dtype, (hipStream_t)stream), "fluid_w4_read");
}
void run_w4_matmul(const W4Params& p, int dtype, void* stream) {
  check((p.splits ? launch_w4_rows : launch_w4_few)(p, dtype, (hipStream_t)stream), "fluid_w4_matmul");
}

}  // namespace fluid
