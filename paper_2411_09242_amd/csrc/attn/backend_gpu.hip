// GPU library: kernels on the caller's stream.
#include "../host/common.h"
#include "backend.h"
#include "launch_attn.h"

namespace fluid {

namespace {
void check(hipError_t e, const char* what) {
  if (e != hipSuccess) fail(FLUID_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}
}  // namespace

void run_kv_io(const KvIoParams& p, int dtype, int head_dim, bool write, void* stream) {
  check(launch_kv_io(p, dtype, head_dim, write, (hipStream_t)stream), write ? "fluid_kv_write" : "fluid_kv_read");
}
void run_kv_attention(const AttnParams& p, int dtype, int head_dim, void* stream) {
  check(launch_kv_attention(p, dtype, head_dim, (hipStream_t)stream), "fluid_kv_attention");
}
void run_attention(const AttnParams& p, int dtype, int head_dim, void* stream) {
  check(launch_attention(p, dtype, head_dim, (hipStream_t)stream), "fluid_attention");
}

}  // namespace fluid
