// Host-only library: arguments are checked, then there is no GPU to run on.
#include "../host/common.h"
#include "w4_backend.h"

namespace fluid {

namespace {
[[noreturn]] void unsupported(const char* what) {
  fail(FLUID_E_UNSUPPORTED, std::string(what) + ": not available in the host-only library (no GPU code)");
}
}  // namespace

void run_w4_pack(const W4Params&, int, void*) { unsupported("fluid_w4_pack"); }
void run_w4_read(const W4Params&, int, void*) { unsupported("fluid_w4_read"); }
void run_w4_matmul(const W4Params&, int, void*) { unsupported("fluid_w4_matmul"); }

}  // namespace fluid
