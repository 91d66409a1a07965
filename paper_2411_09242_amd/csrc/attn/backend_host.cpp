// Host-only library: arguments are checked, then there is no GPU to run on.
#include "../host/common.h"
#include "backend.h"

namespace fluid {

namespace {
[[noreturn]] void unsupported(const char* what) {
  fail(FLUID_E_UNSUPPORTED, std::string(what) + ": not available in the host-only library (no GPU code)");
}
}  // namespace

void run_kv_io(const KvIoParams&, int, int, bool write, void*) { unsupported(write ? "fluid_kv_write" : "fluid_kv_read"); }
void run_kv_attention(const AttnParams&, int, int, void*) { unsupported("fluid_kv_attention"); }
void run_attention(const AttnParams&, int, int, void*) { unsupported("fluid_attention"); }

}  // namespace fluid
