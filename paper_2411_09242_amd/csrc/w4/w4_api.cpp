// Entry points of fluid_w4.h: argument checks and launch sizes.
#include "fluid_w4.h"

#include <algorithm>
#include <cstdint>

#include "../host/handles.h"
#include "../host/kparams.h"
#include "w4_backend.h"

namespace fluid {

namespace {

W4Params check_shape(const fluid_w4* w) {
  require(w != nullptr, "w: NULL");
  require(w->rows >= 1 && w->cols >= 1, "w: rows and cols must be at least 1");
  require(w->group == 32 || w->group == 64 || w->group == 128, "w: group must be 32, 64 or 128");
  require(w->rows <= 1 << 30 && w->cols <= 1 << 30, "w: more than 2^30 rows or cols");
  W4Params p{};
  p.n = w->rows;
  p.k = w->cols;
  p.group = w->group;
  p.tiles = (w->rows + 15) / 16;
  p.blocks = (w->cols + 127) / 128;
  return p;
}
int64_t word_bytes(const W4Params& p) { return int64_t(p.tiles) * p.blocks * 1024; }
uint64_t bytes_of(const W4Params& p) {
  return uint64_t(word_bytes(p)) + uint64_t(p.tiles) * p.blocks * 64 * (128 / p.group);
}
W4Arg held(const W4Params& p, const void* packed, const char* name) {
  require(packed != nullptr, name, ": NULL data");
  require((uintptr_t)packed % 16 == 0, name, ": must be 16-byte aligned");
  return {(const uint8_t*)packed, (const uint8_t*)packed + word_bytes(p)};
}

// Stride of a matrix's rows, in elements.
int64_t check_sizes(const fluid_matrix* d, int32_t cols, const char* name) {
  require(d != nullptr, name, ": NULL description");
  require(d->dtype == FLUID_F32 || d->dtype == FLUID_BF16, name, ": dtype must be f32 or bf16");
  require(d->rows >= 1 && d->cols >= 1, name, ": rows and cols must be at least 1");
  require(d->cols == cols, name, ": cols do not fit the matrix");
  if (d->rows == 1) return 0;
  require(d->stride >= 0 && d->stride <= (int64_t(1) << 40), name, ": stride must lie in 0 .. 2^40");
  return d->stride;
}
int64_t check_matrix(const fluid_matrix* d, const void* data, int32_t cols, const char* name) {
  const int64_t stride = check_sizes(d, cols, name);
  require(data != nullptr, name, ": NULL data");
  require((uintptr_t)data % dtype_bytes(d->dtype) == 0, name, ": misaligned for its type");
  return stride;
}
void check_apart(const fluid_matrix* d, const char* name) {
  require(d->rows == 1 || d->stride >= d->cols, name, ": an output's stride must be at least its cols");
}

// How the channels are shared.
void plan_product(W4Params& p, int32_t rows, bool gate, int dtype) {
  p.m = rows;
  require(rows <= 64 * 65535, "x: too many rows for one launch");
  require(int64_t(p.tiles) * 1024 < int64_t(1) << 32, "w: too large for one launch");
  // 4096 x 11008, 17 and 32 bf16 rows: 13.0 and 14.4 us in one launch, 16.6 in two; fp32,
  // 32 rows: 37 and 25.6.
  if (rows <= (dtype == FLUID_BF16 ? 32 : 16)) {
    // Two tiles to a workgroup share x where there are enough: 8192 x 4096, eight rows 7.5
    // us, with one tile 8.4; one row times 32000 x 4096 14.4 and 16.5, but 11008 x 4096
    // 8.4 and 7.9; 4096 x 11008, 256 tiles, 11.8 and 7.1.  Then, and with a gate, four
    // wavefronts hold the registers for it (32000 x 1024 6.7 us, with eight 7.3; 32 rows 12.2
    // and 15.7); else sixteen, which take fewer blocks each (4096 x 11008, eight rows 8.4
    // us, with eight 8.9).  fp32 x and 32 rows have no room for sixteen.
    p.wide = p.tiles >= (rows > 4 ? 512 : 1024) && !gate;
    const bool many = gate || p.wide;
    p.waves = p.blocks < 8 || (many && dtype == FLUID_BF16) ? 4 : p.blocks < 16 || rows > 16 || dtype != FLUID_BF16 ? 8 : 16;
    return;
  }
  // As many runs as make a workgroup to a compute unit, of four blocks or more: 64
  // rows times 4096 x 11008 take 23 us in 256 workgroups, 28 in 512, 30 in 128.
  const int64_t groups = (int64_t(p.tiles) + 7) / 8 * ((rows + 63) / 64);
  const int64_t runs = std::max<int64_t>(1, std::min<int64_t>(256 / groups, p.blocks / 4));
  p.run = (int32_t)((p.blocks + runs - 1) / runs);
  p.splits = (p.blocks + p.run - 1) / p.run;
}
uint64_t workspace_of(const W4Params& p, bool gate) {
  return p.splits <= 1 ? 0 : uint64_t(p.splits) * (gate ? 2 : 1) * p.m * p.n * 4;
}

}  // namespace

}  // namespace fluid

using namespace fluid;

extern "C" {

fluid_status fluid_w4_bytes(const fluid_w4* w, uint64_t* bytes) {
  return call_guarded([&] {
    const W4Params p = check_shape(w);
    require(bytes != nullptr, "bytes: NULL");
    *bytes = bytes_of(p);
  });
}

fluid_status fluid_w4_pack(const fluid_w4* w, const fluid_matrix* md, const void* m, void* packed, void* hip_stream) {
  return call_guarded([&] {
    W4Params p = check_shape(w);
    p.w = held(p, packed, "packed");
    p.xs = check_matrix(md, m, w->cols, "m");
    require(md->rows == w->rows, "m: rows do not fit the matrix");
    require(int64_t(p.tiles) * p.blocks <= int64_t(1) << 23, "w: too large for one launch");
    p.x = m;
    run_w4_pack(p, md->dtype, hip_stream);
  });
}

fluid_status fluid_w4_read(const fluid_w4* w, const void* packed, const fluid_matrix* md, void* m, void* hip_stream) {
  return call_guarded([&] {
    W4Params p = check_shape(w);
    p.w = held(p, packed, "packed");
    p.os = check_matrix(md, m, w->cols, "m");
    require(md->rows == w->rows, "m: rows do not fit the matrix");
    check_apart(md, "m");
    require(int64_t(p.tiles) * p.blocks <= int64_t(1) << 23, "w: too large for one launch");
    p.out = m;
    run_w4_read(p, md->dtype, hip_stream);
  });
}

fluid_status fluid_w4_matmul_workspace(const fluid_w4* w, const fluid_matrix* xd, int32_t gated, uint64_t* bytes) {
  return call_guarded([&] {
    W4Params p = check_shape(w);
    check_sizes(xd, w->cols, "x");
    require(gated == 0 || gated == 1, "gated must be 0 or 1");
    require(bytes != nullptr, "bytes: NULL");
    plan_product(p, xd->rows, gated, xd->dtype);
    *bytes = workspace_of(p, gated);
  });
}

fluid_status fluid_w4_matmul(const fluid_w4* w, const void* packed, const void* gate, const fluid_matrix* xd,
                             const void* x, const fluid_matrix* ad, const void* add, const fluid_matrix* od, void* out,
                             void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  return call_guarded([&] {
    W4Params p = check_shape(w);
    p.w = held(p, packed, "packed");
    if (gate != nullptr) p.gate = held(p, gate, "gate");
    p.xs = check_matrix(xd, x, w->cols, "x");
    p.os = check_matrix(od, out, w->rows, "out");
    require(od->dtype == xd->dtype && od->rows == xd->rows, "out must have x's dtype and rows");
    check_apart(od, "out");
    if (add != nullptr) {
      p.as = check_matrix(ad, add, w->rows, "add");
      require(ad->dtype == xd->dtype && ad->rows == xd->rows, "add must have x's dtype and rows");
      require(add != out || p.as == p.os, "out: where it is add it must have its stride");
    }
    require(out != x, "out must not be x");
    plan_product(p, xd->rows, gate != nullptr, xd->dtype);
    p.x = x;
    p.add = add;
    p.out = out;
    const uint64_t need = workspace_of(p, gate != nullptr);
    if (need) {
      if (workspace == nullptr || workspace_bytes < need)
        fail(FLUID_E_ARENA_TOO_SMALL, "workspace: " + std::to_string(need) + " bytes needed, " +
                                          std::to_string(workspace ? workspace_bytes : 0) + " given");
      require((uintptr_t)workspace % 256 == 0, "workspace: must be 256-byte aligned");
      p.ws = (float*)workspace;
    }
    run_w4_matmul(p, xd->dtype, hip_stream);
  });
}

}  // extern "C"
