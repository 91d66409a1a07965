// Linear attention: argument checks and launch sizes.
#include <algorithm>

#include "../host/handles.h"
#include "backend.h"
#include "check_tokens.h"

namespace fluid {

namespace {

LinearParams plan_linear(const fluid_tokens* qd, const fluid_tokens* kd) {
  require(qd->dtype == kd->dtype && qd->batch == kd->batch && qd->tokens == kd->tokens && qd->head_dim == kd->head_dim,
          "q and k must have one dtype, batch, tokens and head_dim");
  require(qd->heads % kd->heads == 0, "q: heads must be a multiple of k's");
  LinearParams p{};
  p.batch = qd->batch;
  p.tokens = qd->tokens;
  p.kv_heads = kd->heads;
  p.group = qd->heads / kd->heads;
  p.div_heads = make_fastdiv(p.kv_heads);
  // a workgroup of 256 threads to 32 columns of a state
  const int64_t heads = product({p.batch, p.kv_heads});
  require(product({heads, kd->head_dim / 32, 256}) <= kMostThreads, "q: too large for one launch");
  // Token after token where they are few: 4 tokens of 256 heads of 128 11.3 us, in a
  // chunk 13.0; 8 of them 15.9 and 13.0; 2 tokens of 1024 heads 30 and 43.  The chunk's
  // workgroups take a query head each: 3 tokens of four heads to a state (128 states)
  // 12.5 and 13.3, 4 of them 16.0 and 15.7.
  if (p.tokens <= 2 || int64_t(p.tokens) * p.group <= 4) return p;
  // Runs of two chunks or more, that make two workgroups to a compute unit: 8192
  // tokens of 32 heads of 128 take 140 us with 512, 145 with 256, 156 with 1024; 8 x 512
  // ragged fp32 tokens of 16 heads of 64 30, 39 and 29.
  const int chunk = linear_chunk(qd->dtype);
  const int64_t chunks = (int64_t(p.tokens) + chunk - 1) / chunk;
  const int64_t runs = std::max<int64_t>(1, std::min<int64_t>(512 / (heads * p.group), chunks / 2));
  require(p.group < 65536, "q: more than 65535 heads to one of k's");
  const int64_t each = (chunks + runs - 1) / runs;
  p.run = (int32_t)(each * chunk);
  p.segments = (int32_t)((chunks + each - 1) / each);
  // every query head's workgroups read the states of the runs before theirs: 32 heads
  // over 8 key heads in 16 runs 108 us, with a scan between the launches 101; 64 heads
  // in 8 runs 34 and 36.  One run has nothing before it; with more there are at most
  // 256 states, rows of the scan's grid.
  p.scan = p.segments > 1 && int64_t(p.group) * p.segments > 24;
  return p;
}
uint64_t workspace_of(const LinearParams& p, int head_dim) {
  // one run's state has a place where several heads start from it: it may be
  // overwritten
  const bool none = p.segments == 0 || (p.segments == 1 && p.group == 1);
  return none ? 0 : uint64_t(p.batch) * p.kv_heads * p.segments * (head_dim * head_dim + 1) * 4;
}

}  // namespace

}  // namespace fluid

using namespace fluid;

extern "C" {

fluid_status fluid_linear_attention_workspace(const fluid_tokens* qd, const fluid_tokens* kd, uint64_t* bytes) {
  return call_guarded([&] {
    tokens_arg(qd, nullptr, "q");
    tokens_arg(kd, nullptr, "k");
    require(bytes != nullptr, "bytes: NULL");
    *bytes = workspace_of(plan_linear(qd, kd), qd->head_dim);
  });
}

fluid_status fluid_linear_attention(float scale, const fluid_tokens* qd, const void* q, const fluid_tokens* kd,
                                    const void* k, const fluid_tokens* vd, const void* v, const float* decay,
                                    const int64_t decay_stride[3], const float* state, const int32_t* count,
                                    const fluid_tokens* od, void* out, float* state_out, void* workspace,
                                    uint64_t workspace_bytes, void* hip_stream) {
  return call_guarded([&] {
    const TokensArg qa = tokens_data(qd, q, "q"), ka = tokens_data(kd, k, "k"), va = tokens_data(vd, v, "v"),
                    oa = tokens_data(od, out, "out");
    require(od->dtype == qd->dtype && od->batch == qd->batch && od->tokens == qd->tokens && od->heads == qd->heads &&
                od->head_dim == qd->head_dim,
            "out must have q's dtype and shape");
    require(kd->dtype == vd->dtype && kd->batch == vd->batch && kd->tokens == vd->tokens && kd->heads == vd->heads &&
                kd->head_dim == vd->head_dim,
            "k and v must have one dtype and shape");
    require(scale - scale == 0.0f, "scale must be finite");
    LinearParams p = plan_linear(qd, kd);
    check_apart(od, "out");
    require(decay != nullptr && (uintptr_t)decay % 4 == 0, "decay: NULL or misaligned");
    require(decay_stride != nullptr, "decay_stride: NULL");
    for (int i = 0; i < 3; ++i)
      require(decay_stride[i] >= 0 && decay_stride[i] <= (int64_t(1) << 40), "decay: strides must lie in 0 .. 2^40");
    require((uintptr_t)state % 16 == 0 && (uintptr_t)state_out % 16 == 0, "state: must be 16-byte aligned");
    // workgroups read these while others write
    require(out != q && out != k && out != v, "out: must not be q, k or v");
    const uintptr_t from = (uintptr_t)state, to = (uintptr_t)state_out,
                    bytes = (uintptr_t)product({p.batch, p.kv_heads, qd->head_dim, qd->head_dim, 4});
    require(!state || !state_out || from == to || (from < to ? to - from : from - to) >= bytes,
            "state_out: must be state or apart from it");
    p.q = qa;
    p.k = ka;
    p.v = va;
    p.o = oa;
    p.decay = decay;
    p.gb = decay_stride[0];
    p.gt = decay_stride[1];
    p.gh = decay_stride[2];
    p.state = state;
    p.state_out = state_out;
    p.count = count;
    p.scale = scale;
    // the state to start from is read by others than write the last one
    p.slots = p.segments > 1 || (p.segments == 1 && p.group > 1 && state != nullptr && state == state_out);
    const uint64_t need = workspace_of(p, qd->head_dim);
    if (need) {
      if (workspace == nullptr || workspace_bytes < need)
        fail(FLUID_E_ARENA_TOO_SMALL, "workspace: " + std::to_string(need) + " bytes needed, " +
                                          std::to_string(workspace ? workspace_bytes : 0) + " given");
      require((uintptr_t)workspace % 256 == 0, "workspace: must be 256-byte aligned");
      p.ws = (float*)workspace;
    }
    run_linear_attention(p, qd->dtype, qd->head_dim, hip_stream);
  });
}

}  // extern "C"
