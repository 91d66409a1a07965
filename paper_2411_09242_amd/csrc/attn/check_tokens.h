// Argument checks shared by the entry points that take tensors of tokens.
#pragma once

#include <cstdint>
#include <initializer_list>

#include "../host/common.h"
#include "fluid_attention.h"
#include "params.h"

namespace fluid {

constexpr int64_t kMostTokens = int64_t(1) << 30;  // positions and windows stay within int32 sums
constexpr int64_t kMostThreads = (int64_t(1) << 32) - 1;  // of a launch

constexpr int32_t kMostHeadDim = 1024;                    // where any is taken

// A product of counts, or more than any launch or index can hold.
inline int64_t product(std::initializer_list<int64_t> counts) {
  int64_t n = 1;
  for (int64_t c : counts)
    if (__builtin_mul_overflow(n, c, &n)) return int64_t(1) << 62;
  return n;
}

inline void check_head_dim(int d) { require(d == 32 || d == 64 || d == 128, "head_dim must be 32, 64 or 128"); }

inline TokensArg tokens_arg(const fluid_tokens* d, const void* p, const char* name, bool any_head_dim = false) {
  require(d != nullptr, name, ": NULL description");
  require(d->dtype == FLUID_F32 || d->dtype == FLUID_BF16, name, ": dtype must be f32 or bf16");
  require(d->batch >= 1 && d->tokens >= 1 && d->heads >= 1, name, ": batch, tokens and heads must be at least 1");
  require(d->tokens <= kMostTokens, name, ": more than 2^30 tokens");
  if (any_head_dim) require(d->head_dim >= 1 && d->head_dim <= kMostHeadDim, name, ": head_dim must lie in 1 .. 1024");
  else check_head_dim(d->head_dim);
  const int32_t extent[3] = {d->batch, d->tokens, d->heads};
  const int el = dtype_bytes(d->dtype);
  TokensArg a{const_cast<void*>(p), 0, 0, 0, 1};
  int64_t* const to[3] = {&a.sb, &a.st, &a.sh};
  for (int i = 0; i < 3; ++i) {
    if (extent[i] == 1) continue;  // its stride is never used
    require(d->stride[i] >= 0 && d->stride[i] <= (int64_t(1) << 40), name, ": strides must lie in 0 .. 2^40");
    *to[i] = d->stride[i];
    if (d->stride[i] * el % 16) a.vec = 0;
  }
  if ((uintptr_t)p % 16) a.vec = 0;
  require((uintptr_t)p % el == 0, name, ": misaligned for its type");
  return a;
}
inline TokensArg tokens_data(const fluid_tokens* d, const void* p, const char* name, bool any_head_dim = false) {
  require(p != nullptr, name, ": NULL data");
  return tokens_arg(d, p, name, any_head_dim);
}

// Neighbours of an output must not share elements (equal strides of two
// dimensions remain the caller's to avoid).
inline void check_apart(const fluid_tokens* d, const char* name) {
  const int32_t extent[3] = {d->batch, d->tokens, d->heads};
  for (int i = 0; i < 3; ++i)
    require(extent[i] == 1 || d->stride[i] >= d->head_dim,
            name, ": an output's strides must be at least head_dim");
}

}  // namespace fluid
