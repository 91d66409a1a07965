// Rotary positions: the turns of every pair, argument checks and launch sizes.
#include <algorithm>
#include <cmath>

#include "../host/handles.h"
#include "backend.h"
#include "check_tokens.h"

namespace fluid {

namespace {

void check_rotary(const fluid_rotary* r) {
  require(r != nullptr, "rotary: NULL");
  require(r->dim >= 2 && r->dim <= kMostHeadDim && r->dim % 2 == 0, "rotary: dim must be even and lie in 2 .. 1024");
  require(r->interleaved == 0 || r->interleaved == 1, "rotary: interleaved must be 0 or 1");
  require(r->scaling >= FLUID_ROTARY_NONE && r->scaling <= FLUID_ROTARY_RAMP, "rotary: unknown scaling");
  require(std::isfinite(r->amplitude), "rotary: amplitude must be finite");
  require(r->base >= 1.0 && std::isfinite(r->base), "rotary: base must be finite and at least 1");
  if (r->scaling == FLUID_ROTARY_NONE) return;
  require(r->factor > 0.0 && std::isfinite(r->factor), "rotary: factor must be positive and finite");
  require(r->scaling != FLUID_ROTARY_BASE || r->dim >= 4, "rotary: scaling the base needs a dim of at least 4");
  if (r->scaling == FLUID_ROTARY_RAMP) {
    require(r->length > 0.0 && std::isfinite(r->length), "rotary: length must be positive and finite");
    require(r->low < r->high && std::isfinite(r->low) && std::isfinite(r->high), "rotary: low must be below high");
  }
}

constexpr long double kTwoPi = 6.283185307179586476925286766559005768L;

uint64_t turns_of(const fluid_rotary& r, int i) {
  const long double d = r.dim, base = r.scaling == FLUID_ROTARY_BASE
                                          ? (long double)r.base * powl(r.factor, d / (d - 2.0L))
                                          : (long double)r.base;
  long double theta = powl(base, -2.0L * i / d);
  if (r.scaling == FLUID_ROTARY_LINEAR) theta /= r.factor;
  if (r.scaling == FLUID_ROTARY_RAMP) {
    const long double turns = r.length * theta / kTwoPi;
    const long double kept = std::min(1.0L, std::max(0.0L, (turns - r.low) / ((long double)r.high - r.low)));
    theta = kept * theta + (1.0L - kept) * theta / r.factor;
  }
  const long double turn = theta / kTwoPi, part = rintl(ldexpl(turn - floorl(turn), 64));
  return part < 0x1p64L ? (uint64_t)part : 0;  // also where a turn that no number holds makes a NaN
}

// Channels that can be read and written at once: bytes of them that divide the
// address and all strides, at most 16.  4096 tokens of 40 heads of 80, bf16, half of
// each turned: four at once, 14 us; one by one 28.
int at_once(const TokensArg& a, int el) {
  const uint64_t all = (uint64_t)(uintptr_t)a.p | (uint64_t)(a.sb * el) | (uint64_t)(a.st * el) | (uint64_t)(a.sh * el) | 16;
  return (int)(all & -all) / el;
}

// q or k and where it goes.
void set_pair(RotaryParams& p, int i, const fluid_tokens* xd, const void* x, const fluid_tokens* yd, void* y,
              const char* in, const char* out) {
  p.x[i] = tokens_data(xd, x, in, true);
  p.y[i] = tokens_data(yd, y, out, true);
  require(yd->dtype == xd->dtype && yd->batch == xd->batch && yd->tokens == xd->tokens && yd->heads == xd->heads &&
              yd->head_dim == xd->head_dim,
          out, " must have its input's dtype and shape");
  check_apart(yd, out);
  const TokensArg &a = p.x[i], &b = p.y[i];
  if (x == y)
    require(a.sb == b.sb && a.st == b.st && a.sh == b.sh, out, ": an output that is its input must have its strides");
  else
    p.tail = 1;
  p.heads[i] = xd->heads;
  const int el = dtype_bytes(xd->dtype);
  p.vec = std::min({p.vec, at_once(a, el), at_once(b, el)});
}

}  // namespace

}  // namespace fluid

using namespace fluid;

extern "C" {

fluid_status fluid_rotary_turns(const fluid_rotary* r, uint64_t* turns) {
  return call_guarded([&] {
    check_rotary(r);
    require(turns != nullptr, "turns: NULL");
    for (int i = 0; i < r->dim / 2; ++i) turns[i] = turns_of(*r, i);
  });
}

fluid_status fluid_rotate(const fluid_rotary* r, const uint64_t* turns, const int32_t* start,
                          const int32_t* positions, int64_t position_stride, const int32_t* count, int32_t inverse,
                          const fluid_tokens* qd, const void* q, const fluid_tokens* qod, void* qo,
                          const fluid_tokens* kd, const void* k, const fluid_tokens* kod, void* ko, void* hip_stream) {
  return call_guarded([&] {
    check_rotary(r);
    RotaryParams p{};
    p.vec = 16;
    require(turns != nullptr && (uintptr_t)turns % 8 == 0, "turns: NULL or misaligned");
    require(start == nullptr || positions == nullptr, "start and positions: only one of them");
    require(inverse == 0 || inverse == 1, "inverse must be 0 or 1");
    set_pair(p, 0, qd, q, qod, qo, "q", "q_out");
    if (kd != nullptr) {
      set_pair(p, 1, kd, k, kod, ko, "k", "k_out");
      require(kd->dtype == qd->dtype && kd->batch == qd->batch && kd->tokens == qd->tokens && kd->head_dim == qd->head_dim,
              "q and k must have one dtype, batch, tokens and head_dim");
      // threads read these while others write
      require(qo != ko, "q_out and k_out must not be the same");
      require(qo != k, "q_out must not be k");
      require(ko != q, "k_out must not be q");
    }
    require(r->dim <= qd->head_dim, "rotary: dim is larger than head_dim");
    require(positions == nullptr || qd->batch == 1 || (position_stride >= 0 && position_stride <= (int64_t(1) << 40)),
            "position_stride must lie in 0 .. 2^40");
    p.turns = turns;
    p.start = start;
    p.positions = positions;
    p.position_stride = qd->batch == 1 ? 0 : position_stride;
    p.count = count;
    p.batch = qd->batch;
    p.tokens = qd->tokens;
    p.head_dim = qd->head_dim;
    p.dim = r->dim;
    p.interleaved = r->interleaved;
    p.inverse = inverse;
    p.amplitude = r->amplitude;
    if (p.head_dim == p.dim) p.tail = 0;
    while ((r->interleaved ? r->dim : r->dim / 2) % p.vec || (p.tail && p.head_dim % p.vec)) p.vec /= 2;
    p.pairs = r->interleaved ? r->dim / std::max(p.vec, 2) : r->dim / 2 / p.vec;
    p.units = p.pairs + (p.tail ? (p.head_dim - p.dim) / p.vec : 0);
    const int64_t heads = int64_t(p.heads[0]) + p.heads[1], rows = product({p.batch, p.tokens, p.units});
    // A thread's angles serve up to four heads where that still fills the GPU: 8192
    // tokens of 40 heads take 35 us, with eight heads to a thread 37 and two 38 (2048
    // tokens 10.5, 11.6, 9.9); 1024 tokens of 40 heads 7.5 us with a thread to a
    // head, 8.2 to 11.5 with four.
    const int64_t few = (heads + 3) / 4;
    p.head_threads = (int32_t)(product({rows, few}) >= 131072 ? few : heads);
    const int64_t items = product({rows, p.head_threads});
    require(heads < int64_t(1) << 31 && items <= kMostThreads - 255, "q, k: too large for one launch");
    p.items = (uint32_t)items;
    p.div_units = make_fastdiv(p.units);
    p.div_heads = make_fastdiv(p.head_threads);
    p.div_tokens = make_fastdiv(p.tokens);
    run_rotate(p, qd->dtype, hip_stream);
  });
}

}  // extern "C"
