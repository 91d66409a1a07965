// Attention over fp32 keys and values on the bf16 matrix cores (32x32x16),
// scores kept in registers (attn_rows.h).
//
// Queries, keys, values and weights are three bf16 parts each, x = h + m + l,
// each part what the ones before leave, rounded: 24 bits.  A product is summed
// from the six of the nine products of parts that matter (h h, h m, m h, m m,
// h l, l h); the three left out are together at most 2^-24 of it, an fp32
// rounding.  For 16 channels these are six MFMAs of 32 cycles, where the fp32
// MFMA needs eight of 64.  Keys and values are split on their way from memory
// through registers to LDS, one tile of 32 tokens ahead of the products.
//
// 8 sequences of up to 512 tokens of 16 heads of 64, both directions: 40 to 44 us
// by card (42 before the longest came first, 61 with the fp32 MFMA).  Vector
// instructions (exponentials, splits of the weights and of the keys and values
// that every workgroup loads) are 37 % of the cycles of a busy compute unit, MFMA
// 31 %, and two wavefronts a SIMD do not hide all waits; a third spills (44 ->
// 52 us; 8 x 512 causal queries 45 -> 62).
#include "attn_rows.h"
#include "launch_attn.h"

namespace fluid {

namespace {

constexpr int BN = kF32Tile;

// Two values' parts, packed: the first in the low halves.  Past bf16's largest a
// first part rounds to infinity; `cut` takes such a value's upper bits as they are.
// What the first part leaves is added to `odd` as 0, or as NaN where it is none.
struct Parts {
  uint32_t h, m, l;
};
template <bool CUT>
__device__ __forceinline__ Parts split2(float a, float b, float& odd) {
  Parts r;
  r.h = pack_bf16(a, b);
  if (CUT && (r.h & 0x7f80u) == 0x7f80u) r.h = (r.h & 0xffff0000u) | (__float_as_uint(a) >> 16);
  if (CUT && (r.h & 0x7f800000u) == 0x7f800000u) r.h = (r.h & 0xffffu) | (__float_as_uint(b) & 0xffff0000u);
  const float am = a - __uint_as_float(r.h << 16), bm = b - __uint_as_float(r.h & 0xffff0000u);
  odd = __builtin_fmaf(bm, 0.0f, __builtin_fmaf(am, 0.0f, odd));
  r.m = pack_bf16(am, bm);
  r.l = pack_bf16(am - __uint_as_float(r.m << 16), bm - __uint_as_float(r.m & 0xffff0000u));
  return r;
}
// Eight values' parts as operands.
struct Split8 {
  piece h, m, l;
  float odd = 0.0f;
  template <bool CUT>
  __device__ __forceinline__ void split(const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Parts r = split2<CUT>(x[2 * i], x[2 * i + 1], odd);
      h[i] = r.h, m[i] = r.m, l[i] = r.l;
    }
  }
  __device__ __forceinline__ explicit Split8(const float* x) { split<false>(x); }
  // some value is an infinity, a NaN or past bf16's largest
  __device__ __forceinline__ bool past() const { return odd != odd; }
};
__device__ __forceinline__ v8i16 op(piece x) { return __builtin_bit_cast(v8i16, x); }

template <int D, int TEAMS, bool VEC>
__global__ __launch_bounds__(kTeam * TEAMS) __attribute__((amdgpu_waves_per_eu(D == 128 ? 1 : 2)))
void attention_f32_kernel(AttnParams p) {
  using At = Bf16Place<D>;
  constexpr int PPR = D / 8, PIECES = BN * PPR, CT = D / 32, PLANE = BN * D;
  constexpr int NP = 2 * PIECES / kTeam;  // pieces a thread moves, keys first
  static_assert(NP * kTeam == 2 * PIECES && PIECES % 64 == 0, "whole pieces, one operand to a wavefront");
  struct Stage {
    uint16_t k[3 * PLANE], v[3 * PLANE];
    uint32_t odd_key[kTeamWaves];  // whether a wavefront's keys hold an infinity or a NaN
  };
  __shared__ __attribute__((aligned(1024))) Stage st[2][TEAMS];
  __shared__ float ml[2][TEAMS == 2 ? kTeam : 1];

  Rows<float, D, TEAMS> w(p);
  if (!w.find()) return;
  const int tid = w.tid, col = w.col, half = w.half, n = w.n;
  v8i16 qh[D / 16], qm[D / 16], ql[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = w.q[16 * s + 8 * half + e];
    Split8 r(x);
    if (r.past()) r.split<true>(x);
    qh[s] = op(r.h), qm[s] = op(r.m), ql[s] = op(r.l);
  }

  // Tile u's pieces of this thread, in registers; rows past the last token
  // repeat it.
  Eight<float> raw[NP];
  auto fetch = [&](int u) {
    const int t0 = w.start(u), last = n - 1 - t0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = tid + kTeam * i;
      const bool values = kTeam * i + 64 * w.wave >= PIECES;
      const int x = at % PIECES, row = min(x / PPR, last);
      raw[i].load((values ? w.v + t0 * p.v.st + row * p.v.st : w.k + t0 * p.k.st + row * p.k.st) + 8 * (x % PPR), VEC);
    }
  };
  // And in LDS.  Values that are no numbers become zeros (Rows::add_odd); keys
  // that are none are flagged.
  bool dirty = false;
  auto park = [&](Stage& to) {
    bool odd_key = false;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = tid + kTeam * i;
      const bool values = kTeam * i + 64 * w.wave >= PIECES;
      const int x = at % PIECES, t = x / PPR, c = x % PPR;
      float f[8];
      raw[i].floats(f);
      Split8 r(f);
      if (r.past()) {
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          odd |= odd_value(f[e]);
          f[e] = odd_value(f[e]) ? 0.0f : f[e];
        }
        if (values) dirty |= odd;
        else odd_key |= odd;
        r.split<true>(f);
      }
      uint16_t* const dst = values ? to.v + At::v(t, c) : to.k + At::k(t, c);
      *(piece*)dst = r.h;
      *(piece*)(dst + PLANE) = r.m;
      *(piece*)(dst + 2 * PLANE) = r.l;
    }
    const bool any = __ballot(odd_key) != 0;
    if (w.lane == 0) to.odd_key[w.wave] = any;
  };

  auto step = [&](int at, Stage& now, Stage& next) {
    __syncthreads();
    const int u = at + w.team, t0 = w.start(u);
    const bool more = u + TEAMS < w.u1;
    if (more) fetch(u + TEAMS);
    if (w.live && u < w.u1) {
      f32x16 s[1] = {}, rest = {};
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint16_t* const at_k = now.k + At::k(col, 2 * k + half);
        const v8i16 kh = *(const v8i16*)at_k, km = *(const v8i16*)(at_k + PLANE), kl = *(const v8i16*)(at_k + 2 * PLANE);
        rest = mfma_bf16(kl, qh[k], rest);
        s[0] = mfma_bf16(kh, qh[k], s[0]);
        rest = mfma_bf16(kh, ql[k], rest);
        rest = mfma_bf16(km, qm[k], rest);
        rest = mfma_bf16(km, qh[k], rest);
        rest = mfma_bf16(kh, qm[k], rest);
      }
      s[0] += rest;
      const piece odd = *(const piece*)now.odd_key;
      if (__builtin_expect((odd[0] | odd[1] | odd[2] | odd[3]) != 0, 0)) {
        // rare: what the products left out of the scores, term by term
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = t0 + w.token(0, e);
          if (t < n)
            for (int c = 0; c < D; ++c) {
              const float x = w.k[t * p.k.st + c];
              if (odd_value(x)) s[0][e] += x * w.q[c];
            }
        }
      }
      w.weigh(s, t0);
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += s[0][e];
      w.l += sum;
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // tokens 16 k + 8 (e / 4) + 4 half + e % 4
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[0][8 * k + e];
        const Split8 pr(x);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          const v8i16 vh = read_values<D>(now.v, k, c, w.lane), vm = read_values<D>(now.v + PLANE, k, c, w.lane),
                      vl = read_values<D>(now.v + 2 * PLANE, k, c, w.lane);
          w.acc[c] = mfma_bf16(vl, op(pr.h), w.acc[c]);
          w.acc[c] = mfma_bf16(vh, op(pr.l), w.acc[c]);
          w.acc[c] = mfma_bf16(vm, op(pr.m), w.acc[c]);
          w.acc[c] = mfma_bf16(vm, op(pr.h), w.acc[c]);
          w.acc[c] = mfma_bf16(vh, op(pr.m), w.acc[c]);
          w.acc[c] = mfma_bf16(vh, op(pr.h), w.acc[c]);
        }
      }
    }
    if (more) park(next);
  };

  if (w.u0 + w.team < w.u1) {
    fetch(w.u0 + w.team);
    park(st[0][w.team]);
  }
  for (int at = w.u0; at < w.u1; at += 2 * TEAMS) {
    step(at, st[0][w.team], st[1][w.team]);
    if (at + TEAMS < w.u1) step(at + TEAMS, st[1][w.team], st[0][w.team]);
  }
  if (__syncthreads_or(dirty) && w.live) w.add_odd(true);
  w.join_teams((f32x4*)&st[0][0], (f32x4*)&st[1][0], (float(*)[kTeam])ml);
  if (w.team == 0) w.template store<VEC>();
}

template <int D, int TEAMS>
hipError_t launch(const AttnParams& p, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.row_tiles * p.splits)), block(kTeam * TEAMS);
  if (p.k.vec && p.v.vec && p.o.vec)
    hipLaunchKernelGGL((attention_f32_kernel<D, TEAMS, true>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((attention_f32_kernel<D, TEAMS, false>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_f32(const AttnParams& p, int head_dim, hipStream_t s) {
  switch (head_dim) {
    case 32: return p.teams == 2 ? launch<32, 2>(p, s) : launch<32, 1>(p, s);
    case 64: return p.teams == 2 ? launch<64, 2>(p, s) : launch<64, 1>(p, s);
    default: return launch<128, 1>(p, s);
  }
}

hipError_t launch_attention(const AttnParams& p, int dtype, int head_dim, hipStream_t s) {
  const hipError_t e = dtype == DT_BF16 ? launch_attention_bf16(p, head_dim, s) : launch_attention_f32(p, head_dim, s);
  return e != hipSuccess || p.splits == 1 ? e : launch_attention_join(p, dtype, head_dim, s);
}

}  // namespace fluid
