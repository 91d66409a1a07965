// Attention over bf16 keys and values on the bf16 matrix cores (32x32x16),
// scores kept in registers (attn_rows.h).  Keys and values go from memory to
// LDS without registers, one tile of 64 tokens ahead of the products; V is
// read back by transposing reads.
//
// 8192 queries of 32 heads of 128 (8 of keys), window 2048: 267 to 292 us (by
// card), 820 to 900 TFLOP/s of the products needed, where a library product of 8192^3
// reaches 1140.  MFMA are 46 % and vector instructions 44 % of the cycles, at a
// clock of 1.8 GHz of 2.4: power bounds it.  The products alone, without copies
// and weights, take 193 us; with LDS operands read further ahead, copies a step
// and a half ahead behind two barriers, or one of a SIMD's two wavefronts
// preferred the time is the same or worse.  2048 queries of 32 heads (window
// 1024) take 42 to 50 us: two workgroups to a compute unit, of 2 to 19 steps each.
//
// Weights are rounded to bf16, the type that the values' products take: a second
// part of them would double those products.  That, averaged over the tokens, is
// below the output's own rounding: the error of 8192 queries against 64 bits is
// 0.21 % of the output, 0.15 % with fp32 weights.
#include "attn_rows.h"
#include "launch_attn.h"

namespace fluid {

namespace {

constexpr int BN = kBf16Tile, NT = BN / 32;

// 16 bytes from memory to LDS, lane l's to `to` + 16 l.
__device__ __forceinline__ void copy_to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// One team of narrow heads fits a SIMD three times: 8 x 2048 causal queries of
// 16 heads of 64 channels take 126 us, 16 x 1024 of 32 channels 64; with two of
// them 143 and 72.
constexpr int waves_per_simd(int D, int teams) { return teams == 1 && D < 128 ? 3 : 2; }

template <int D, int TEAMS, bool VEC>
__global__ __launch_bounds__(kTeam * TEAMS)
__attribute__((amdgpu_waves_per_eu(waves_per_simd(D, TEAMS), waves_per_simd(D, TEAMS))))
void attention_bf16_kernel(AttnParams p) {
  using At = Bf16Place<D>;
  constexpr int PPR = D / 8, PIECES = BN * PPR, CT = D / 32;
  // an object per stage and operand, so that the compiler can tell a copy
  // into one from reads of another
  __shared__ __attribute__((aligned(1024))) uint16_t sk0[TEAMS][BN * D], sk1[TEAMS][BN * D];
  __shared__ __attribute__((aligned(1024))) uint16_t sv0[TEAMS][BN * D], sv1[TEAMS][BN * D];
  __shared__ float ml[2][TEAMS == 2 ? kTeam : 1];

  Rows<uint16_t, D, TEAMS> w(p);
  if (!w.find()) return;
  const int tid = w.tid, col = w.col, half = w.half, n = w.n;
  v8i16 q[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const uint16_t* const from = w.q + 16 * s + 8 * half;
    if (VEC) {
      q[s] = __builtin_bit_cast(v8i16, *(const piece*)from);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[s][e] = (short)from[e];
    }
  }

  // Tile u's keys and values into a stage; rows past the last token repeat it.
  auto stage = [&](int u, uint16_t* sk, uint16_t* sv) {
    const int t0 = w.start(u), last = n - 1 - t0;
    const uint16_t* const k0 = w.k + t0 * p.k.st;
    const uint16_t* const v0 = w.v + t0 * p.v.st;
#pragma unroll
    for (int i = 0; i < PIECES / kTeam; ++i) {
      const int at = tid + kTeam * i, t = at / PPR, c = at % PPR, row = min(t, last);
      if constexpr (VEC) {
        const int to = 8 * (kTeam * i + 64 * w.wave);
        copy_to_lds((const char*)k0 + (uint32_t)((row * (int)p.k.st + 8 * (c ^ At::kx(t))) * 2), sk + to);
        copy_to_lds((const char*)v0 + (uint32_t)((row * (int)p.v.st + 8 * (c ^ At::vx(t))) * 2), sv + to);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sk[at * 8 + e] = k0[row * p.k.st + 8 * (c ^ At::kx(t)) + e];
          sv[at * 8 + e] = v0[row * p.v.st + 8 * (c ^ At::vx(t)) + e];
        }
      }
    }
  };
  // Values that are no numbers become zeros, in the tiles that Rows::add_odd
  // goes through.
  uint32_t dirty = 0;
  auto clean = [&](uint16_t* sv) {
#pragma nounroll
    for (int at = tid; at < PIECES; at += kTeam) {
      piece x = *(const piece*)(sv + 8 * at), keep;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        keep[i] = ((x[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((x[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
      const uint32_t odd = ~(keep[0] & keep[1] & keep[2] & keep[3]);
      if (odd) *(piece*)(sv + 8 * at) = x & keep;
      dirty |= odd;
    }
  };

  // The teams' tiles from step `at` on, one to a team, are in sk and sv.
  auto step = [&](int at, uint16_t* sk, uint16_t* sv, uint16_t* next_k, uint16_t* next_v) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int u = at + w.team, t0 = w.start(u);
    bool masked = false;  // some team's tile is
#pragma unroll
    for (int i = 0; i < TEAMS; ++i) masked |= at + i < w.u1 && !w.whole_for_all(w.start(at + i));
    if (masked) {  // a tile that all rows see whole may have one beside it that they do not
      if (u < w.u1 && !w.whole_for_all(t0)) clean(sv);
      __syncthreads();
    }
    if (u + TEAMS < w.u1) stage(u + TEAMS, next_k, next_v);
    if (!w.live || u >= w.u1) return;
    f32x16 s[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      s[i] = f32x16{};
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
        s[i] = mfma_bf16(*(const v8i16*)(sk + At::k(32 * i + col, 2 * k + half)), q[k], s[i]);
    }
    w.weigh(s, t0);
    v8i16 pr[2 * NT];  // part c: tokens 16 c + 8 (e / 4) + 4 half + e % 4
#pragma unroll
    for (int c = 0; c < 2 * NT; ++c)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        // the sum is taken of the rounded weights
        const s16x2 x = __builtin_bit_cast(
            s16x2, __builtin_convertvector(f32x2{s[c >> 1][8 * (c & 1) + e], s[c >> 1][8 * (c & 1) + e + 1]}, bf16x2));
        w.l = __builtin_amdgcn_fdot2_f32_bf16(x, s16x2{0x3f80, 0x3f80}, w.l, false);
        pr[c][e] = x[0], pr[c][e + 1] = x[1];
      }
#pragma unroll
    for (int k = 0; k < 2 * NT; ++k)
#pragma unroll
      for (int c = 0; c < CT; ++c) w.acc[c] = mfma_bf16(read_values<D>(sv, k, c, w.lane), pr[k], w.acc[c]);
  };

  uint16_t *const k0 = sk0[w.team], *const k1 = sk1[w.team], *const v0 = sv0[w.team], *const v1 = sv1[w.team];
  if (w.u0 + w.team < w.u1) stage(w.u0 + w.team, k0, v0);
  for (int at = w.u0; at < w.u1; at += 2 * TEAMS) {
    step(at, k0, v0, k1, v1);
    if (at + TEAMS < w.u1) step(at + TEAMS, k1, v1, k0, v0);
  }
  if (__syncthreads_or(dirty) && w.live) w.add_odd(false);
  w.join_teams((f32x4*)sk0, (f32x4*)sk1, (float(*)[kTeam])ml);
  if (w.team == 0) w.template store<VEC>();
}

template <int D, int TEAMS>
hipError_t launch(const AttnParams& p, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.row_tiles * p.splits)), block(kTeam * TEAMS);
  // a tile's rows have to lie within 32-bit offsets
  const int64_t most = (int64_t(1) << 31) / (BN * 2) - D;
  if (p.q.vec && p.k.vec && p.v.vec && p.o.vec && p.k.st < most && p.v.st < most)
    hipLaunchKernelGGL((attention_bf16_kernel<D, TEAMS, true>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((attention_bf16_kernel<D, TEAMS, false>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_bf16(const AttnParams& p, int head_dim, hipStream_t s) {
  switch (head_dim) {
    case 32: return p.teams == 2 ? launch<32, 2>(p, s) : launch<32, 1>(p, s);
    case 64: return p.teams == 2 ? launch<64, 2>(p, s) : launch<64, 1>(p, s);
    default: return p.teams == 2 ? launch<128, 2>(p, s) : launch<128, 1>(p, s);
  }
}

}  // namespace fluid
