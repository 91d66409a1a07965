// What the attention kernels over keys and values share: the rows of a
// workgroup and of a wavefront, the running softmax, and the way out.
//
// A workgroup takes 128 rows of one kv head -- (query, head of its group)
// pairs, so that the heads that share keys also share their loads.  Four
// wavefronts, a team, have 32 rows each; a workgroup of two teams has the same
// rows twice and its teams take tiles of tokens in turn, which keeps two
// wavefronts on every SIMD where there is only one workgroup to a compute
// unit.
//
// S^T = K Q^T leaves a lane with one row's scores for 16 of 32 tokens, and
// taking the tokens in just that order as the contraction of O^T = V^T P^T
// makes them its operand: nothing is exchanged between lanes but the row
// maximum of two lanes.
#pragma once

#include "dev_attn.h"

namespace fluid {

typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t piece __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

constexpr int kTeamWaves = 4, kTeam = 64 * kTeamWaves, kRows = 32 * kTeamWaves;

// The running maximum may lag a row's largest score by this much (in powers
// of two): weights are then at most 256, and the sums are hardly ever scaled.
constexpr float kRowSlack = 8.0f;

// Places of bf16 keys and values in LDS: piece c (16 bytes) of token t lies at
// c ^ x(t) of its row, so that reads of equal pieces of sixteen tokens (K) and
// of equal 64-byte runs of four tokens (V) hit different banks.
template <int D>
struct Bf16Place {
  static constexpr int PPR = D / 8;  // pieces of a token
  __device__ static __forceinline__ int kx(int t) { return PPR >= 16 ? t & 15 : (t / (16 / PPR)) & (PPR - 1); }
  __device__ static __forceinline__ int vx(int t) { return D == 128 ? 4 * (t & 3) : D == 64 ? 4 * ((t >> 1) & 1) : 0; }
  __device__ static __forceinline__ int k(int t, int c) { return t * D + 8 * (c ^ kx(t)); }
  __device__ static __forceinline__ int v(int t, int c) { return t * D + 8 * (c ^ vx(t)); }
};
// Part k (16 tokens) of 32-channel run c of V^T as an operand: a transposing
// read hands a lane one channel of four tokens, of which its source lane is
// one token's, four channels of sixteen.
template <int D>
__device__ __forceinline__ v8i16 read_values(uint16_t* sv, int k, int c, int lane) {
  const int t = 16 * k + 4 * (lane >> 5) + ((lane & 15) >> 2), ch = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto at = [&](int t) { return (lds_v4i16*)(sv + Bf16Place<D>::v(t, (32 * c + ch) >> 3) + (ch & 7)); };
  const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(t));
  const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(t + 8));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x16 mfma_bf16(v8i16 a, v8i16 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ bool odd_value(float x) { return !(fabsf(x) <= 3.402823466e38f); }

template <typename T, int D, int TEAMS>
struct Rows {
  static constexpr int CT = D / 32;
  const AttnParams& p;
  Share sh;
  int lane, wave, team, tid;  // within the workgroup's team
  int col, half;              // row of 32; half of the tokens
  int n, u0, u1;              // tokens; steps
  int first, past;            // this wavefront's rows
  bool live;
  int bp_min, bp_max, wp_min, wp_max;  // positions of the workgroup's and the wavefront's rows
  int query, head;                     // of this lane's row
  Sight eye;
  const T *q, *k, *v;
  float m, l;
  bool wide;  // some row of the wavefront is past_fused
  f32x16 acc[CT];

  __device__ __forceinline__ explicit Rows(const AttnParams& p_) : p(p_) {}
  __device__ __forceinline__ bool find() {
    if (!sh.find(p, blockIdx.x)) return false;
    const Item& it = sh.item;
    lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    team = w / kTeamWaves;
    wave = w % kTeamWaves;
    tid = 64 * wave + lane;
    col = lane & 31;
    half = lane >> 5;
    n = it.n;
    u0 = sh.first;
    u1 = sh.end;
    first = it.r0 + 32 * wave;
    past = min(first + 32, it.r1);
    live = first < it.r1;
    bp_min = it.p_min(p);
    bp_max = it.p_max(p);
    wp_min = it.p0 + (int)fdiv(first, p.div_group);
    wp_max = it.p0 + (int)fdiv(past - 1, p.div_group);
    const int r = min(first + col, it.r1 - 1);
    query = (int)fdiv(r, p.div_group);
    head = it.h * p.group + (r - query * p.group);
    eye = sight(p, it.p0 + query, n);
    q = (const T*)p.q.p + it.b * p.q.sb + query * p.q.st + head * p.q.sh;
    k = (const T*)p.k.p + it.b * p.k.sb + it.h * p.k.sh;
    v = (const T*)p.v.p + it.b * p.v.sb + it.h * p.v.sh;
    m = kLow;
    l = 0.0f;
    wide = false;
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = f32x16{};
    return true;
  }
  __device__ __forceinline__ int start(int u) const { return sh.item.range.tile(u) * p.token_tile; }
  // whether all rows from position a to z see every token of the tile from t0 on
  __device__ __forceinline__ bool whole(int t0, int a, int z) const {
    const int t1 = t0 + p.token_tile;
    return t1 <= n && (!p.causal || t1 - 1 <= a) &&
           (p.window <= 0 || t1 <= p.sinks || (t0 > z - p.window && (p.causal || t1 <= a + p.window)));
  }
  __device__ __forceinline__ bool whole_for_all(int t0) const { return whole(t0, bp_min, bp_max); }
  // token of score e of 32-token part i: this lane's half of them
  __device__ __forceinline__ int token(int i, int e) const { return 32 * i + 8 * (e >> 2) + 4 * half + (e & 3); }

  // Masks the scores of the tile from t0 on and makes them weights, 2 to the
  // power of what they are below the running maximum.
  template <int NT>
  __device__ __forceinline__ void weigh(f32x16 (&s)[NT], int t0) {
    if (!whole(t0, wp_min, wp_max)) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!eye.sees(t0 + token(i, e))) s[i][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[i][e]);
    top *= p.cs;
    if (__ballot(top - m > kRowSlack)) {
      const float m1 = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
      const float a = __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= a;
#pragma unroll
      for (int c = 0; c < CT; ++c) acc[c] *= a;
      wide = __ballot(past_fused(m)) != 0;
    }
    float factor = p.cs, shift = -m;
    if (__builtin_expect(wide, 0)) {
#pragma clang fp contract(off)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[i][e] = s[i][e] * p.cs - m;
      factor = 1.0f;
      shift = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], factor, shift));
  }

  // Weight 0 times a value that is no number would still be none, so such
  // values are zeros in LDS where rows differ in what they see (in every tile
  // if `all`), and are added here, at the end, to the rows that do see them.
  __device__ __forceinline__ void add_odd(bool all) {
#pragma nounroll
    for (int u = u0 + team; u < u1; u += TEAMS) {
      const int t0 = start(u);
      if (!all && whole_for_all(t0)) continue;
#pragma nounroll
      for (int t = t0; t < min(t0 + p.token_tile, n); ++t) {
        if (!eye.sees(t)) continue;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = Elem<T>::load(v, t * p.v.st + 32 * c + token(0, e));
            if (odd_value(x)) acc[c][e] += x;
          }
      }
    }
  }

  // Adds the second team's sums to the first's, through a and b (8 KiB of LDS
  // for every 32 channels each) and ml.
  __device__ __forceinline__ void join_teams(f32x4* a, f32x4* b, float (*ml)[kTeam]) {
    if constexpr (TEAMS == 2) {
      __syncthreads();
      if (team == 1) {
        ml[0][tid] = m;
        ml[1][tid] = l;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            (i < 2 ? a : b)[(2 * c + (i & 1)) * kTeam + tid] =
                f32x4{acc[c][4 * i], acc[c][4 * i + 1], acc[c][4 * i + 2], acc[c][4 * i + 3]};
      }
      __syncthreads();
      if (team == 1) return;
      const float m2 = ml[0][tid], top = fmaxf(m, m2);
      const float x = __builtin_amdgcn_exp2f(m - top), y = __builtin_amdgcn_exp2f(m2 - top);
      m = top;
      l = l * x + ml[1][tid] * y;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 o = (i < 2 ? a : b)[(2 * c + (i & 1)) * kTeam + tid];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[c][4 * i + e] = acc[c][4 * i + e] * x + o[e] * y;
        }
    }
  }

  // The rows, or their sums where other workgroups have a share of them.
  template <bool VEC>
  __device__ __forceinline__ void store() {
    if (!live || first + col >= sh.item.r1) return;
    l += __shfl_xor(l, 32);
    if (!sh.whole()) {
      float* const to = sh.slot(p, D);
      const int r = first - sh.item.r0 + col;
      if (half == 0) {
        to[r] = m;
        to[kRows + r] = l;
      }
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(to + 2 * kRows + r * D + 32 * c + 8 * i + 4 * half) =
              f32x4{acc[c][4 * i], acc[c][4 * i + 1], acc[c][4 * i + 2], acc[c][4 * i + 3]};
      return;
    }
    const float inv = 1.0f / l;
    T* const op = (T*)p.o.p + sh.item.b * p.o.sb + query * p.o.st + head * p.o.sh;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = l == 0.0f ? 0.0f : acc[c][4 * i + e] * inv;
        T* const to = op + 32 * c + 8 * i + 4 * half;
        if (VEC) {
          if constexpr (sizeof(T) == 2) *(uint2*)to = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
          else *(f32x4*)to = f32x4{o[0], o[1], o[2], o[3]};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) Elem<T>::store(to, e, o[e]);
        }
      }
  }
};

}  // namespace fluid
