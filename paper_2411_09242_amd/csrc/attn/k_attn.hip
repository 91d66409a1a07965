// Attention over keys and values in bf16 or fp32, scores kept in registers.
//
// A workgroup takes 128 rows of one kv head -- (query, head of its group)
// pairs, so that the heads that share keys also share their loads -- and
// walks the tiles of tokens that some row sees; each of its four wavefronts
// has 32 rows.  S^T = K Q^T leaves a lane with one row's scores for 16 of 32
// tokens, and taking the tokens in just that order as the contraction of
// O^T = V^T P^T makes them its operand: nothing is exchanged between lanes
// but the row maximum of two lanes.  bf16 runs 32x32x16 MFMAs (V read from
// LDS by transposing reads), fp32 32x32x2 ones.  Keys and values go from
// memory to LDS without registers, one tile ahead of the products.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t piece __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves;

// The running maximum may lag a row's largest score by this much (in powers
// of two): weights are then at most 256, and the sums are hardly ever scaled.
constexpr float kSlack = 8.0f;

template <typename T, int D>
struct Shape {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int BN = kBf16 ? kBf16Tile : kF32Tile;
  static constexpr int EPP = 16 / sizeof(T);       // elements of a 16-byte piece
  static constexpr int PPR = D / EPP;              // pieces of a token
  static constexpr int NP = BN * PPR / kThreads;   // pieces a thread moves, of K and of V
  static_assert(NP * kThreads == BN * PPR, "whole pieces");
  // Piece c of token t lies at place c ^ x(t) of its row, so that reads of
  // equal pieces of eight tokens (K), of equal 64-byte runs of four tokens
  // (bf16 V) or of tokens t and t + 4 (fp32 V) hit different banks.
  __device__ static __forceinline__ int kx(int t) { return PPR >= 16 ? t & 15 : (t / (16 / PPR)) & (PPR - 1); }
  __device__ static __forceinline__ int vx(int t) {
    if (kBf16) return D == 128 ? 4 * (t & 3) : D == 64 ? 4 * ((t >> 1) & 1) : 0;
    return PPR >= 16 ? 8 * ((t >> 2) & 1) : 0;
  }
  __device__ static __forceinline__ int k(int t, int c) { return t * D + EPP * (c ^ kx(t)); }
  __device__ static __forceinline__ int v(int t, int c) { return t * D + EPP * (c ^ vx(t)); }
};

__device__ __forceinline__ bool odd_value(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// 16 bytes from memory to LDS, lane l's to `to` + 16 l.
__device__ __forceinline__ void copy_to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <typename T, int D, bool VEC>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attention_kernel(AttnParams p) {
  using S = Shape<T, D>;
  constexpr bool kBf16 = S::kBf16;
  constexpr int BN = S::BN, NT = BN / 32, CT = D / 32, NP = S::NP, PPR = S::PPR, EPP = S::EPP;
  // an object per stage and operand, so that the compiler can tell a copy
  // into one from reads of another
  __shared__ __attribute__((aligned(1024))) T sk0[BN * D], sk1[BN * D];
  __shared__ __attribute__((aligned(1024))) T sv0[BN * D], sv1[BN * D];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;

  Share sh;
  if (!sh.find(p, blockIdx.x)) return;
  const Item& it = sh.item;
  const int b = it.b, h = it.h, n = it.n, r0 = it.r0, r1 = it.r1, p0 = it.p0;
  const TileRange range = it.range;
  const int u0 = sh.first, u1 = sh.end;
  const int bp_min = it.p_min(p), bp_max = it.p_max(p);

  // this wavefront's rows
  const int w0 = r0 + 32 * wave;
  const bool live = w0 < r1;
  const int w1 = min(w0 + 32, r1);
  const int wp_min = p0 + (int)fdiv(w0, p.div_group), wp_max = p0 + (int)fdiv(w1 - 1, p.div_group);
  const int r = min(w0 + col, r1 - 1);
  const int qi = (int)fdiv(r, p.div_group), hq = h * p.group + (r - qi * p.group);
  const Sight eye = sight(p, p0 + qi, n);
  const T* const qp = (const T*)p.q.p + b * p.q.sb + qi * p.q.st + hq * p.q.sh;
  bf16x8 qb[kBf16 ? D / 16 : 1];
  float qf[kBf16 ? 1 : D / 2];
  if constexpr (kBf16) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const T* const from = qp + 16 * s + 8 * half;
      if (VEC) {
        qb[s] = __builtin_bit_cast(bf16x8, *(const piece*)from);
      } else {
        v8i16 t;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (short)from[e];
        qb[s] = __builtin_bit_cast(bf16x8, t);
      }
    }
  } else {
#pragma unroll
    for (int s = 0; s < D / 8; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[4 * s + e] = qp[8 * s + 4 * half + e];
  }

  const T* const kb = (const T*)p.k.p + b * p.k.sb + h * p.k.sh;
  const T* const vb = (const T*)p.v.p + b * p.v.sb + h * p.v.sh;
  // Tile u's keys and values into a stage; rows past the last token repeat it.
  auto stage = [&](int u, T* sk, T* sv) {
    const int t0 = range.tile(u) * BN, last = n - 1 - t0;
    const T* const k0 = kb + t0 * p.k.st;
    const T* const v0 = vb + t0 * p.v.st;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = tid + kThreads * i, t = at / PPR, c = at % PPR, row = min(t, last);
      if constexpr (VEC) {
        const int to = EPP * (kThreads * i + 64 * wave);
        copy_to_lds((const char*)k0 + (uint32_t)((row * (int)p.k.st + EPP * (c ^ S::kx(t))) * (int)sizeof(T)), sk + to);
        copy_to_lds((const char*)v0 + (uint32_t)((row * (int)p.v.st + EPP * (c ^ S::vx(t))) * (int)sizeof(T)), sv + to);
      } else {
#pragma unroll
        for (int e = 0; e < EPP; ++e) {
          sk[at * EPP + e] = k0[row * p.k.st + EPP * (c ^ S::kx(t)) + e];
          sv[at * EPP + e] = v0[row * p.v.st + EPP * (c ^ S::vx(t)) + e];
        }
      }
    }
  };
  // token of score v of 32-token part i (this lane's half of them)
  auto token = [&](int i, int v) { return 32 * i + 8 * (v >> 2) + 4 * half + (v & 3); };

  float m = kLow, l = 0.0f;
  f32x16 acc[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) acc[c] = f32x16{};

  // whether all rows from position a to z see every token from t0 on of a tile
  auto whole_for = [&](int t0, int a, int z) {
    const int t1 = t0 + BN;
    return t1 <= n && (!p.causal || t1 - 1 <= a) &&
           (p.window <= 0 || t1 <= p.sinks || (t0 > z - p.window && (p.causal || t1 <= a + p.window)));
  };
  // Weight 0 times a value that is no number would still be none.  Where rows
  // differ in what they see, such values become zeros in LDS, and the rows that
  // do see them get them added at the end.
  uint32_t dirty = 0;
  auto clean = [&](T* sv) {
#pragma nounroll
    for (int at = tid; at < (BN * PPR); at += kThreads) {
      piece w = *(const piece*)(sv + EPP * at), keep;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kBf16)
          keep[i] = ((w[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
        else
          keep[i] = (w[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffffffffu;
      }
      const uint32_t odd = ~(keep[0] & keep[1] & keep[2] & keep[3]);
      if (odd) *(piece*)(sv + EPP * at) = w & keep;
      dirty |= odd;
    }
    __syncthreads();
  };
  auto add_odd = [&]() {
#pragma nounroll
    for (int u = u0; u < u1; ++u) {
      const int t0 = range.tile(u) * BN;
      if (whole_for(t0, bp_min, bp_max)) continue;
#pragma nounroll
      for (int t = t0; t < min(t0 + BN, n); ++t) {
        if (!eye.sees(t)) continue;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float x = Elem<T>::load(vb, t * p.v.st + 32 * c + 8 * (v >> 2) + 4 * half + (v & 3));
            if (odd_value(x)) acc[c][v] += x;
          }
      }
    }
  };

  auto step = [&](int u, T* sk, T* sv, T* next_k, T* next_v) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int t0 = range.tile(u) * BN;
    if (!whole_for(t0, bp_min, bp_max)) clean(sv);
    if (u + 1 < u1) stage(u + 1, next_k, next_v);
    if (!live) return;
    f32x16 s[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      s[i] = f32x16{};
      if constexpr (kBf16) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const bf16x8 a = *(const bf16x8*)(sk + S::k(32 * i + col, 2 * k + half));
          s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qb[k], s[i], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const f32x4 a = *(const f32x4*)(sk + S::k(32 * i + col, 2 * k + half));
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qf[4 * k + e], s[i], 0, 0, 0);
        }
      }
    }
    if (!whole_for(t0, wp_min, wp_max)) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!eye.sees(t0 + token(i, v))) s[i][v] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[i][v]);
    top *= p.cs;
    if (__ballot(top > m + kSlack)) {
      const float m1 = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
      const float a = __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= a;
#pragma unroll
      for (int c = 0; c < CT; ++c) acc[c] *= a;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[i][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][v], p.cs, -m));
        if constexpr (!kBf16) l += s[i][v];
      }
    if constexpr (kBf16) {
      bf16x8 pr[2 * NT];  // part c: tokens 16 c + 8 (e / 4) + 4 half + e % 4
#pragma unroll
      for (int c = 0; c < 2 * NT; ++c)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const bf16x2 w = __builtin_convertvector(f32x2{s[c >> 1][8 * (c & 1) + e], s[c >> 1][8 * (c & 1) + e + 1]}, bf16x2);
          l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(s16x2, w), s16x2{0x3f80, 0x3f80}, l, false);
          pr[c][e] = w[0], pr[c][e + 1] = w[1];
        }
      // this lane's source of a transposing read: one token of four, four
      // channels of sixteen
      const int tr = 4 * half + ((lane & 15) >> 2), ch = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
      for (int k = 0; k < 2 * NT; ++k)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          auto at = [&](int t) { return (lds_v4i16*)(sv + S::v(t, (32 * c + ch) >> 3) + (ch & 7)); };
          const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(16 * k + tr));
          const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(16 * k + 8 + tr));
          const v8i16 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), pr[k], acc[c], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int t = token(0, v), e = 32 * c + col;
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(sv[S::v(t, e >> 2) + (e & 3)], s[0][v], acc[c], 0, 0, 0);
        }
    }
  };

  if (u0 < u1) stage(u0, sk0, sv0);
  for (int u = u0; u < u1; u += 2) {
    step(u, sk0, sv0, sk1, sv1);
    if (u + 1 < u1) step(u + 1, sk1, sv1, sk0, sv0);
  }

  if (__syncthreads_or(dirty) && live) add_odd();
  if (live && w0 + col < r1) {
    l += __shfl_xor(l, 32);
    if (!sh.whole()) {
      float* const to = sh.slot(p, D);
      const int rr = w0 - r0 + col;
      if (half == 0) {
        to[rr] = m;
        to[kRows + rr] = l;
      }
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(to + 2 * kRows + rr * D + 32 * c + 8 * i + 4 * half) =
              f32x4{acc[c][4 * i], acc[c][4 * i + 1], acc[c][4 * i + 2], acc[c][4 * i + 3]};
    } else {
      const float inv = 1.0f / l;
      T* const op = (T*)p.o.p + b * p.o.sb + qi * p.o.st + hq * p.o.sh;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = l == 0.0f ? 0.0f : acc[c][4 * i + e] * inv;
          T* const to = op + 32 * c + 8 * i + 4 * half;
          if (VEC) {
            if constexpr (kBf16) *(uint2*)to = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
            else *(f32x4*)to = f32x4{o[0], o[1], o[2], o[3]};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) Elem<T>::store(to, e, o[e]);
          }
        }
    }
  }
}

template <typename T, int D>
hipError_t launch_dim(const AttnParams& p, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.row_tiles * p.splits)), block(kThreads);
  // a tile's rows have to lie within 32-bit offsets
  const int64_t most = (int64_t(1) << 31) / (64 * sizeof(T)) - D;
  if (p.q.vec && p.k.vec && p.v.vec && p.o.vec && p.k.st < most && p.v.st < most)
    hipLaunchKernelGGL((attention_kernel<T, D, true>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((attention_kernel<T, D, false>), grid, block, 0, s, p);
  return hipGetLastError();
}
template <typename T>
hipError_t launch(const AttnParams& p, int D, hipStream_t s) {
  switch (D) {
    case 32: return launch_dim<T, 32>(p, s);
    case 64: return launch_dim<T, 64>(p, s);
    default: return launch_dim<T, 128>(p, s);
  }
}

}  // namespace

hipError_t launch_attention(const AttnParams& p, int dtype, int head_dim, hipStream_t s) {
  const hipError_t e = dtype == DT_BF16 ? launch<uint16_t>(p, head_dim, s) : launch<float>(p, head_dim, s);
  return e != hipSuccess || p.splits == 1 ? e : launch_attention_join(p, dtype, head_dim, s);
}

}  // namespace fluid
