// Attention over keys and values in bf16 or fp32, scores kept in registers.
//
// A workgroup takes 128 rows of one kv head -- (query, head of its group)
// pairs, so that the heads that share keys also share their loads -- and
// walks the tiles of tokens that some row sees; each of its four wavefronts
// has 32 rows.  S^T = K Q^T leaves a lane with one row's scores for 16 of 32
// tokens, and taking the tokens in just that order as the contraction of
// O^T = V^T P^T makes them its operand: nothing is exchanged between lanes
// but the row maximum of two lanes.  bf16 runs 32x32x16 MFMAs (V read from
// LDS by transposing reads), fp32 32x32x2 ones.  Keys and values pass through
// registers into LDS while the tile before is multiplied.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4, kRows = 32 * kWaves;

template <typename T>
struct Cfg;
template <>
struct Cfg<uint16_t> { static constexpr int BN = 64; };
template <>
struct Cfg<float> { static constexpr int BN = 32; };

// LDS places (in elements) of 16-byte piece c of token t.  bf16: pieces are
// exchanged within a row so that eight tokens' equal pieces (K) or four
// tokens' 64-byte runs (V) lie in different banks; fp32 rows are padded.
template <typename T, int D>
struct Place;
template <int D>
struct Place<uint16_t, D> {
  static constexpr int KROW = D, VROW = D;
  __device__ static __forceinline__ int k(int t, int c) { return t * D + 8 * (c ^ (D == 32 ? (t >> 1) & 3 : t & 7)); }
  __device__ static __forceinline__ int v(int t, int c) {
    return t * D + 8 * (c ^ (D == 128 ? 4 * (t & 3) : D == 64 ? 4 * ((t >> 1) & 1) : 0));
  }
};
template <int D>
struct Place<float, D> {
  static constexpr int KROW = D + 4, VROW = D + 8;
  __device__ static __forceinline__ int k(int t, int c) { return t * KROW + 4 * c; }
  __device__ static __forceinline__ int v(int t, int c) { return t * VROW + 4 * c; }
};

template <typename T, int D, bool VEC>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attention_kernel(AttnParams p) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int BN = Cfg<T>::BN, NT = BN / 32, CT = D / 32;
  constexpr int EPP = 16 / sizeof(T), PPR = D / EPP;      // elements a piece, pieces a row
  constexpr int NP = BN * PPR / (64 * kWaves);            // pieces a thread stages of K, and of V
  static_assert(NP * 64 * kWaves == BN * PPR, "whole pieces");
  using Pl = Place<T, D>;
  typedef uint32_t piece __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(1024))) T sk[BN * Pl::KROW];
  __shared__ __attribute__((aligned(1024))) T sv[BN * Pl::VROW];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  // row tiles from the last: with a causal mask the longest start first
  const int rt = p.row_tiles - 1 - x % p.row_tiles;
  x /= p.row_tiles;
  const int h = x % p.kv_heads, b = x / p.kv_heads;
  const int item = (b * p.kv_heads + h) * p.row_tiles + rt;

  const int n = clamp_len(p.kv_len, b, p.kv_tokens);
  const int rows = clamp_len(p.q_len, b, p.q_tokens) * p.group;
  const int r0 = rt * kRows, r1 = min(r0 + kRows, rows);
  if (r0 >= rows) return;
  const int p0 = n - rows / p.group;
  const TileRange range = tile_range(p, p0 + r0 / p.group, p0 + (r1 - 1) / p.group, n, BN);
  const int per = share_tiles(p, range), shares = (range.count + per - 1) / per;
  if (split >= max(shares, 1)) return;
  const int u0 = split * per, u1 = min(u0 + per, range.count);

  // this wavefront's rows
  const int w0 = r0 + 32 * wave;
  const bool live = w0 < r1;
  const int w1 = min(w0 + 32, r1);
  const int wp_min = p0 + w0 / p.group, wp_max = p0 + (w1 - 1) / p.group;
  const int r = min(w0 + col, r1 - 1);
  const int qi = r / p.group, hq = h * p.group + (r - qi * p.group);
  const int pos = p0 + qi;
  const T* qp = (const T*)p.q.p + b * p.q.sb + qi * p.q.st + hq * p.q.sh;
  bf16x8 qb[kBf16 ? D / 16 : 1];
  float qf[kBf16 ? 1 : D / 2];
  if constexpr (kBf16) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      if (VEC) {
        qb[s] = __builtin_bit_cast(bf16x8, *(const piece*)(qp + 16 * s + 8 * half));
      } else {
        v8i16 t;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (short)qp[16 * s + 8 * half + e];
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
  piece kreg[NP], vreg[NP];
  auto fetch_piece = [&](const T* base, int64_t st, int t, int c) -> piece {
    piece w = {0, 0, 0, 0};  // tokens past the end read as zeros
    if (t < n) {
      const T* s = base + t * st + EPP * c;
      if (VEC) {
        w = *(const piece*)s;
      } else {
        T e[EPP];
#pragma unroll
        for (int i = 0; i < EPP; ++i) e[i] = s[i];
        __builtin_memcpy(&w, e, 16);
      }
    }
    return w;
  };
  auto fetch = [&](int u) {
    const int t0 = range.tile(u) * BN;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int k = tid + 64 * kWaves * i, t = t0 + k / PPR, c = k % PPR;
      kreg[i] = fetch_piece(kb, p.k.st, t, c);
      vreg[i] = fetch_piece(vb, p.v.st, t, c);
    }
  };
  auto park = [&]() {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int k = tid + 64 * kWaves * i, t = k / PPR, c = k % PPR;
      *(piece*)(sk + Pl::k(t, c)) = kreg[i];
      *(piece*)(sv + Pl::v(t, c)) = vreg[i];
    }
  };
  const Sight eye = sight(p, pos, n);
  // token of score v of 32-token part i (this lane's half of them)
  auto token = [&](int i, int v) { return 32 * i + 8 * (v >> 2) + 4 * half + (v & 3); };

  float m, l;
  f32x16 acc[CT];
  auto pass = [&](bool safe) -> bool {
    bool masked_any = false;
    m = kLow;
    l = 0.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = f32x16{};
    if (u0 < u1) fetch(u0);
    for (int u = u0; u < u1; ++u) {
      __syncthreads();
      park();
      __syncthreads();
      if (u + 1 < u1) fetch(u + 1);
      if (!live) continue;
      const int t0 = range.tile(u) * BN, t1 = t0 + BN;
      const bool whole = t1 <= n && (!p.causal || t1 - 1 <= wp_min) &&
                         (p.window <= 0 || t1 <= p.sinks ||
                          (t0 > wp_max - p.window && (p.causal || t1 <= wp_min + p.window)));
      masked_any |= !whole;
      f32x16 s[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        s[i] = f32x16{};
        if constexpr (kBf16) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const bf16x8 a = *(const bf16x8*)(sk + Pl::k(32 * i + col, 2 * k + half));
            s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qb[k], s[i], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int k = 0; k < D / 8; ++k) {
            const f32x4 a = *(const f32x4*)(sk + Pl::k(32 * i + col, 2 * k + half));
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qf[4 * k + e], s[i], 0, 0, 0);
          }
        }
      }
      if (!whole) {
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
      if (__ballot(top > m)) {
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
          l += s[i][v];
        }
      if constexpr (kBf16) {
        bf16x8 pr[2 * NT];  // part c: tokens 16 c + 8 (e / 4) + 4 half + e % 4
#pragma unroll
        for (int c = 0; c < 2 * NT; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) pr[c][e] = (__bf16)s[c >> 1][8 * (c & 1) + e];
        // this lane's source of a transposing read: token e % 4 of four, four
        // channels of sixteen
        const int tr = 4 * half + ((lane & 15) >> 2), ch = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
#pragma unroll
          for (int k = 0; k < 2 * NT; ++k) {
            auto at = [&](int t) {
              const int e = 32 * c + ch;
              return (__attribute__((address_space(3))) v4i16*)(sv + Pl::v(t, e >> 3) + (e & 7));
            };
            const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(16 * k + tr));
            const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(16 * k + 8 + tr));
            v8i16 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            if (!safe || whole) {
              acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), pr[k], acc[c], 0, 0, 0);
            } else {
              f32x16 sum = acc[c];
              for (int row = 0; row < 32; ++row) {
                const Sight other = sight(p, __shfl(pos, row), n);
                v8i16 w = a;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (!other.sees(t0 + 16 * k + 8 * (e >> 2) + 4 * half + (e & 3))) w[e] = 0;
                const f32x16 one =
                    __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pr[k], acc[c], 0, 0, 0);
                if (col == row) sum = one;
              }
              acc[c] = sum;
            }
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int t = token(0, v), e = 32 * c + col;
            const float a = sv[Pl::v(t, e >> 2) + (e & 3)];
            if (!safe || whole) {
              acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, s[0][v], acc[c], 0, 0, 0);
            } else {
              f32x16 sum = acc[c];
              for (int row = 0; row < 32; ++row) {
                const float w = sight(p, __shfl(pos, row), n).sees(t0 + t) ? a : 0.0f;
                const f32x16 one = __builtin_amdgcn_mfma_f32_32x32x2f32(w, s[0][v], acc[c], 0, 0, 0);
                if (col == row) sum = one;
              }
              acc[c] = sum;
            }
          }
      }
    }
    bool odd = false;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int v = 0; v < 16; ++v) odd |= !(fabsf(acc[c][v]) <= 3.402823466e38f);
    return __syncthreads_or(masked_any && odd);
  };
  if (pass(false)) pass(true);
  if (!live || w0 + col >= r1) return;

  l += __shfl_xor(l, 32);
  if (shares > 1) {
    float* to = p.ws + ((int64_t)item * p.splits + split) * (kRows * (D + 2));
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
    return;
  }
  const float inv = 1.0f / l;
  T* op = (T*)p.o.p + b * p.o.sb + qi * p.o.st + hq * p.o.sh;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = l == 0.0f ? 0.0f : acc[c][4 * i + e] * inv;
      T* to = op + 32 * c + 8 * i + 4 * half;
      if (VEC) {
        if constexpr (kBf16) *(uint2*)to = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
        else *(f32x4*)to = f32x4{o[0], o[1], o[2], o[3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) Elem<T>::store(to, e, o[e]);
      }
    }
}

template <typename T, int D>
hipError_t launch_dim(const AttnParams& p, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.row_tiles * p.splits)), block(64 * kWaves);
  if (p.q.vec && p.k.vec && p.v.vec && p.o.vec)
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
