// Attention over the 4-bit cache.
//
// S^T = K Q^T and O^T = V^T P^T on the f16 matrix cores (16x16x32), one
// wavefront on 32 tokens at a time with nothing in LDS.  Row t of a K operand
// may be any token and slot k of a V operand likewise, as long as P agrees:
// with tokens 8 (t / 4) + t % 4 (and + 4) as the rows of the two K operands,
// the scores a lane gets back are those of the eight tokens of octet
// lane / 16, which is what the P operand wants of it, and the V operand wants
// that octet's eight nibbles of one channel: a word of the cache.  A nibble
// pair becomes two f16 in one AND-OR and one fused multiply-add, with the
// shift about 1.5 instructions a value; the cache's values are exact f16, so
// a dequantised operand loses nothing.
//
// Queries are scaled by a power of two per row before they become f16 (bf16
// ones then are exact but for what lies 2^-14 below a row's largest); fp32
// queries and probabilities are two f16 parts each and two products.
// Probabilities are scaled by 2^15, where f16 has its whole range below them.
//
// The wavefronts of a workgroup take token tiles in turn and join their sums
// in LDS; long caches are split over workgroups, joined by a second kernel.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

constexpr int kWaves = 4;
constexpr float kPBits = 15.0f;

__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// over the four lanes that share lane % 16
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t w[N]) {
  typedef uint32_t vec __attribute__((ext_vector_type(N)));
  if constexpr (N == 1) {
    w[0] = *(const uint32_t*)p;
  } else {
    const vec v = *(const vec*)p;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = v[i];
  }
}

// The cache's words of one tile that a lane needs.
template <int D>
struct KvTile {
  static constexpr int G = D / 32, WPL = D == 32 ? 2 : 4, NC = D == 32 ? 1 : D / 64;
  uint32_t kw[2][G], kp[2][G];
  uint32_t vw[NC][WPL], vs[NC][4], vb[NC][4];

  __device__ __forceinline__ void load(const uint8_t* blk, int P, int slot, int lane) {
    const int m = lane & 15, g = lane >> 4;
    const int t = slot + 8 * (m >> 2) + (m & 3);
    const uint8_t* kpairs = blk + P * (D / 2);
    const uint8_t* v = kpairs + P * (4 * G) + ((slot >> 3) + g) * (4 * D);
    const uint8_t* vpairs = kpairs + P * (4 * G + D / 2) + ((slot >> 3) + g) * (32 * G);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_words<G>(blk + (t + 4 * i) * (D / 2) + g * (4 * G), kw[i]);
      load_words<G>(kpairs + (t + 4 * i) * (4 * G), kp[i]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      load_words<WPL>(v + 256 * c + 4 * WPL * m, vw[c]);
      const uint8_t* sp = vpairs + 32 * (D == 32 ? 0 : 2 * c + (m >> 3));
      load_words<4>(sp, vs[c]);
      load_words<4>(sp + 16, vb[c]);
    }
  }
};

template <typename T, int D, int MT>
__global__ __launch_bounds__(64 * kWaves) void kv_attention_kernel(AttnParams p) {
  constexpr bool kTwo = sizeof(T) == 4;  // operands in two f16 parts
  constexpr int G = D / 32, R = 16 * MT;
  using Tile = KvTile<D>;
  constexpr int WPL = Tile::WPL, NC = Tile::NC;
  __shared__ float sh_m[kWaves][R], sh_l[kWaves][R];
  __shared__ __attribute__((aligned(16))) float sh_o[kWaves][R][D + 4];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  int x = blockIdx.x;
  const int split = x % p.splits;
  x /= p.splits;
  const int item = x;
  const int rt = x % p.row_tiles;
  x /= p.row_tiles;
  const int h = x % p.kv_heads, b = x / p.kv_heads;

  const int n = clamp_len(p.kv_len, b, p.kv_tokens);
  const int rows = clamp_len(p.q_len, b, p.q_tokens) * p.group;
  const int r0 = rt * R, r1 = min(r0 + R, rows);
  if (r0 >= rows) return;
  const int p0 = n - rows / p.group;  // position of row 0's query
  const int p_min = p0 + r0 / p.group, p_max = p0 + (r1 - 1) / p.group;
  const TileRange range = tile_range(p, p_min, p_max, n, kKvTile);
  const int per = share_tiles(p, range), shares = (range.count + per - 1) / per;
  if (split >= max(shares, 1)) return;
  const int u0 = split * per, u1 = min(u0 + per, range.count);

  // queries, as the second operand: lane holds channels 32 j + 8 g4 .. +7 of
  // its row
  f16x8 qh[MT][G], ql[MT][kTwo ? G : 1];
  float cs[MT];   // score to a power of two's exponent
  int pos[MT];
  Sight eye[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = min(r0 + 16 * mt + col, r1 - 1);
    const int i = r / p.group, hq = h * p.group + (r - i * p.group);
    pos[mt] = p0 + i;
    eye[mt] = sight(p, pos[mt], n);
    const T* q = (const T*)p.q.p + b * p.q.sb + i * p.q.st + hq * p.q.sh + 8 * g4;
    float f[G][8], top = 0.0f;
#pragma unroll
    for (int j = 0; j < G; ++j) {
      load8(q + 32 * j, p.q.vec, f[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[j][e]));
    }
    top = col_max(top);
    // 2^-e brings the largest to [1, 2); a row of zeros, infinities or NaN
    // keeps its values
    int e = (int)((__float_as_uint(top) >> 23) & 0xff) - 127;
    if (e == 128 || e == -127) e = 0;
    const float down = __builtin_ldexpf(1.0f, -e);
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float y = f[j][k] * down;
        const _Float16 hi = (_Float16)y;
        qh[mt][j][k] = hi;
        if constexpr (kTwo) ql[mt][j][k] = (_Float16)(y - (float)hi);
      }
    cs[mt] = p.cs * __builtin_ldexpf(1.0f, e);
  }

  float m[MT], l[MT];
  f32x4 acc[MT][NC][WPL];
  const int P = 1 << p.c.log_page;
  const int32_t* const pages = p.c.pages + b * p.c.table_stride;
  auto page_of = [&](int u) -> int {
    const int id = u < u1 ? pages[(range.tile(u) * kKvTile) >> p.c.log_page] : -1;
    return id < p.c.n_pages ? id : -1;
  };

  // A pass over the tokens; `safe` takes the rows of a tile with masked tokens
  // one by one, which keeps what a masked token's value holds (0 times an
  // infinity) out of the other rows.
  auto pass = [&](bool safe) -> bool {
    bool masked_any = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt] = kLow;
      l[mt] = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < WPL; ++j) acc[mt][c][j] = f32x4{0, 0, 0, 0};
    }
    for (int u = u0 + wave; u < u1; u += kWaves) {
      const int t0 = range.tile(u) * kKvTile;
      const int page = page_of(u);
      if (page < 0) continue;
      Tile tile;
      tile.load(p.c.pool + ((int64_t)page * p.c.kv_heads + h) * p.c.block, P, t0 & (P - 1), lane);
      // every row sees every token
      const bool whole = t0 + kKvTile - 1 <= p_min &&
                         (p.window <= 0 || t0 > p_max - p.window || t0 + kKvTile <= p.sinks);
      masked_any |= !whole;
      float s[MT][2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x4 sc[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sc[mt] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const f16x8 k = word_values(tile.kw[i][j], tile.kp[i][j]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            if constexpr (kTwo) sc[mt] = mfma(k, ql[mt][j], sc[mt]);
            sc[mt] = mfma(k, qh[mt][j], sc[mt]);
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[mt][i][r] = sc[mt][r] * cs[mt];
      }
      if (!whole) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (!eye[mt].sees(t0 + 8 * g4 + 4 * i + r)) s[mt][i][r] = -INFINITY;
      }
      f16x8 ph[MT], pl[kTwo ? MT : 1];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float top = s[mt][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[mt][e >> 2][e & 3]);
        if (__ballot(top > m[mt])) {
          const float m1 = fmaxf(m[mt], col_max(top));
          const float a = __builtin_amdgcn_exp2f(m[mt] - m1);
          m[mt] = m1;
          l[mt] *= a;
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < WPL; ++j) acc[mt][c][j] *= a;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = __builtin_amdgcn_exp2f(s[mt][e >> 2][e & 3] - m[mt] + kPBits);
          l[mt] += f;
          const _Float16 hi = (_Float16)f;
          ph[mt][e] = hi;
          if constexpr (kTwo) pl[mt][e] = (_Float16)(f - (float)hi);
        }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < WPL; ++j) {
          f16x2 vs[4], vb[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            vs[i] = __builtin_bit_cast(f16x2, tile.vs[c][i]);
            vb[i] = __builtin_bit_cast(f16x2, tile.vb[c][i]);
          }
          const f16x8 v = word_values(tile.vw[c][j], vs, vb);
          if (!safe || whole) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              if constexpr (kTwo) acc[mt][c][j] = mfma(v, pl[mt], acc[mt][c][j]);
              acc[mt][c][j] = mfma(v, ph[mt], acc[mt][c][j]);
            }
          } else {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              f32x4 sum = acc[mt][c][j];
              for (int row = 0; row < 16; ++row) {
                const Sight other = sight(p, __shfl(pos[mt], row), n);
                f16x8 w = v;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (!other.sees(t0 + 8 * g4 + e)) w[e] = (_Float16)0.0f;
                f32x4 one = acc[mt][c][j];
                if constexpr (kTwo) one = mfma(w, pl[mt], one);
                one = mfma(w, ph[mt], one);
                if (col == row) sum = one;
              }
              acc[mt][c][j] = sum;
            }
          }
        }
    }
    bool odd = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < WPL; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) odd |= !(fabsf(acc[mt][c][j][r]) <= 3.402823466e38f);
    }
    return masked_any && __ballot(odd) != 0;
  };
  if (pass(false)) pass(true);

  // join the wavefronts
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float sum = col_sum(l[mt]);
    const int r = 16 * mt + col;
    if (g4 == 0) {
      sh_m[wave][r] = m[mt];
      sh_l[wave][r] = sum;
    }
    float* o = sh_o[wave][r];
    if constexpr (D == 32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) o[8 * g4 + 2 * i + j] = acc[mt][0][j][i];
    } else {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(o + 64 * c + 16 * g4 + 4 * i) =
              f32x4{acc[mt][c][0][i], acc[mt][c][1][i], acc[mt][c][2][i], acc[mt][c][3][i]};
    }
  }
  __syncthreads();
  constexpr int TPR = D / 8;  // threads a row
  for (int k = threadIdx.x; k < R * TPR; k += 64 * kWaves) {
    const int r = k / TPR, c = 8 * (k - r * TPR);
    if (r0 + r >= r1) continue;
    float top = sh_m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh_m[w][r]);
    float sum = 0.0f, o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float a = __builtin_amdgcn_exp2f(sh_m[w][r] - top);
      sum += a * sh_l[w][r];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += a * sh_o[w][r][c + e];
    }
    if (shares > 1) {
      float* to = p.ws + ((int64_t)item * p.splits + split) * (R * (D + 2));
      if (c == 0) {
        to[r] = top;
        to[R + r] = sum;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) to[2 * R + r * D + c + e] = o[e];
    } else {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = sum == 0.0f ? 0.0f : o[e] * inv;
      const int i = (r0 + r) / p.group, hq = h * p.group + (r0 + r - i * p.group);
      store8((T*)p.o.p + b * p.o.sb + i * p.o.st + hq * p.o.sh + c, p.o.vec, o);
    }
  }
}

template <typename T, int D, int MT>
hipError_t launch_rows(const AttnParams& p, hipStream_t s) {
  const int64_t items = (int64_t)p.batch * p.kv_heads * p.row_tiles;
  hipLaunchKernelGGL((kv_attention_kernel<T, D, MT>), dim3((uint32_t)(items * p.splits)), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}
template <typename T>
hipError_t launch(const AttnParams& p, int D, hipStream_t s) {
  const bool two = p.row_tile == 32;
  switch (D) {
    case 32: return two ? launch_rows<T, 32, 2>(p, s) : launch_rows<T, 32, 1>(p, s);
    case 64: return two ? launch_rows<T, 64, 2>(p, s) : launch_rows<T, 64, 1>(p, s);
    default: return two ? launch_rows<T, 128, 2>(p, s) : launch_rows<T, 128, 1>(p, s);
  }
}

}  // namespace

hipError_t launch_kv_attention(const AttnParams& p, int dtype, int head_dim, hipStream_t s) {
  const hipError_t e = dtype == DT_BF16 ? launch<uint16_t>(p, head_dim, s) : launch<float>(p, head_dim, s);
  return e != hipSuccess || p.splits == 1 ? e : launch_attention_join(p, dtype, head_dim, s);
}

}  // namespace fluid
