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
// ones then are exact but for what lies 2^-14 below a row's largest, rounded to
// 2^-25 of it).  The weights of bf16 queries are rounded to f16: 11 bits, where
// the output has 8, and half the products of two parts (32 x 8192 tokens: error
// against 64 bits 0.17 % of the output, as with fp32 weights).  fp32 queries and
// weights are two f16 parts each and two products: 22 bits.
//
// The wavefronts of a workgroup take token tiles in turn and join their sums
// in LDS; long caches are split over workgroups, joined by a second kernel.
//
// Bound by reading the cache once it is long: 131072 tokens of 8 heads of 128,
// 168 MB, take 30 to 32 us (5.4 TB/s; a copy of 4 GiB has 4.7, reads alone up to
// 7.2) and 5 for the join; 32 sequences of 2581 to 8192 tokens, 222 MB, 48.
// Vector instructions are 60 % of the cycles and MFMA 13 %, so that three
// wavefronts a SIMD have to cover the loads; a fourth has 128 registers and
// spills, a whole tile ahead in registers of its own was slower too.  Short
// caches are bound by the launch and four dependent loads (lengths, page, keys
// and values): 8 sequences of up to 1000 tokens of 12 heads of 64 in fp32, up to
// five queries each, 10 us.
#include "kv_tile.h"
#include "launch_attn.h"

namespace fluid {

namespace {

// The running maximum may lag a row's largest score by kSlack powers of two, so
// that the sums are hardly ever scaled; weights are scaled by 2^kPBits, at most
// 2^15 then, where f16 has its whole range below them.
constexpr float kSlack = 4.0f, kPBits = 15.0f - kSlack;

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

// Which halves of a word of pairs (two tokens' s and b) may stand for an infinity
// or a NaN, as bits 0 and 1: values lie between those of nibbles 0 and 15.  Slots
// that were never written hold any bytes, and their finite pairs may have values
// past f16's range.
__device__ __forceinline__ uint32_t odd_pairs(uint32_t s, uint32_t b) {
  const f16x2 ss = __builtin_bit_cast(f16x2, s), bb = __builtin_bit_cast(f16x2, b);
  const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(f16x2{16, 16}, ss, bb));
  const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(f16x2{31, 31}, ss, bb));
  auto none = [](uint32_t w, uint32_t exponent) -> uint32_t { return (w & exponent) == exponent; };
  return none(lo, 0x7c00u) | none(hi, 0x7c00u) | (none(lo, 0x7c000000u) | none(hi, 0x7c000000u)) << 1;
}

template <typename T, int D, int MT, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 16 ? 4 : MT == 1 && NW == 4 ? 3 : 2)))
void kv_attention_kernel(AttnParams p) {
  constexpr bool kTwo = sizeof(T) == 4;  // operands in two f16 parts
  constexpr int G = D / 32, R = 16 * MT;
  using Tile = KvTile<D>;
  constexpr int WPL = Tile::WPL, NC = Tile::NC;
  __shared__ float sh_m[NW][R], sh_l[NW][R];
  __shared__ __attribute__((aligned(16))) float sh_o[NW][R][D + 4];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  const typename Tile::Lane at = Tile::lane_offsets(lane);
  const int P = 1 << p.c.log_page;
  const Magic mg;

  Share sh;
  if (!sh.find(p, blockIdx.x)) return;
  const Item& it = sh.item;
  const int b = it.b, h = it.h, n = it.n, r0 = it.r0, r1 = it.r1, p0 = it.p0;
  const int p_min = it.p_min(p), p_max = it.p_max(p);
  const TileRange range = it.range;
  const int u0 = sh.first, u1 = sh.end;

  // queries: a lane holds channels 32 j + 8 g4 .. +7 of its row
  Eight<T> raw[MT][G];
  int pos[MT];
  Sight eye[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = min(r0 + 16 * mt + col, r1 - 1);
    const int i = (int)fdiv(r, p.div_group), hq = h * p.group + (r - i * p.group);
    pos[mt] = p0 + i;
    eye[mt] = sight(p, pos[mt], n);
    const T* q = (const T*)p.q.p + b * p.q.sb + i * p.q.st + hq * p.q.sh + 8 * g4;
#pragma unroll
    for (int j = 0; j < G; ++j) raw[mt][j].load(q + 32 * j, p.q.vec);
  }

  const int32_t* const pages = p.c.pages + b * p.c.table_stride;
  // A page outside the pool holds no tokens: its tiles are read from page 0 and
  // none of their tokens is seen.
  auto page_of = [&](int u) { return uniform_load(pages, (range.tile(u) * kKvTile) >> p.c.log_page); };
  auto block = [&](int page) {
    return p.c.pool + ((int64_t)((uint32_t)page < (uint32_t)p.c.n_pages ? page : 0) * p.c.kv_heads + h) * p.c.block;
  };
  auto slot = [&](int u) { return (range.tile(u) * kKvTile) & (P - 1); };
  int u = u0 + wave, page = -1;
  Tile tile;
  if (u < u1) {
    page = page_of(u);
    tile.load_k(block(page), P, slot(u), at);
    tile.load_v(block(page), P, slot(u), at);
  }

  f16x8 qh[MT][G], ql[MT][kTwo ? G : 1];
  float cs[MT];  // the scale with the power of two taken out of the row
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float f[G][8], top = 0.0f;
#pragma unroll
    for (int j = 0; j < G; ++j) {
      raw[mt][j].floats(f[j]);
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
    // kept within fp32: 0 would make NaN of a hidden score, infinity of a score of
    // 0; past the ends scores are 0, or too far apart for two weights, all the same
    cs[mt] = fminf(fmaxf(p.cs * __builtin_ldexpf(1.0f, e), 1.17549435e-38f), 3.402823466e38f);
  }

  float m[MT], l[MT];
  bool wide[MT];  // some row is past_fused
  f32x4 acc[MT][NC][WPL];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = kLow;
    l[mt] = 0.0f;
    wide[mt] = false;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < WPL; ++j) acc[mt][c][j] = f32x4{0, 0, 0, 0};
  }

  // A tile's keys are loaded once those of the tile before are used, its values
  // likewise: about half a tile is always on its way, in the same registers.
  while (u < u1) {
    const int t0 = range.tile(u) * kKvTile;
    const int after = min(u + NW, u1 - 1), next = page_of(after);
    const bool dark = (uint32_t)page >= (uint32_t)p.c.n_pages;
    // every row sees every token
    const bool whole = !dark && t0 + kKvTile - 1 <= p_min &&
                       (p.window <= 0 || t0 > p_max - p.window || t0 + kKvTile <= p.sinks);
    f32x4 sc[MT][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) sc[mt][i] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < G; ++j) {
        const f16x8 k = word_values(mg, tile.kw[i][j], tile.kp[i][j]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if constexpr (kTwo) sc[mt][i] = mfma(k, ql[mt][j], sc[mt][i]);
          sc[mt][i] = mfma(k, qh[mt][j], sc[mt][i]);
        }
      }
    }
    tile.load_k(block(next), P, slot(after), at);
    if (!whole) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (dark | !eye[mt].sees(t0 + 8 * g4 + 4 * i + r)) sc[mt][i][r] = -INFINITY;
      // Weight 0 times a value that is no number would still be none.  So the
      // groups that may hold one become zeros here, and NaN goes into the sums of
      // the rows that do see them.
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uint32_t odd = 0;  // of this lane's octet and group
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= odd_pairs(tile.vs[c][i], tile.vb[c][i]) << (2 * i);
        if (__builtin_expect(__ballot(odd != 0) != 0, 0)) {
          // a lane's sums belong to the channels 64 c + 16 g4 .. +15, of the
          // group that the source lanes 8 (g4 / 2) of each sixteen hold
          uint32_t of = 0;
#pragma unroll
          for (int o = 0; o < 4; ++o) of |= __shfl(odd, 16 * o + (D == 32 ? 0 : 8 * (g4 >> 1))) << (8 * o);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            bool hit = false;
            for (int t = 0; t < kKvTile; ++t) hit |= !dark && (of >> t & 1) && eye[mt].sees(t0 + t);
            if (hit) {
#pragma unroll
              for (int j = 0; j < WPL; ++j) acc[mt][c][j] = f32x4{NAN, NAN, NAN, NAN};
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t keep = ((odd >> (2 * i)) & 1 ? 0u : 0xffffu) | ((odd >> (2 * i + 1)) & 1 ? 0u : 0xffff0000u);
            tile.vs[c][i] &= keep;
            tile.vb[c][i] &= keep;
          }
        }
      }
    }
    f16x8 ph[MT], pl[kTwo ? MT : 1];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float top = sc[mt][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[mt][e >> 2][e & 3]);
      top *= cs[mt];
      if (__ballot(top - m[mt] > kSlack)) {
        const float m1 = fmaxf(m[mt], col_max(top));
        const float a = __builtin_amdgcn_exp2f(m[mt] - m1);
        m[mt] = m1;
        l[mt] *= a;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < WPL; ++j) acc[mt][c][j] *= a;
        wide[mt] = __ballot(past_fused(m[mt])) != 0;
      }
      float factor = cs[mt], shift = kPBits - m[mt];
      if (__builtin_expect(wide[mt], 0)) {
#pragma clang fp contract(off)
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[mt][e >> 2][e & 3] = sc[mt][e >> 2][e & 3] * cs[mt] - m[mt];
        factor = 1.0f;
        shift = kPBits;
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const f32x2 f = {__builtin_amdgcn_exp2f(__builtin_fmaf(sc[mt][e >> 2][e & 3], factor, shift)),
                         __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mt][e >> 2][(e & 3) + 1], factor, shift))};
        l[mt] += f[0];
        l[mt] += f[1];
        const f16x2 hi = __builtin_convertvector(f, f16x2);
        ph[mt][e] = hi[0], ph[mt][e + 1] = hi[1];
        if constexpr (kTwo) pl[mt][e] = (_Float16)(f[0] - (float)hi[0]), pl[mt][e + 1] = (_Float16)(f[1] - (float)hi[1]);
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
        const f16x8 v = word_values(mg, tile.vw[c][j], vs, vb);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if constexpr (kTwo) acc[mt][c][j] = mfma(v, pl[mt], acc[mt][c][j]);
          acc[mt][c][j] = mfma(v, ph[mt], acc[mt][c][j]);
        }
      }
    tile.load_v(block(next), P, slot(after), at);
    u += NW;
    page = next;
  }

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
  for (int k = threadIdx.x; k < R * TPR; k += 64 * NW) {
    const int r = k / TPR, c = 8 * (k - r * TPR);
    if (r0 + r >= r1) continue;
    float top = sh_m[0][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, sh_m[w][r]);
    float sum = 0.0f, o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float a = __builtin_amdgcn_exp2f(sh_m[w][r] - top);
      sum += a * sh_l[w][r];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += a * sh_o[w][r][c + e];
    }
    if (!sh.whole()) {
      float* to = sh.slot(p, D);
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
      const int i = (int)fdiv(r0 + r, p.div_group), hq = h * p.group + (r0 + r - i * p.group);
      store8((T*)p.o.p + b * p.o.sb + i * p.o.st + hq * p.o.sh + c, p.o.vec, o);
    }
  }
}

template <typename T, int D>
hipError_t launch_dim(const AttnParams& p, hipStream_t s) {
  constexpr int MANY = kv_waves(D);
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.row_tiles * p.splits)), block(64 * p.waves);
  if (p.row_tile == 32) hipLaunchKernelGGL((kv_attention_kernel<T, D, 2, 4>), grid, block, 0, s, p);
  else if (p.waves == MANY) hipLaunchKernelGGL((kv_attention_kernel<T, D, 1, MANY>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((kv_attention_kernel<T, D, 1, 4>), grid, block, 0, s, p);
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

hipError_t launch_kv_attention(const AttnParams& p, int dtype, int head_dim, hipStream_t s) {
  const hipError_t e = dtype == DT_BF16 ? launch<uint16_t>(p, head_dim, s) : launch<float>(p, head_dim, s);
  return e != hipSuccess || p.splits == 1 ? e : launch_attention_join(p, dtype, head_dim, s);
}

}  // namespace fluid
