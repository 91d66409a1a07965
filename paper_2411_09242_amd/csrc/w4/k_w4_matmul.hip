// A few rows times a matrix in 4 bits, on the bf16 matrix cores (16x16x32).
//
// A nibble in bits 3 .. 6 of a bf16 with the exponent of 16 reads 16 + n, exact,
// so a word becomes an operand in eight instructions; a group's products with x
// are summed in fp32, and so are x's own (a product with ones): the group adds
// s sum x (16 + n) + b sum x.  No weight is rounded.  A lane's words are one row's,
// so it needs that row's pair alone.
//
// A workgroup has 16 rows of the matrix (and of the gate), whose blocks of 128
// channels its wavefronts take in turn; their sums are added through LDS in the
// order of the wavefronts.
#include "../attn/dev_attn.h"
#include "launch_w4.h"

namespace fluid {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A word's eight levels as 16 + n in bf16.
__device__ __forceinline__ u32x4 levels(uint32_t w) {
  constexpr uint32_t mask = 0x00780078, sixteen = 0x41804180;
  return u32x4{((w << 3) & mask) | sixteen, ((w >> 1) & mask) | sixteen, ((w >> 5) & mask) | sixteen,
               ((w >> 9) & mask) | sixteen};
}

// Eight channels of x as operands whose sum they are.
template <typename T>
struct Parts;
template <>
struct Parts<uint16_t> {
  static constexpr int N = 1;
  u32x4 p[1];
  __device__ __forceinline__ void load(const uint16_t* x, int left, bool vec) {
    if (left >= 8 && vec) {
      p[0] = *(const u32x4*)x;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        p[0][i] = (2 * i < left ? x[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)x[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void clear() { p[0] = u32x4{}; }
};
template <>
struct Parts<float> {
  static constexpr int N = 3;
  u32x4 p[3];
  __device__ __forceinline__ void load(const float* x, int left, bool vec) {
    float v[8];
    if (left >= 8 && vec) {
      const f32x4 a = ((const f32x4*)x)[0], b = ((const f32x4*)x)[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < left ? x[e] : 0.0f;
    }
    // the first two parts are cut off, so that what is left is exact
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = v[2 * i], b = v[2 * i + 1];
      const uint32_t ah = __float_as_uint(a) & 0xffff0000u, bh = __float_as_uint(b) & 0xffff0000u;
      const float a1 = a - __uint_as_float(ah), b1 = b - __uint_as_float(bh);
      const uint32_t am = __float_as_uint(a1) & 0xffff0000u, bm = __float_as_uint(b1) & 0xffff0000u;
      p[0][i] = (ah >> 16) | bh;
      p[1][i] = (am >> 16) | bm;
      p[2][i] = pack_bf16(a1 - __uint_as_float(am), b1 - __uint_as_float(bm));
    }
  }
  __device__ __forceinline__ void clear() { p[0] = p[1] = p[2] = u32x4{}; }
};

// MT: tiles of 16 rows of x
template <typename T, int G, int MT, bool GATE>
__global__ __launch_bounds__(MT == 1 ? 1024 : 512) void w4_matmul_kernel(W4Params p) {
  constexpr int MATS = GATE ? 2 : 1, GROUPS = 128 / G, STEPS = G / 32;
  extern __shared__ float sums[];  // [wavefront][matrix][row tile][256]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int tile = blockIdx.x, m0 = blockIdx.y * (16 * MT);
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  f32x4 y[MATS][MT] = {};
  for (int c = wave; c < p.blocks; c += p.waves) {
    const int64_t at = (int64_t)tile * p.blocks + c;
    u32x4 w[MATS];
    f16x2 sb[MATS][GROUPS];
#pragma unroll
    for (int a = 0; a < MATS; ++a) {
      const W4Arg& of = a ? p.gate : p.w;
      w[a] = *(const u32x4*)(of.words + at * 1024 + lane * 16);
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) sb[a][i] = *(const f16x2*)(of.pairs + (at * 16 + r) * (4 * GROUPS) + 4 * i);
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      f32x4 part[MATS][MT] = {}, all[MT] = {};
#pragma unroll
      for (int j = i * STEPS; j < (i + 1) * STEPS; ++j) {
        const int ch = 128 * c + 32 * j + 8 * g;
        Parts<T> x[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int row = m0 + 16 * t + r;
          x[t].clear();
          if (row < p.m && ch < p.k) x[t].load((const T*)p.x + row * p.xs + ch, p.k - ch, p.vec);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int k = 0; k < Parts<T>::N; ++k) all[t] = mfma(x[t].p[k], ones, all[t]);
#pragma unroll
        for (int a = 0; a < MATS; ++a) {
          const u32x4 l = levels(w[a][j]);
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int k = 0; k < Parts<T>::N; ++k) part[a][t] = mfma(x[t].p[k], l, part[a][t]);
        }
      }
#pragma unroll
      for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[a][t][e] += __builtin_fmaf((float)sb[a][i][0], part[a][t][e], (float)sb[a][i][1] * all[t][e]);
    }
  }
#pragma unroll
  for (int a = 0; a < MATS; ++a)
#pragma unroll
    for (int t = 0; t < MT; ++t) *(f32x4*)(sums + (((wave * MATS + a) * MT + t) * 64 + lane) * 4) = y[a][t];
  __syncthreads();
  for (int at = threadIdx.x; at < MT * 256; at += blockDim.x) {
    const int t = at >> 8, m = m0 + (at >> 4), n = 16 * tile + (at & 15);
    if (m >= p.m || n >= p.n) continue;
    const int from = (16 * ((at >> 6) & 3) + (at & 15)) * 4 + ((at >> 4) & 3);
    float v[MATS];
#pragma unroll
    for (int a = 0; a < MATS; ++a) {
      v[a] = 0.0f;
      for (int u = 0; u < p.waves; ++u) v[a] += sums[((u * MATS + a) * MT + t) * 256 + from];
    }
    float o = v[0];
    if constexpr (GATE) o *= v[1] / (1.0f + expf(-v[1]));
    if (p.add) o += Elem<T>::load((const T*)p.add + m * p.as, n);
    Elem<T>::store((T*)p.out + m * p.os, n, o);
  }
}

template <typename T, int G, int MT, bool GATE>
hipError_t launch(const W4Params& p, hipStream_t s) {
  const dim3 grid(p.tiles, (p.m + 16 * MT - 1) / (16 * MT)), block(64 * p.waves);
  hipLaunchKernelGGL((w4_matmul_kernel<T, G, MT, GATE>), grid, block, p.waves * (GATE ? 2 : 1) * MT * 1024, s, p);
  return hipGetLastError();
}
template <typename T, int G>
hipError_t launch_rows(const W4Params& p, hipStream_t s) {
  const bool gate = p.gate.words != nullptr;
  if (p.m <= 16) return gate ? launch<T, G, 1, true>(p, s) : launch<T, G, 1, false>(p, s);
  if (p.m <= 32) return gate ? launch<T, G, 2, true>(p, s) : launch<T, G, 2, false>(p, s);
  return gate ? launch<T, G, 4, true>(p, s) : launch<T, G, 4, false>(p, s);
}
template <typename T>
hipError_t launch_group(const W4Params& p, hipStream_t s) {
  switch (p.group) {
    case 32: return launch_rows<T, 32>(p, s);
    case 64: return launch_rows<T, 64>(p, s);
    default: return launch_rows<T, 128>(p, s);
  }
}

}  // namespace

hipError_t launch_w4_matmul(const W4Params& p, int dtype, hipStream_t s) {
  return dtype == DT_BF16 ? launch_group<uint16_t>(p, s) : launch_group<float>(p, s);
}

}  // namespace fluid
