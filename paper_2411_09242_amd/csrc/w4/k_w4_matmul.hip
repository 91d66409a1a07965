// Up to 16 rows times a matrix in 4 bits, on the bf16 matrix cores (16x16x32).
//
// A workgroup has 16 or 32 rows of the matrix (and of the gate), whose blocks of
// 128 channels its wavefronts take in turn, one ahead of the products; their sums
// are added through LDS in the order of the wavefronts.
//
// Bound by memory where the matrix is large: one row times 4096 x 11008 (24 MB) 8.2 us,
// the gated product with two of 11008 x 4096 (48 MB) 11.0 us (4.4 TB/s).  More rows
// are bound by x, which every workgroup reads from L2: 16 rows times 4096 x 11008 take
// 15 us.  Small ones are the launch and two rounds of loads, 4.6 to 4.9 us.
#include "launch_w4.h"
#include "w4_tile.h"

namespace fluid {

namespace {

// NT: tiles of 16 rows of the matrix.
template <typename T, int G, int NT, bool GATE, Load HOW>
__global__ __launch_bounds__(GATE || NT == 2 || sizeof(T) == 4 ? 512 : 1024) void w4_few_kernel(W4Params p) {
  constexpr int MATS = GATE ? 2 : 1, GROUPS = 128 / G, STEPS = G / 32, P = Rows<T>::N;
  extern __shared__ float sums[];  // [wavefront][matrix][tile][256]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int tile0 = blockIdx.x * NT;
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

  const int row = min(r, p.m - 1);  // those behind the last are not stored

  // a block of 128 channels of the matrices and of x
  struct Block {
    u32x4 w[MATS][NT];
    f16x2 sb[MATS][NT][GROUPS];
    Piece<T, HOW> x[4];
  };
  auto fetch = [&](int c, Block& to) {
#pragma unroll
    for (int a = 0; a < MATS; ++a)
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const W4Arg& of = a ? p.gate : p.w;
        const int64_t at = (int64_t)min(tile0 + i, p.tiles - 1) * p.blocks + c;
        to.w[a][i] = *(const u32x4*)(of.words + at * 1024 + lane * 16);
        const uint8_t* const pairs = of.pairs + at * (64 * GROUPS) + r * (4 * GROUPS);
        load_pairs<GROUPS>(pairs, to.sb[a][i]);
      }
    const T* const x = (const T*)p.x + row * p.xs;
#pragma unroll
    for (int j = 0; j < 4; ++j) to.x[j].fetch(x, 128 * c + 32 * j + 8 * g, p.k);
  };

  f32x4 y[MATS][NT] = {};
  auto multiply = [&](int c, Block& in) {
    const bool end = 128 * c + 128 > p.k;
#pragma unroll
    for (int j = 0; j < 4; ++j) in.x[j].settle(128 * c + 32 * j + 8 * g, p.k, end);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      f32x4 part[MATS][NT] = {}, all = {};
#pragma unroll
      for (int j = i * STEPS; j < (i + 1) * STEPS; ++j) {
        u32x4 x[P];
        in.x[j].parts(x);
#pragma unroll
        for (int k = 0; k < P; ++k) all = mfma(x[k], ones, all);
#pragma unroll
        for (int a = 0; a < MATS; ++a)
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const u32x4 l = Rows<T>::levels(in.w[a][u][j]);
#pragma unroll
            for (int k = 0; k < P; ++k) part[a][u] = mfma(x[k], l, part[a][u]);
          }
      }
#pragma unroll
      for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int u = 0; u < NT; ++u) add_group<T>(in.sb[a][u][i], part[a][u], all, y[a][u]);
    }
  };
  // The next block is on its way while one is multiplied.  The last one is loaded
  // twice rather than not: behind a branch that may have loads or not, the compiler
  // waits for all of them.
  Block one, two;
  const int last = p.blocks - 1;
  int c = wave;
  fetch(min(c, last), one);
  while (c <= last) {
    fetch(min(c + p.waves, last), two);
    multiply(c, one);
    c += p.waves;
    if (c > last) break;
    fetch(min(c + p.waves, last), one);
    multiply(c, two);
    c += p.waves;
  }
#pragma unroll
  for (int a = 0; a < MATS; ++a)
#pragma unroll
    for (int u = 0; u < NT; ++u) *(f32x4*)(sums + (((wave * MATS + a) * NT + u) * 64 + lane) * 4) = y[a][u];
  __syncthreads();
  for (int at = threadIdx.x; at < NT * 256; at += blockDim.x) {
    const int n = at & 15, m = (at >> 4) & 15, u = at >> 8, col = 16 * (tile0 + u) + n;
    if (m >= p.m || col >= p.n) continue;
    const int from = u * 256 + (16 * (m >> 2) + n) * 4 + (m & 3);
    float v[MATS];
#pragma unroll
    for (int a = 0; a < MATS; ++a) {
      v[a] = 0.0f;
      for (int i = 0; i < p.waves; ++i) v[a] += sums[(i * MATS + a) * (NT * 256) + from];
    }
    finish<T>(p, m, col, v[0], GATE ? v[MATS - 1] : 0.0f, GATE);
  }
}

template <typename T, int G, int NT, bool GATE>
hipError_t launch(const W4Params& p, hipStream_t s) {
  const dim3 grid((p.tiles + NT - 1) / NT), block(64 * p.waves);
  const int lds = p.waves * (GATE ? 2 : 1) * NT * 1024;
  if (p.k < 8) hipLaunchKernelGGL((w4_few_kernel<T, G, NT, GATE, kOneByOne>), grid, block, lds, s, p);
  else if (!by_words<T>(p)) hipLaunchKernelGGL((w4_few_kernel<T, G, NT, GATE, kAtOnce>), grid, block, lds, s, p);
  else if constexpr (sizeof(T) == 2)
    hipLaunchKernelGGL((w4_few_kernel<T, G, NT, GATE, kByWords>), grid, block, lds, s, p);
  return hipGetLastError();
}
template <typename T, int G, bool GATE>
hipError_t launch_rows(const W4Params& p, hipStream_t s) {
  if constexpr (!GATE)
    if (p.wide) return launch<T, G, 2, GATE>(p, s);
  return launch<T, G, 1, GATE>(p, s);
}
template <typename T>
hipError_t launch_group(const W4Params& p, hipStream_t s) {
  switch (p.group) {
    case 32: return p.gate.words ? launch_rows<T, 32, true>(p, s) : launch_rows<T, 32, false>(p, s);
    case 64: return p.gate.words ? launch_rows<T, 64, true>(p, s) : launch_rows<T, 64, false>(p, s);
    default: return p.gate.words ? launch_rows<T, 128, true>(p, s) : launch_rows<T, 128, false>(p, s);
  }
}

}  // namespace

hipError_t launch_w4_few(const W4Params& p, int dtype, hipStream_t s) {
  return dtype == DT_BF16 ? launch_group<uint16_t>(p, s) : launch_group<float>(p, s);
}

}  // namespace fluid
