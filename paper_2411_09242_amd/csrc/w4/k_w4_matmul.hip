// Up to 32 rows (fp32: 16) times a matrix in 4 bits, on the bf16 matrix cores (16x16x32).
//
// A workgroup has 16 or 32 rows of the matrix (and of the gate), whose blocks of
// 128 channels its wavefronts take in turn, one ahead of the products (words four
// ahead: 1 to 3 us slower); their sums are added through LDS in the order of the
// wavefronts.
//
// Bound by memory where the matrix is large: one row times 4096 x 11008 (24 MB) 7.2 us,
// the gated product with two of 11008 x 4096 (48 MB) 10.5 us (4.6 TB/s).  Every
// workgroup reads x from L2, 256 bytes of a row at once: 16 rows times 4096 x 11008 take
// 9.6 us (15.3 in the pieces of 64 bytes that operands are), 32 rows 14.4, where that
// is half the time.  Small ones are the launch and two rounds of loads, 4.5 to 5.1 us.
#include "launch_w4.h"
#include "w4_tile.h"

namespace fluid {

namespace {

// 16 bytes of LDS of a wavefront: of x, and then of its sums
constexpr int area_of(int loads, int planes, int tiles) {
  const int x = 64 * planes * (loads < 4 ? loads : 4), sums = 64 * tiles * (loads > 4 ? loads / 4 : 1);
  return x > sums ? x : sums;
}

// What a wavefront's lanes put into LDS before is what they read behind it.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// NT: tiles of 16 rows of the matrix.  XL: loads of x for a block, of four rows each.
// With eight, sixteen wavefronts would spill (32 rows times 4096 x 11008 18.6 us).
template <typename T, int G, int NT, int XL, bool GATE, Load HOW>
__global__ __launch_bounds__(GATE || NT == 2 || XL == 8 || sizeof(T) == 4 ? 512 : 1024) void w4_few_kernel(W4Params p) {
  constexpr int MATS = GATE ? 2 : 1, GROUPS = 128 / G, STEPS = G / 32, P = Rows<T>::N;
  constexpr int MT = XL > 4 ? XL / 4 : 1, TL = XL / MT;  // tiles of 16 rows of x, loads of one
  constexpr int AREA = area_of(XL, Rows<T>::PLANES, MATS * NT);
  extern __shared__ u32x4 shared[];  // [wavefront][AREA]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int tile0 = blockIdx.x * NT;
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

  // A wavefront's own piece of LDS turns x as it is loaded, 256 bytes of each of four
  // rows, into operands, 64 bytes of 16 rows.  Both meet all banks.
  u32x4* const area = shared + wave * AREA;
  auto place = [](int row, int piece) { return 16 * row + (piece ^ row); };

  // a block of 128 channels of the matrices and of x
  struct Block {
    u32x4 w[MATS][NT];
    f16x2 sb[MATS][NT][GROUPS];
    Piece<T, HOW> x[XL];
  };
  const int ch = 8 * r;
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
    // rows behind the last are not stored
#pragma unroll
    for (int j = 0; j < XL; ++j)
      to.x[j].fetch((const T*)p.x + min(4 * j + g, p.m - 1) * p.xs, 128 * c + ch, p.k);
  };

  f32x4 y[MATS][NT][MT] = {};
  auto multiply = [&](int c, Block& in) {
    const bool end = 128 * c + 128 > p.k;
    Rows<T> x[MT][4];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
      for (int j = 0; j < TL; ++j) {
        Piece<T, HOW>& piece = in.x[t * TL + j];
        piece.settle(128 * c + ch, p.k, end);
        piece.put(area + place(4 * j + g, r), 64 * TL);
      }
      wave_order();
#pragma unroll
      for (int j = 0; j < 4; ++j) x[t][j].get(area + place(r % (4 * TL), 4 * j + g), 64 * TL);
      wave_order();
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      f32x4 part[MATS][NT][MT] = {}, all[MT] = {};
#pragma unroll
      for (int j = i * STEPS; j < (i + 1) * STEPS; ++j) {
        u32x4 of[MT][P];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          x[t][j].parts(of[t]);
#pragma unroll
          for (int k = 0; k < P; ++k) all[t] = mfma(of[t][k], ones, all[t]);
        }
#pragma unroll
        for (int a = 0; a < MATS; ++a)
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const u32x4 l = Rows<T>::levels(in.w[a][u][j]);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
              for (int k = 0; k < P; ++k) part[a][u][t] = mfma(of[t][k], l, part[a][u][t]);
          }
      }
#pragma unroll
      for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int t = 0; t < MT; ++t) add_group<T>(in.sb[a][u][i], part[a][u][t], all[t], y[a][u][t]);
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
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t) ((f32x4*)area)[((a * NT + u) * MT + t) * 64 + lane] = y[a][u][t];
  __syncthreads();
  const float* const sums = (const float*)shared;
  for (int at = threadIdx.x; at < MT * NT * 256; at += blockDim.x) {
    const int u = at / (MT * 256), m = at / 16 % (16 * MT), col = 16 * (tile0 + u) + at % 16;
    if (m >= p.m || col >= p.n) continue;
    const int from = (u * MT + m / 16) * 256 + (16 * (m % 16 >> 2) + at % 16) * 4 + (m & 3);
    float v[MATS];
#pragma unroll
    for (int a = 0; a < MATS; ++a) {
      v[a] = 0.0f;
      for (int i = 0; i < p.waves; ++i) v[a] += sums[i * (4 * AREA) + a * (NT * MT * 256) + from];
    }
    finish<T>(p, m, col, v[0], GATE ? v[MATS - 1] : 0.0f, GATE);
  }
}

template <typename T, int G, int NT, int XL, bool GATE>
hipError_t launch(const W4Params& p, hipStream_t s) {
  const dim3 grid((p.tiles + NT - 1) / NT), block(64 * p.waves);
  const int lds = p.waves * area_of(XL, Rows<T>::PLANES, (GATE ? 2 : 1) * NT) * 16;
  if (p.k < 8) hipLaunchKernelGGL((w4_few_kernel<T, G, NT, XL, GATE, kOneByOne>), grid, block, lds, s, p);
  else if (!by_words<T>(p)) hipLaunchKernelGGL((w4_few_kernel<T, G, NT, XL, GATE, kAtOnce>), grid, block, lds, s, p);
  else if constexpr (sizeof(T) == 2)
    hipLaunchKernelGGL((w4_few_kernel<T, G, NT, XL, GATE, kByWords>), grid, block, lds, s, p);
  return hipGetLastError();
}
template <typename T, int G, int NT, bool GATE>
hipError_t launch_few(const W4Params& p, hipStream_t s) {
  if (p.m <= 4) return launch<T, G, NT, 1, GATE>(p, s);
  if constexpr (sizeof(T) == 2)
    if (p.m > 16) return launch<T, G, NT, 8, GATE>(p, s);
  return launch<T, G, NT, 4, GATE>(p, s);
}
template <typename T, int G, bool GATE>
hipError_t launch_rows(const W4Params& p, hipStream_t s) {
  if constexpr (!GATE)
    if (p.wide) return launch_few<T, G, 2, GATE>(p, s);
  return launch_few<T, G, 1, GATE>(p, s);
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
