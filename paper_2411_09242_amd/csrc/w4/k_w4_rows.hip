// Many rows times a matrix in 4 bits, on the bf16 matrix cores (16x16x32).
//
// A workgroup has 128 rows of the matrix (and of the gate), 16 to a wavefront,
// and 32 or 64 rows of x, whose blocks of 128 channels it brings to LDS once for all
// its wavefronts, as operands: two blocks in turn, the loads another one ahead.
// Where that are too few workgroups, runs of channels go to workgroups of their own,
// whose sums a second launch adds in order.
//
// 64 rows times 4096 x 11008: 23 us, 4 of them the second launch; 32 fp32 rows 25.6 us
// (x in pieces of 64 bytes of a row, not 256: 26.2; 4096 x 4096 15.5 and 16.4).  Vector
// instructions (levels, and sums times s and b), the words' first loads and the sums'
// way to memory are most of it.
#include "launch_w4.h"
#include "w4_tile.h"

namespace fluid {

namespace {

constexpr int kWaves = 8;

// MT: tiles of 16 rows of x.
template <typename T, int G, int MT, bool GATE, Load HOW>
__global__ __launch_bounds__(64 * kWaves) void w4_rows_kernel(W4Params p) {
  constexpr int MATS = GATE ? 2 : 1, GROUPS = 128 / G, STEPS = G / 32, P = Rows<T>::N;
  constexpr int PIECES = MT * 4 / kWaves;  // of x, of a thread
  static_assert(PIECES * kWaves == MT * 4, "whole pieces");
  // [step][tile][part][16 g + (r ^ piece)], a piece being 4 step + g: what is written, 16
  // pieces of a row, and what is read, one of 16 rows, both meet all banks
  __shared__ u32x4 sx[2][4 * MT * P * 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  const int tile = blockIdx.x * kWaves + wave, m0 = blockIdx.z * (16 * MT);
  const int first = blockIdx.y * p.run, past = min(first + p.run, p.blocks);
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

  struct Words {
    u32x4 w[MATS];
    f16x2 sb[MATS][GROUPS];
  };
  auto fetch_words = [&](int c, Words& to) {
#pragma unroll
    for (int a = 0; a < MATS; ++a) {
      const W4Arg& of = a ? p.gate : p.w;
      const int64_t at = (int64_t)min(tile, p.tiles - 1) * p.blocks + c;
      to.w[a] = *(const u32x4*)(of.words + at * 1024 + lane * 16);
      load_pairs<GROUPS>(of.pairs + at * (64 * GROUPS) + r * (4 * GROUPS), to.sb[a]);
    }
  };
  typedef Piece<T, HOW> X;
  // a thread's pieces: eight channels each, a wavefront's 256 bytes of each of the four
  // rows from 4 (wave + kWaves i) on
  const int ch = 8 * r;
  auto fetch_x = [&](int c, X to[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      // rows behind the last are not stored, channels behind the last dropped below
      const int row = min(m0 + 4 * (wave + kWaves * i) + g, p.m - 1);
      to[i].fetch((const T*)p.x + row * p.xs, 128 * c + ch, p.k);
    }
  };
  auto put = [&](int c, X from[PIECES], u32x4* to) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int u = wave + kWaves * i;
      from[i].settle(128 * c + ch, p.k, 128 * c + 128 > p.k);
      u32x4 part[P];
      from[i].parts(part);
#pragma unroll
      for (int k = 0; k < P; ++k)
        to[((r / 4 * MT + u / 4) * P + k) * 64 + 16 * (r % 4) + ((4 * (u % 4) + g) ^ r)] = part[k];
    }
  };

  f32x4 y[MATS][MT] = {};
  auto multiply = [&](const Words& in, const u32x4* x) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      f32x4 part[MATS][MT] = {}, all[MT] = {};
#pragma unroll
      for (int j = i * STEPS; j < (i + 1) * STEPS; ++j) {
        u32x4 l[MATS];
#pragma unroll
        for (int a = 0; a < MATS; ++a) l[a] = Rows<T>::levels(in.w[a][j]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int k = 0; k < P; ++k) {
            const u32x4 of = x[((j * MT + t) * P + k) * 64 + 16 * g + (r ^ (4 * j + g))];
            all[t] = mfma(of, ones, all[t]);
#pragma unroll
            for (int a = 0; a < MATS; ++a) part[a][t] = mfma(of, l[a], part[a][t]);
          }
      }
#pragma unroll
      for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int t = 0; t < MT; ++t) add_group<T>(in.sb[a][i], part[a][t], all[t], y[a][t]);
    }
  };

  // Words are on their way four blocks ahead, x three: two in registers, one in LDS.
  // The last block is loaded again rather than nothing: behind a branch that may
  // have loads or not, the compiler waits for all of them.
  Words words[4];
  X xr[2][PIECES];
  const int last = past - 1;
  fetch_x(first, xr[0]);
#pragma unroll
  for (int i = 0; i < 4; ++i) fetch_words(min(first + i, last), words[i]);
  fetch_x(min(first + 1, last), xr[1]);
  put(first, xr[0], sx[0]);
  fetch_x(min(first + 2, last), xr[0]);
  lds_barrier();
  for (int c = first; c < past; c += 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (c + i >= past) break;
      put(min(c + i + 1, last), xr[(i + 1) % 2], sx[(i + 1) % 2]);
      fetch_x(min(c + i + 3, last), xr[(i + 1) % 2]);
      multiply(words[i], sx[i % 2]);
      fetch_words(min(c + i + 4, last), words[i]);
      lds_barrier();
    }
  }

  const int col = 16 * tile + r;
  if (col >= p.n) return;
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int m = m0 + 16 * t + 4 * g + e;
      if (m >= p.m) continue;
      if (p.splits == 1) {
        finish<T>(p, m, col, y[0][t][e], y[MATS - 1][t][e], GATE);
      } else {
#pragma unroll
        for (int a = 0; a < MATS; ++a)
          p.ws[((int64_t)(blockIdx.y * MATS + a) * p.m + m) * p.n + col] = y[a][t][e];
      }
    }
}

// The sums of all runs of channels, in order.
template <typename T, bool GATE>
__global__ __launch_bounds__(256) void w4_join_kernel(W4Params p) {
  constexpr int MATS = GATE ? 2 : 1;
  const int col = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
  if (col >= p.n) return;
  float v[MATS] = {};
  for (int i = 0; i < p.splits; ++i)
#pragma unroll
    for (int a = 0; a < MATS; ++a) v[a] += p.ws[((int64_t)(i * MATS + a) * p.m + m) * p.n + col];
  finish<T>(p, m, col, v[0], v[MATS - 1], GATE);
}

template <typename T, int G, int MT, bool GATE>
hipError_t launch(const W4Params& p, hipStream_t s) {
  const dim3 grid((p.tiles + kWaves - 1) / kWaves, p.splits, (p.m + 16 * MT - 1) / (16 * MT)), block(64 * kWaves);
  if (p.k < 8) hipLaunchKernelGGL((w4_rows_kernel<T, G, MT, GATE, kOneByOne>), grid, block, 0, s, p);
  else if (!by_words<T>(p)) hipLaunchKernelGGL((w4_rows_kernel<T, G, MT, GATE, kAtOnce>), grid, block, 0, s, p);
  else if constexpr (sizeof(T) == 2)
    hipLaunchKernelGGL((w4_rows_kernel<T, G, MT, GATE, kByWords>), grid, block, 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL((w4_join_kernel<T, GATE>), dim3((p.n + 255) / 256, p.m), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int G>
hipError_t launch_rows(const W4Params& p, hipStream_t s) {
  const bool gate = p.gate.words != nullptr;
  if constexpr (sizeof(T) == 4)
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

hipError_t launch_w4_rows(const W4Params& p, int dtype, hipStream_t s) {
  return dtype == DT_BF16 ? launch_group<uint16_t>(p, s) : launch_group<float>(p, s);
}

}  // namespace fluid
