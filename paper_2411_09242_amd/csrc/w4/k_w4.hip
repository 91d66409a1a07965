// Matrices into 4 bits and back (format: fluid_w4.h).  Both run once a matrix.
#include "../attn/dev_attn.h"
#include "launch_w4.h"

namespace fluid {

namespace {

// A workgroup has a tile of 16 rows and 128 channels: thread 16 r + i the
// channels 8 i .. + 7 of row r, which are one word.
template <typename T>
__global__ __launch_bounds__(256) void w4_pack_kernel(W4Params p) {
  const int tid = threadIdx.x, r = tid >> 4, i = tid & 15, tile = blockIdx.x / p.blocks;
  const int row = 16 * tile + r, ch = 128 * (blockIdx.x - tile * p.blocks) + 8 * i;
  const T* const from = (const T*)p.x + row * p.xs + ch;
  float x[8], lo = INFINITY, hi = -INFINITY, odd = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool there = row < p.n && ch + e < p.k;
    x[e] = there ? Elem<T>::load(from, e) : 0.0f;
    odd = __builtin_fmaf(x[e], 0.0f, odd);  // NaN from an infinity or a NaN on
    x[e] = fminf(fmaxf(x[e], -kLimit), kLimit);
    if (there) lo = fminf(lo, x[e]), hi = fmaxf(hi, x[e]);
  }
  const int lanes = p.group / 8;
  for (int m = 1; m < lanes; m <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, m));
    hi = fmaxf(hi, __shfl_xor(hi, m));
    odd += __shfl_xor(odd, m);
  }
  _Float16 s = 0, b = 0;
  if (lo <= hi) {
    s = half_of((hi - lo) / 15.0f);
    b = half_of(lo - 16.0f * (float)s);
  }
  if (odd != odd) s = 0, b = (_Float16)__builtin_nanf("");
  const float sf = (float)s, bf = (float)b;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float n = rintf((x[e] - bf) / sf) - 16.0f;
    const uint32_t level = sf > 0.0f && row < p.n && ch + e < p.k ? (uint32_t)fminf(fmaxf(n, 0.0f), 15.0f) : 0;
    w |= level << (4 * ((e >> 1) + 4 * (e & 1)));
  }
  uint32_t* const words = (uint32_t*)p.w.words + (int64_t)blockIdx.x * 256;
  words[(16 * (i & 3) + r) * 4 + (i >> 2)] = w;
  if (i % lanes == 0) {
    uint32_t* const pairs = (uint32_t*)p.w.pairs + (int64_t)blockIdx.x * (16 * 16 / lanes);
    pairs[r * (16 / lanes) + i / lanes] =
        __builtin_bit_cast(uint16_t, s) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void w4_read_kernel(W4Params p) {
  const int tid = threadIdx.x, r = tid >> 4, i = tid & 15, tile = blockIdx.x / p.blocks;
  const int row = 16 * tile + r, ch = 128 * (blockIdx.x - tile * p.blocks) + 8 * i;
  if (row >= p.n) return;
  const int lanes = p.group / 8;
  const uint32_t w = ((const uint32_t*)p.w.words)[(int64_t)blockIdx.x * 256 + (16 * (i & 3) + r) * 4 + (i >> 2)];
  const f16x2 sb = __builtin_bit_cast(
      f16x2, ((const uint32_t*)p.w.pairs)[(int64_t)blockIdx.x * (256 / lanes) + r * (16 / lanes) + i / lanes]);
  T* const to = (T*)p.out + row * p.os + ch;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (ch + e < p.k) {
      const float level = 16.0f + (float)((w >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15);
      Elem<T>::store(to, e, __builtin_fmaf((float)sb[0], level, (float)sb[1]));
    }
}

}  // namespace

hipError_t launch_w4_pack(const W4Params& p, int dtype, hipStream_t s) {
  const dim3 grid((uint32_t)p.tiles * p.blocks), block(256);
  if (dtype == DT_BF16) hipLaunchKernelGGL(w4_pack_kernel<uint16_t>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(w4_pack_kernel<float>, grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_w4_read(const W4Params& p, int dtype, hipStream_t s) {
  const dim3 grid((uint32_t)p.tiles * p.blocks), block(256);
  if (dtype == DT_BF16) hipLaunchKernelGGL(w4_read_kernel<uint16_t>, grid, block, 0, s, p);
  else hipLaunchKernelGGL(w4_read_kernel<float>, grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace fluid
