// Joins the shares of rows whose tokens were split over workgroups: the
// running maxima and sums of a softmax rescaled to a common maximum, in the
// order of the shares.  A workgroup per row: D / 4 threads of four channels,
// the rest of it over the shares.  Bound by latency: a few kilobytes a row.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnParams p) {
  constexpr int C = D / 4, S = 256 / C;
  __shared__ float sh[S][D + 1];
  const int R = p.row_tile;
  int x = blockIdx.x;
  const int item = x / R, r = x - item * R;
  x = item / p.row_tiles;
  const int rt = item - x * p.row_tiles;
  const int h = x % p.kv_heads, b = x / p.kv_heads;
  const int n = clamp_len(p.kv_len, b, p.kv_tokens);
  const int rows = clamp_len(p.q_len, b, p.q_tokens) * p.group;
  const int r0 = rt * R, r1 = min(r0 + R, rows);
  if (r0 + r >= r1) return;
  const int p0 = n - rows / p.group;
  const TileRange range = tile_range(p, p0 + r0 / p.group, p0 + (r1 - 1) / p.group, n, p.token_tile);
  const int per = share_tiles(p, range), shares = (range.count + per - 1) / per;
  if (shares <= 1) return;  // written by its one workgroup
  const int64_t step = (int64_t)R * (D + 2);
  const float* from = p.ws + (int64_t)item * p.splits * step;
  float top = kLow;
  for (int s = 0; s < shares; ++s) top = fmaxf(top, from[s * step + r]);
  const int c = threadIdx.x % C, s0 = threadIdx.x / C;
  float sum = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  for (int s = s0; s < shares; s += S) {
    const float* f = from + s * step;
    const float a = __builtin_amdgcn_exp2f(f[r] - top);
    sum += a * f[R + r];
    o += *(const f32x4*)(f + 2 * R + r * D + 4 * c) * a;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sh[s0][4 * c + e] = o[e];
  if (c == 0) sh[s0][D] = sum;
  __syncthreads();
  if (threadIdx.x >= D) return;
  float t = 0.0f, all = 0.0f;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    t += sh[s][threadIdx.x];
    all += sh[s][D];
  }
  t = all == 0.0f ? 0.0f : t / all;
  const int i = (r0 + r) / p.group, hq = h * p.group + (r0 + r - i * p.group);
  Elem<T>::store(p.o.p, b * p.o.sb + i * p.o.st + hq * p.o.sh + threadIdx.x, t);
}

template <typename T>
hipError_t launch(const AttnParams& p, int D, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.row_tiles * p.row_tile)), block(256);
  switch (D) {
    case 32: hipLaunchKernelGGL((attention_join_kernel<T, 32>), grid, block, 0, s, p); break;
    case 64: hipLaunchKernelGGL((attention_join_kernel<T, 64>), grid, block, 0, s, p); break;
    default: hipLaunchKernelGGL((attention_join_kernel<T, 128>), grid, block, 0, s, p); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_join(const AttnParams& p, int dtype, int head_dim, hipStream_t s) {
  return dtype == DT_BF16 ? launch<uint16_t>(p, head_dim, s) : launch<float>(p, head_dim, s);
}

}  // namespace fluid
