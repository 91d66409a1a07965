// Joins the shares of rows whose tokens were split over workgroups: the
// running maxima and sums of a softmax rescaled to a common maximum, in the
// order of the shares.  A workgroup per row: D / 4 threads of four channels,
// the rest of it over the shares, all of whose loads are on their way before
// the first is used.  Bound by latency: two round trips to memory.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnParams p) {
  constexpr int C = D / 4, S = 256 / C, AHEAD = 8;  // channel threads, share threads, loads in flight
  __shared__ __attribute__((aligned(16))) float sh_o[S][D + 4];
  __shared__ float sh_sum[4], sh_top[4];
  const int t = threadIdx.x, R = p.row_tile;
  int x = blockIdx.x;
  const int per_head = p.q_tokens * p.group;
  const int row = x % per_head;
  x /= per_head;
  const int b = (int)fdiv(x, p.div_heads);
  Item it;
  it.sequence(p, b);
  it.h = x - b * p.kv_heads;
  if (row >= it.rows) return;
  const int rt = row / R, r = row - rt * R;
  Share sh;
  it.tile(p, rt);
  sh.item = it;
  sh.index = (b * p.kv_heads + it.h) * p.row_tiles + (p.row_tiles - 1 - rt);
  sh.split = 0;
  sh.steps(p);
  const int shares = sh.shares;
  if (shares <= 1) return;  // written by its one workgroup
  const int64_t step = (int64_t)R * (D + 2);
  const float* const from = sh.slot(p, D);
  auto part = [&](int s) { return from + s * step; };

  const int c = t % C, s0 = t / C;
  f32x4 ahead[AHEAD];
  float at[AHEAD];
  auto fetch = [&](int s) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i, s += S)
      if (s < shares) {
        ahead[i] = *(const f32x4*)(part(s) + 2 * R + r * D + 4 * c);
        at[i] = part(s)[r];
      }
  };
  fetch(s0);
  float top = kLow, sum = 0.0f;
  for (int s = t; s < shares; s += 256) {
    const float m = part(s)[r], l = part(s)[R + r], m1 = fmaxf(top, m);
    sum = sum * __builtin_amdgcn_exp2f(top - m1) + l * __builtin_amdgcn_exp2f(m - m1);
    top = m1;
  }
  const float mine = top;
  top = wave_max(top);
  if ((t & 63) == 0) sh_top[t >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sh_top[0], sh_top[1]), fmaxf(sh_top[2], sh_top[3]));
  sum = wave_sum(sum * __builtin_amdgcn_exp2f(mine - top));
  if ((t & 63) == 0) sh_sum[t >> 6] = sum;
  f32x4 o = {0, 0, 0, 0};
  for (int s = s0; s < shares; s += AHEAD * S) {
    if (s != s0) fetch(s);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (s + i * S < shares) o += ahead[i] * __builtin_amdgcn_exp2f(at[i] - top);
  }
  *(f32x4*)&sh_o[s0][4 * c] = o;
  __syncthreads();
  if (t >= D) return;
  const float all = (sh_sum[0] + sh_sum[1]) + (sh_sum[2] + sh_sum[3]);
  float v = 0.0f;
#pragma unroll
  for (int s = 0; s < S; ++s) v += sh_o[s][t];
  v = all == 0.0f ? 0.0f : v / all;
  const int i = (int)fdiv(row, p.div_group), hq = it.h * p.group + (row - i * p.group);
  Elem<T>::store(p.o.p, b * p.o.sb + i * p.o.st + hq * p.o.sh + t, v);
}

template <typename T>
hipError_t launch(const AttnParams& p, int D, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)p.batch * p.kv_heads * p.q_tokens * p.group)), block(256);
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
