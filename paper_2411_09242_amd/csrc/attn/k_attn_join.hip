// Joins the shares of rows whose tokens were split over workgroups: the
// running maxima and sums of a softmax rescaled to a common maximum, in the
// order of the shares.  All loads of a row's sums are on their way before the
// first is used.  Bound by latency, two round trips to memory (3 to 5 us); for
// many rows by reading the sums.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

// Row `row` of kv head x: its first share, and its place in it.
struct JoinRow {
  Share sh;
  int row, r;
  // false: nothing to join; x is the same for a wavefront, row need not be
  __device__ __forceinline__ bool find(const AttnParams& p, int x, int row_) {
    row = row_;
    Item& it = sh.item;
    const int b = (int)fdiv(x, p.div_heads);
    it.sequence(p, b);
    it.h = x - b * p.kv_heads;
    if (row >= it.rows) return false;
    const int rt = row / p.row_tile;
    r = row - rt * p.row_tile;
    it.tile(p, rt);
    sh.index = x * p.row_tiles + (p.row_tiles - 1 - rt);
    sh.split = 0;
    sh.steps(p);
    return sh.shares > 1;  // else written by its one workgroup
  }
  template <typename T>
  __device__ __forceinline__ T* out(const AttnParams& p) const {
    const int i = (int)fdiv(row, p.div_group), hq = sh.item.h * p.group + (row - i * p.group);
    return (T*)p.o.p + sh.item.b * p.o.sb + i * p.o.st + hq * p.o.sh;
  }
};

// Up to kJoinFew shares: D / 8 threads a row, of eight channels each, which
// need nothing from one another.  Two shares of 16384 rows of 128 channels
// take 12 us more than half the steps alone; a workgroup per row, 45.
constexpr int kJoinFew = 16;
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_join_few_kernel(AttnParams p) {
  constexpr int C = D / 8;
  const int R = p.row_tile, c = threadIdx.x % C;
  JoinRow w;
  if (!w.find(p, blockIdx.x, blockIdx.y * (256 / C) + threadIdx.x / C)) return;
  const float* const from = w.sh.slot(p, D);
  const int64_t step = (int64_t)R * (D + 2);
  f32x4 part[kJoinFew][2];
  float m[kJoinFew], l[kJoinFew];
#pragma unroll
  for (int s = 0; s < kJoinFew; ++s)
    if (s < w.sh.shares) {
      const float* const at = from + s * step;
      m[s] = at[w.r];
      l[s] = at[R + w.r];
      part[s][0] = *(const f32x4*)(at + 2 * R + w.r * D + 8 * c);
      part[s][1] = *(const f32x4*)(at + 2 * R + w.r * D + 8 * c + 4);
    }
  float top = m[0];
#pragma unroll
  for (int s = 1; s < kJoinFew; ++s)
    if (s < w.sh.shares) top = fmaxf(top, m[s]);
  float sum = 0.0f, o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < kJoinFew; ++s)
    if (s < w.sh.shares) {
      const float a = __builtin_amdgcn_exp2f(m[s] - top);
      sum += a * l[s];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += a * part[s][e >> 2][e & 3];
    }
  const float inv = 1.0f / sum;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = sum == 0.0f ? 0.0f : o[e] * inv;
  store8(w.out<T>(p) + 8 * c, p.o.vec, o);
}

// More of them: a workgroup a row, D / 4 threads of four channels, the rest of
// it over the shares.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnParams p) {
  constexpr int C = D / 4, S = 256 / C, AHEAD = 8;  // channel threads, share threads, loads in flight
  __shared__ __attribute__((aligned(16))) float sh_o[S][D + 4];
  __shared__ float sh_sum[4], sh_top[4];
  const int t = threadIdx.x, R = p.row_tile;
  JoinRow w;
  if (!w.find(p, blockIdx.x, blockIdx.y)) return;
  const Share& sh = w.sh;
  const int shares = sh.shares, r = w.r;
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
  Elem<T>::store(w.out<T>(p), t, v);
}

template <typename T, int D>
void launch_dim(const AttnParams& p, hipStream_t s) {
  constexpr int AT_ONCE = 256 / (D / 8);
  // rows are split where they are few: far fewer than a grid may have along y
  const uint32_t heads = p.batch * p.kv_heads, rows = p.q_tokens * p.group;
  if (p.splits <= kJoinFew)
    hipLaunchKernelGGL((attention_join_few_kernel<T, D>), dim3(heads, (rows + AT_ONCE - 1) / AT_ONCE), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((attention_join_kernel<T, D>), dim3(heads, rows), dim3(256), 0, s, p);
}

template <typename T>
hipError_t launch(const AttnParams& p, int D, hipStream_t s) {
  switch (D) {
    case 32: launch_dim<T, 32>(p, s); break;
    case 64: launch_dim<T, 64>(p, s); break;
    default: launch_dim<T, 128>(p, s); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_join(const AttnParams& p, int dtype, int head_dim, hipStream_t s) {
  return dtype == DT_BF16 ? launch<uint16_t>(p, head_dim, s) : launch<float>(p, head_dim, s);
}

}  // namespace fluid
