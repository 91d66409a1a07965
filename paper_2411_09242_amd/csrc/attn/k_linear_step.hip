// Linear attention token after token: the state in registers, fp32 throughout.
//
// A workgroup has 32 columns (channels of the values) of one kv head's state,
// which need nothing of the others: a thread four of them, of every 32nd row
// (channel of the keys).  Bound by memory, the state read and written once: a token
// of 2048 heads of 128, 270 MB, in 52 us (5.2 TB/s, part of it from the last-level
// cache).  A token of 32 heads takes 3.8 us: the launch and a few dependent loads.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void linear_step_kernel(LinearParams p) {
  constexpr int R = D / 32;  // rows of a thread: 32 i + its own
  __shared__ f32x4 part[2][4][8];
  const int tid = threadIdx.x, col = tid & 7, row = tid >> 3, wave = tid >> 6;
  const int x = blockIdx.x / (D / 32), c0 = (blockIdx.x % (D / 32)) * 32 + 4 * col;
  const int b = (int)fdiv(x, p.div_heads), h = x - b * p.kv_heads;
  const int n = clamp_len(p.count, b, p.tokens);
  const int64_t at = (int64_t)x * D * D + c0;
  f32x4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = p.state ? *(const f32x4*)(p.state + at + (32 * i + row) * D) : f32x4{};
  const T* const k = (const T*)p.k.p + b * p.k.sb + h * p.k.sh;
  const T* const v = (const T*)p.v.p + b * p.v.sb + h * p.v.sh;
  const float* const g = p.decay + b * p.gb + h * p.gh;
  int turn = 0;
  for (int t = 0; t < n; ++t) {
    const float gt = g[t * p.gt], keep = expf(gt < -200.0f ? -200.0f : gt);
    f32x4 vt;
#pragma unroll
    for (int e = 0; e < 4; ++e) vt[e] = Elem<T>::load(v, t * p.v.st + c0 + e);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float kt = Elem<T>::load(k, t * p.k.st + 32 * i + row);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = __builtin_fmaf(keep, s[i][e], kt * vt[e]);
    }
    for (int j = 0; j < p.group; ++j) {
      const int64_t head = (int64_t)h * p.group + j;
      const T* const q = (const T*)p.q.p + b * p.q.sb + t * p.q.st + head * p.q.sh;
      f32x4 o = {};
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float qt = Elem<T>::load(q, 32 * i + row);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(qt, s[i][e], o[e]);
      }
#pragma unroll
      for (int m = 8; m < 64; m <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m);
      // two places in turn: one is read while the next is written
      if ((tid & 63) < 8) part[turn][wave][col] = o;
      __syncthreads();
      if (tid < 32) {
        const float* const w = (const float*)part[turn] + tid;
        const float sum = (w[0] + w[32]) + (w[64] + w[96]);
        Elem<T>::store((T*)p.o.p + b * p.o.sb + t * p.o.st + head * p.o.sh, c0 - 4 * col + tid, p.scale * sum);
      }
      turn ^= 1;
    }
  }
  if (!p.state_out) return;
#pragma unroll
  for (int i = 0; i < R; ++i) *(f32x4*)(p.state_out + at + (32 * i + row) * D) = s[i];
}

template <typename T, int D>
hipError_t launch(const LinearParams& p, hipStream_t s) {
  const uint32_t groups = (uint32_t)((int64_t)p.batch * p.kv_heads * (D / 32));
  hipLaunchKernelGGL((linear_step_kernel<T, D>), dim3(groups), dim3(256), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_dim(const LinearParams& p, int D, hipStream_t s) {
  switch (D) {
    case 32: return launch<T, 32>(p, s);
    case 64: return launch<T, 64>(p, s);
    default: return launch<T, 128>(p, s);
  }
}

}  // namespace

hipError_t launch_linear_step(const LinearParams& p, int dtype, int head_dim, hipStream_t s) {
  return dtype == DT_BF16 ? launch_dim<uint16_t>(p, head_dim, s) : launch_dim<float>(p, head_dim, s);
}

}  // namespace fluid
