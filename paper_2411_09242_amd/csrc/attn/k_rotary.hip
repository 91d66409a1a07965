// Rotary positions: pairs of channels turned by position times frequency.
//
// A position times a pair's turns a token, both integers, is the angle modulo
// whole turns in units of 2^-64 turn: far positions cost no precision and no
// reduction.  The nearest quarter turn is its upper bits; sine and cosine of the
// rest, at most an eighth of a turn, are the sums of their power series up to
// x^9 and x^10, within 2^-28 of themselves.
//
// A thread has a few neighbouring pairs of one token, and their angles once for
// some of its heads.  Bound by memory, every value read and written once: 8192
// tokens of 40 heads of 128 in bf16, 168 MB, in 35 us (4.8 TB/s; a copy of 4 GiB has
// 4.7).  One token takes 3 us, the launch and two dependent loads.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

// Sine and cosine of an angle in units of 2^-64 turn.
__device__ __forceinline__ void sin_cos(uint64_t turn, float& s, float& c) {
  const uint32_t quarter = (uint32_t)((turn + (uint64_t(1) << 61)) >> 62);
  const int64_t rest = (int64_t)(turn - ((uint64_t)quarter << 62));
  // from the upper and lower half: small angles keep their precision
  const float x = __builtin_fmaf((float)(int32_t)(rest >> 32), 6.283185307179586f * 0x1p-32f,
                                 (float)(uint32_t)rest * (6.283185307179586f * 0x1p-64f));
  const float z = x * x;
  float a = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040);
  a = __builtin_fmaf(z, a, 1.0f / 120);
  a = __builtin_fmaf(z, a, -1.0f / 6);
  a = __builtin_fmaf(x * z, a, x);
  float b = __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320);
  b = __builtin_fmaf(z, b, -1.0f / 720);
  b = __builtin_fmaf(z, b, 1.0f / 24);
  b = __builtin_fmaf(z, b, -0.5f);
  b = __builtin_fmaf(z, b, 1.0f);
  const float u = quarter & 1 ? b : a, v = quarter & 1 ? a : b;
  s = quarter & 2 ? -u : u;
  c = (quarter + 1) & 2 ? -v : v;
}

// N neighbouring channels, loaded and stored at once.
template <typename T, int N>
struct Run {
  float x[N];
  typedef T bits __attribute__((ext_vector_type(N)));
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (N == 1) {
      x[0] = Elem<T>::load(p, 0);
    } else {
      const bits v = *(const bits*)p;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const T e = v[i];
        x[i] = Elem<T>::load(&e, 0);
      }
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (N == 1) {
      Elem<T>::store(p, 0, x[0]);
    } else if constexpr (sizeof(T) == 4) {
      bits v;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = x[i];
      *(bits*)p = v;
    } else {
      typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
      words v;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
      *(words*)p = v;
    }
  }
};

// N: channels at once
template <typename T, int N, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  constexpr int P = INTER && N > 1 ? N / 2 : N;  // pairs of a thread
  const uint32_t item = blockIdx.x * 256u + threadIdx.x;
  if (item >= p.items) return;
  const uint32_t a = fdiv(item, p.div_units), unit = item - a * p.units;
  const uint32_t row = fdiv(a, p.div_heads), first = a - row * p.head_threads;
  const uint32_t b = fdiv(row, p.div_tokens), t = row - b * p.tokens;
  if (p.count && (int)t >= p.count[b]) return;
  const int all = p.heads[0] + p.heads[1];
  const bool turned = unit < (uint32_t)p.pairs;
  const int pair = unit * P;
  float s[P], c[P];
  if (turned) {
    const int64_t at = p.positions ? (int64_t)p.positions[b * p.position_stride + t]
                                   : (int64_t)(p.start ? p.start[b] : 0) + t;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      sin_cos((uint64_t)at * p.turns[pair + i], s[i], c[i]);
      s[i] *= p.inverse ? -p.amplitude : p.amplitude;
      c[i] *= p.amplitude;
    }
  }
  for (int h = first; h < all; h += p.head_threads) {
    const bool second = h >= p.heads[0];
    const TokensArg &xa = p.x[second], &ya = p.y[second];
    const int at = second ? h - p.heads[0] : h;
    const T* const x = (const T*)xa.p + (b * xa.sb + t * xa.st + at * xa.sh);
    T* const y = (T*)ya.p + (b * ya.sb + t * ya.st + at * ya.sh);
    if (!turned) {
      const int ch = p.dim + (unit - p.pairs) * N;
      typedef T bits __attribute__((ext_vector_type(N)));
      *(bits*)(y + ch) = *(const bits*)(x + ch);
    } else if constexpr (INTER) {
      constexpr int C = 2 * P;
      float v[C], w[C];
      if constexpr (N > 1) {
        Run<T, N> r;
        r.load(x + 2 * pair);
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = r.x[i];
      } else {
        v[0] = Elem<T>::load(x, 2 * pair);
        v[1] = Elem<T>::load(x, 2 * pair + 1);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        w[2 * i] = v[2 * i] * c[i] - v[2 * i + 1] * s[i];
        w[2 * i + 1] = v[2 * i + 1] * c[i] + v[2 * i] * s[i];
      }
      if constexpr (N > 1) {
        Run<T, N> r;
#pragma unroll
        for (int i = 0; i < C; ++i) r.x[i] = w[i];
        r.store(y + 2 * pair);
      } else {
        Elem<T>::store(y, 2 * pair, w[0]);
        Elem<T>::store(y, 2 * pair + 1, w[1]);
      }
    } else {
      const int half = p.dim / 2;
      Run<T, N> u, v, uo, vo;
      u.load(x + pair);
      v.load(x + half + pair);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        uo.x[i] = u.x[i] * c[i] - v.x[i] * s[i];
        vo.x[i] = v.x[i] * c[i] + u.x[i] * s[i];
      }
      uo.store(y + pair);
      vo.store(y + half + pair);
    }
  }
}

template <typename T, int N>
hipError_t launch(const RotaryParams& p, hipStream_t s) {
  const dim3 grid((p.items + 255u) / 256u), block(256);
  if (p.interleaved) hipLaunchKernelGGL((rotary_kernel<T, N, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((rotary_kernel<T, N, false>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotaryParams& p, int dtype, hipStream_t s) {
  const bool bf16 = dtype == DT_BF16;
  switch (p.vec) {
    case 8: return launch<uint16_t, 8>(p, s);  // of two bytes
    case 4: return bf16 ? launch<uint16_t, 4>(p, s) : launch<float, 4>(p, s);
    case 2: return bf16 ? launch<uint16_t, 2>(p, s) : launch<float, 2>(p, s);
    default: return bf16 ? launch<uint16_t, 1>(p, s) : launch<float, 1>(p, s);
  }
}

}  // namespace fluid
