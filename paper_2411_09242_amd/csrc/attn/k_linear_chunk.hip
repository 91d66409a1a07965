// Linear attention, a chunk of C tokens at a time, on the matrix cores.
//
// With c_i the sum of the chunk's log decays up to token i, and S the state
// before the chunk,
//     o_i = scale (e^{c_i} S^T q_i + sum_{j <= i} e^{c_i - c_j} (q_i k_j) v_j)
//     S  <- e^{c_C} S + sum_j k_j (e^{c_C - c_j} v_j)^T.
// The sums c are fp64, so that a difference of two has the precision of its own
// size, and weights between tokens are never above what the decays between them
// make.
//
// A workgroup has one kv head's run of tokens.  Its wavefronts have 32 or 16
// columns (channels of the values) of S each, in the registers of the matrix
// cores' results; which rows of S a tile has is chosen so that these registers
// are the second operand of S^T q as they are, and likewise the products k_j q_i
// the first one of the sum over j.  They alone go through LDS: every wavefront
// makes those of some rows.
//
// Where there are too few heads to fill the GPU, runs of tokens go to workgroups of
// their own: a first launch makes what each run adds to a state, and the second
// one's workgroups fold those before their run, in order.
//
// bf16: S and the weighted products are two bf16 parts (cut off, and the rest
// rounded: 2^-16), v with its decay three (2^-24): S is as exact as with fp32
// products.  fp32: the fp32 matrix cores.
#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

__device__ __forceinline__ bool odd_value(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// Eight values as N operands whose sum they are, the first ones cut off so that
// what is left is exact.
template <int N>
__device__ __forceinline__ void split(f32x4 a, f32x4 b, u32x4 out[N]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x = i < 2 ? a[2 * i] : b[2 * i - 4], y = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (k == N - 1) {
        out[k][i] = pack_bf16(x, y);
      } else {
        const uint32_t xh = __float_as_uint(x) & 0xffff0000u, yh = __float_as_uint(y) & 0xffff0000u;
        out[k][i] = (xh >> 16) | yh;
        x -= __uint_as_float(xh);
        y -= __uint_as_float(yh);
      }
    }
  }
}

// Operands of 16 rows or columns, KS of what is summed over: lane 16 g + r has
// those of row r and places g.
template <typename T, int D>
struct Core;

template <int D>
struct Core<uint16_t, D> {
  static constexpr int C = 64, KS = 32, LD = D + 8;  // tokens of a chunk; a row's elements in LDS
  static constexpr int PS = 2, PP = 2, PV = 3;       // parts of S, of the weighted products, of v
  typedef u32x4 Frag;
  __device__ static __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  // channels 32 s + 8 g .. + 7 of token row
  __device__ static __forceinline__ Frag rows(const uint16_t* m, int row, int s, int g) {
    return *(const u32x4*)(m + row * LD + 32 * s + 8 * g);
  }
  // channels ch .. + 3 (and the other lanes' of their sixteen) of tokens
  // 32 ks + 4 g .. + 3 and 16 more, transposed: a lane gets its own channel's
  __device__ static __forceinline__ Frag tokens(uint16_t* m, int ks, int ch, int lane) {
    uint16_t* const at = m + (32 * ks + 4 * (lane >> 4) + ((lane & 15) >> 2)) * LD + ch;
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)at);
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(at + 16 * LD));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // column col0 + r
  __device__ static __forceinline__ Frag values(uint16_t* m, int ks, int col0, int lane) {
    return tokens(m, ks, col0 + 4 * (lane & 3), lane);
  }
  // the channels of tile t of S's rows: 32 (t / 2) + 8 (r / 4) + 4 (t % 2) + r % 4
  __device__ static __forceinline__ Frag keys(uint16_t* m, int ks, int t, int lane) {
    return tokens(m, ks, 32 * (t >> 1) + 8 * (lane & 3) + 4 * (t & 1), lane);
  }
  __device__ static __forceinline__ int channel(int t, int g) { return 32 * (t >> 1) + 8 * g + 4 * (t & 1); }
  template <int N>
  __device__ static __forceinline__ void parts(const f32x4* tiles, int step, Frag out[N]) {
    split<N>(tiles[0], tiles[step], out);
  }
  // the values of token places, times w of the first and last four places
  template <int N>
  __device__ static __forceinline__ void weigh(Frag v, f32x4 w0, f32x4 w1, Frag out[N]) {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      a[2 * i] = __uint_as_float(v[i] << 16) * w0[2 * i], a[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u) * w0[2 * i + 1];
      b[2 * i] = __uint_as_float(v[i + 2] << 16) * w1[2 * i];
      b[2 * i + 1] = __uint_as_float(v[i + 2] & 0xffff0000u) * w1[2 * i + 1];
    }
    split<N>(a, b, out);
  }
  __device__ static __forceinline__ Frag clean(Frag v) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] &= ((v[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((v[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
    return v;
  }
  __device__ static __forceinline__ float element(const Frag f[PP], int e) {
    float x = 0.0f;
#pragma unroll
    for (int k = 0; k < PP; ++k) x += __uint_as_float(e & 1 ? f[k][e >> 1] & 0xffff0000u : f[k][e >> 1] << 16);
    return x;
  }
};

template <int D>
struct Core<float, D> {
  static constexpr int C = 32, KS = 16, LD = D + 4;
  static constexpr int PS = 1, PP = 1, PV = 1;
  typedef f32x4 Frag;
  __device__ static __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  // channels 16 s + 4 g .. + 3 of token row
  __device__ static __forceinline__ Frag rows(const float* m, int row, int s, int g) {
    return *(const f32x4*)(m + row * LD + 16 * s + 4 * g);
  }
  // tokens 16 ks + 4 g .. + 3 of column col0 + r
  __device__ static __forceinline__ Frag values(const float* m, int ks, int col0, int lane) {
    const float* const at = m + (16 * ks + 4 * (lane >> 4)) * LD + col0 + (lane & 15);
    return f32x4{at[0], at[LD], at[2 * LD], at[3 * LD]};
  }
  __device__ static __forceinline__ Frag keys(const float* m, int ks, int t, int lane) { return values(m, ks, 16 * t, lane); }
  __device__ static __forceinline__ int channel(int t, int g) { return 16 * t + 4 * g; }
  template <int N>
  __device__ static __forceinline__ void parts(const f32x4* tiles, int, Frag out[N]) { out[0] = tiles[0]; }
  template <int N>
  __device__ static __forceinline__ void weigh(Frag v, f32x4 w0, f32x4, Frag out[N]) { out[0] = v * w0; }
  __device__ static __forceinline__ Frag clean(Frag v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = odd_value(v[i]) ? 0.0f : v[i];
    return v;
  }
  __device__ static __forceinline__ float element(const Frag f[PP], int e) { return f[0][e]; }
};

constexpr int linear_waves(int D) { return D == 32 ? 2 : 4; }

// STATES: the first of two launches, what runs add to a state.
template <typename T, int D, bool STATES>
__global__ __launch_bounds__(64 * linear_waves(D), 2) void linear_chunk_kernel(LinearParams p) {
  typedef Core<T, D> At;
  typedef typename At::Frag Frag;
  constexpr int NW = linear_waves(D), THREADS = 64 * NW, NT = D / 16 / NW, MT = D / 16;
  constexpr int C = At::C, KS = At::KS, LD = At::LD, IT = C / 16, TPK = KS / 16, STEPS = D / KS, KSTEPS = C / KS;
  __shared__ __attribute__((aligned(16))) T sk[C * LD], sv[C * LD], sq[STATES ? 8 : C * LD];
  __shared__ Frag sp[STATES ? 1 : IT * KSTEPS * At::PP * 64];
  __shared__ __attribute__((aligned(16))) double sum[C];      // c_i, in powers of two
  __shared__ __attribute__((aligned(16))) float from[C], to[C];  // 2^{c_i}, 2^{c_C - c_i}
  __shared__ float kept;                                       // 2^{c_C}

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  const int x = blockIdx.x, seg = blockIdx.y;
  const int b = (int)fdiv(x, p.div_heads), h = x - b * p.kv_heads;
  const int n = clamp_len(p.count, b, p.tokens);
  const int first = seg * p.run, past = min(first + p.run, n);
  const int col0 = wave * (16 * NT);
  float* const slots = p.ws + (int64_t)x * p.segments * (D * D);
  float* const decays = p.ws + (int64_t)gridDim.x * p.segments * (D * D) + (int64_t)x * p.segments;
  auto place = [&](int mt, int nt) { return (((wave * MT + mt) * NT + nt) * 64 + lane) * 4; };

  f32x4 S[MT][NT];
  auto given = [&](const float* state) {  // of the caller
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          S[mt][nt][e] = state ? state[(int64_t)x * D * D + (At::channel(mt, g) + e) * D + col0 + 16 * nt + r] : 0.0f;
  };
  auto keep_slot = [&](int i) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) *(f32x4*)(slots + (int64_t)i * (D * D) + place(mt, nt)) = S[mt][nt];
  };
  if (STATES) {
    // the last run's share is not needed: its place has the state to start from,
    // which may be overwritten by the second launch
    if (seg == p.segments - 1) {
      if (p.state) given(p.state), keep_slot(seg);
      return;
    }
    if (past <= first) return;
    given(nullptr);
  } else {
    if (past <= first && seg > 0) return;
    if (p.segments == 1) {
      given(p.state);
    } else {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          S[mt][nt] = p.state ? *(const f32x4*)(slots + (int64_t)(p.segments - 1) * (D * D) + place(mt, nt)) : f32x4{};
      for (int i = 0; i < seg; ++i) {
        const float a = decays[i];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            S[mt][nt] = S[mt][nt] * a + *(const f32x4*)(slots + (int64_t)i * (D * D) + place(mt, nt));
      }
    }
  }
  const bool last = past == n || p.segments == 1;  // its state is the last one

  const T* const k = (const T*)p.k.p + b * p.k.sb + h * p.k.sh;
  const T* const v = (const T*)p.v.p + b * p.v.sb + h * p.v.sh;
  const float* const decay = p.decay + b * p.gb + h * p.gh;
  // rows t0 .. of a tensor into LDS, zeros behind the last; whether one is no number
  auto stage = [&](const T* m, const TokensArg& a, int t0, int rows, T* s) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < C * D / 8 / THREADS; ++i) {
      const int at = tid + THREADS * i, t = at / (D / 8), c = at % (D / 8) * 8;
      Eight<T> e;
      float f[8] = {};
      if (t < rows) {
        e.load(m + (int64_t)(t0 + t) * a.st + c, a.vec);
        e.floats(f);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) odd |= odd_value(f[j]);
      store8(s + t * LD + c, true, f);
    }
    return odd;
  };
  double total = 0.0;  // of the run's log decays

  for (int t0 = first; t0 < past; t0 += C) {
    const int rows = min(C, past - t0);
    __syncthreads();  // the chunk before is done with LDS
    stage(k, p.k, t0, rows, sk);
    const bool odd = stage(v, p.v, t0, rows, sv);
    if (wave == 0) {
      double c = 0.0;
      if (lane < rows) {
        const float gt = decay[(int64_t)(t0 + lane) * p.gt];
        c = (gt < -200.0f ? -200.0 : (double)gt) * 1.4426950408889634;
      }
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const double o = __shfl_up(c, m);
        if (lane >= m) c += o;
      }
      const double all = __shfl(c, 63);
      total += all;
      if (lane < C) {
        sum[lane] = c;
        from[lane] = __builtin_amdgcn_exp2f((float)c);
        to[lane] = __builtin_amdgcn_exp2f((float)(all - c));
      }
      const float a = (float)exp2(all);  // every chunk's rounding stays in S
      if (lane == 0) kept = a;
    }
    const bool dirty = __syncthreads_or(odd);

    if constexpr (!STATES) {
      for (int j = 0; j < p.group; ++j) {
        const int64_t head = (int64_t)h * p.group + j;
        if (j) __syncthreads();  // the head before is done with sq and sp
        stage((const T*)p.q.p + b * p.q.sb + head * p.q.sh, p.q, t0, rows, sq);
        __syncthreads();
        // k_j q_i of the rows i of some tiles, token j in a lane's registers
        for (int it = wave; it < IT; it += NW) {
          Frag qf[STEPS];
#pragma unroll
          for (int s = 0; s < STEPS; ++s) qf[s] = At::rows(sq, 16 * it + r, s, g);
          const double ci = sum[16 * it + r];
#pragma unroll
          for (int ks = 0; ks < KSTEPS; ++ks) {
            if (ks * KS > 16 * it + 15) break;
            f32x4 w[TPK];
#pragma unroll
            for (int u = 0; u < TPK; ++u) {
              const int jt = ks * TPK + u;
              w[u] = f32x4{};
              if (jt > it) continue;
#pragma unroll
              for (int s = 0; s < STEPS; ++s) w[u] = At::mma(At::rows(sk, 16 * jt + r, s, g), qf[s], w[u]);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int tj = 16 * jt + 4 * g + e;
                const float f = __builtin_amdgcn_exp2f((float)(ci - sum[tj])) * w[u][e];
                w[u][e] = tj <= 16 * it + r ? f : 0.0f;
              }
            }
            Frag f[At::PP];
            At::template parts<At::PP>(w, 1, f);
#pragma unroll
            for (int k = 0; k < At::PP; ++k) sp[((it * KSTEPS + ks) * At::PP + k) * 64 + lane] = f[k];
          }
        }
        __syncthreads();
        f32x4 o[IT][NT] = {};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          Frag f[NT][At::PS];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) At::template parts<At::PS>(&S[s * TPK][nt], NT, f[nt]);
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            const Frag a = At::rows(sq, 16 * it + r, s, g);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int k = 0; k < At::PS; ++k) o[it][nt] = At::mma(a, f[nt][k], o[it][nt]);
          }
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const f32x4 e = *(const f32x4*)(from + 16 * it + 4 * g);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[it][nt] *= e;
        }
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
          Frag f[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) f[nt] = At::values(sv, ks, col0 + 16 * nt, lane);
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            if (16 * it + 15 < ks * KS) continue;
            // 0 times a later value that is no number would still be none: where a
            // row's tokens and later ones share a step, such values are left out
            // and added below
            const bool shared = 16 * it + 15 < (ks + 1) * KS;
            Frag a[At::PP];
#pragma unroll
            for (int k = 0; k < At::PP; ++k) a[k] = sp[((it * KSTEPS + ks) * At::PP + k) * 64 + lane];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int k = 0; k < At::PP; ++k)
                o[it][nt] = At::mma(a[k], shared && dirty ? At::clean(f[nt]) : f[nt], o[it][nt]);
          }
        }
        if (__builtin_expect(dirty, 0)) {
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            const int ks = 16 * it / KS;
#pragma nounroll
            for (int t = ks * KS; t < min((ks + 1) * KS, 16 * it + 16); ++t)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const float val = Elem<T>::load(sv, t * LD + col0 + 16 * nt + r);
                if (!odd_value(val)) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int i = 16 * it + 4 * g + e;
                  if (t > i) continue;
                  Frag a[At::PP];
#pragma unroll
                  for (int k = 0; k < At::PP; ++k)
                    a[k] = sp[((it * KSTEPS + ks) * At::PP + k) * 64 + 16 * ((t & 15) >> 2) + (i & 15)];
                  o[it][nt][e] += At::element(a, 4 * ((t % KS) >> 4) + (t & 3)) * val;
                }
              }
          }
        }
        T* const out = (T*)p.o.p + b * p.o.sb + head * p.o.sh;
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 16 * it + 4 * g + e;
            if (i >= rows) continue;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              Elem<T>::store(out + (int64_t)(t0 + i) * p.o.st, col0 + 16 * nt + r, p.scale * o[it][nt][e]);
          }
      }
      if (t0 + C >= past && !(last && p.state_out)) break;  // nobody reads this state
    }

    const float a = kept;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) S[mt][nt] *= a;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      Frag f[NT][At::PV];
      const f32x4 w0 = *(const f32x4*)(to + KS * ks + 4 * g), w1 = *(const f32x4*)(to + KS * ks + (KS - 16) + 4 * g);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) At::template weigh<At::PV>(At::values(sv, ks, col0 + 16 * nt, lane), w0, w1, f[nt]);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const Frag kt = At::keys(sk, ks, mt, lane);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < At::PV; ++i) S[mt][nt] = At::mma(kt, f[nt][i], S[mt][nt]);
      }
    }
  }
  if (STATES) {
    keep_slot(seg);
    if (tid == 0) decays[seg] = (float)exp2(total);
  } else if (last && p.state_out) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          p.state_out[(int64_t)x * D * D + (At::channel(mt, g) + e) * D + col0 + 16 * nt + r] = S[mt][nt][e];
  }
}

template <typename T, int D>
hipError_t launch(const LinearParams& p, hipStream_t s) {
  const dim3 grid((uint32_t)(p.batch * p.kv_heads), p.segments), block(64 * linear_waves(D));
  if (p.segments > 1) {
    hipLaunchKernelGGL((linear_chunk_kernel<T, D, true>), grid, block, 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((linear_chunk_kernel<T, D, false>), grid, block, 0, s, p);
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

hipError_t launch_linear_chunk(const LinearParams& p, int dtype, int head_dim, hipStream_t s) {
  return dtype == DT_BF16 ? launch_dim<uint16_t>(p, head_dim, s) : launch_dim<float>(p, head_dim, s);
}

}  // namespace fluid
