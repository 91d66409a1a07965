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
// A workgroup has one query head's run of tokens.  Its wavefronts have 16 columns
// (channels of the values) of S each, in the registers of the matrix cores'
// results; which rows of S a tile has is chosen so that these registers
// are an operand of S^T q as they are, and likewise the products k_j q_i one of
// the sum over j.  They alone go through LDS: every wavefront makes those of some
// rows.  The next chunk's tensors are on their way meanwhile.
//
// The query heads of a kv head make the same states: sharing them in a workgroup
// took a loop over the heads, registers that the compiler spilled, and longer
// runs.  Where there are too few heads to fill the GPU, runs of tokens go to
// workgroups of their own: a first launch makes what each run adds to a state, and
// the last one's workgroups fold those before their run, in order; where those
// are many, a launch between them makes each run's first state.
//
// 8192 tokens of 32 heads of 128, bf16, in 16 runs: 129 to 140 us by card, 39 of them
// for the runs' states.  Keys and values are read twice, 400 MB in all, 86 us at the
// rate of a copy.  A chunk takes 15200 cycles of a workgroup with another one beside it:
// products of keys and queries 22 %, S^T q 20 %, the sum over j 11 %, the state 19 %, LDS
// and its barriers 18 %, results and the next loads 10 %.  Of the outputs' 100 us matrix
// cores are busy for 24 and vector instructions for 35; what is left is the latency of
// LDS reads, one after another, since 128 registers leave no room for more of them at
// once.  512 heads of 1024 tokens, in one launch: 180 us (3.0 TB/s).  Measured with two
// parts of S and of the weighted products, at 128 us: 256 registers and one workgroup to
// a compute unit 140 us, in 8 runs 126; 24 and 32 runs 141 and 150; without the loads of
// later chunks ahead 345.
//
// bf16: S, the weighted products and v with its decay are three bf16 parts each (the
// first two cut off, the rest rounded: 2^-24), as exact as with fp32 products.  In
// two parts (2^-16) the rows of 8192 tokens were four times as far from the rounded
// exact ones, and took 121 us where they take 129 (130 and 140 on another card).
// fp32: the fp32 matrix cores.
#include <type_traits>

#include "dev_attn.h"
#include "launch_attn.h"

namespace fluid {

namespace {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
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
        out[k][i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);  // the upper halves
        x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
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
  static constexpr int C = 64, KS = 32, LD = D + 16;  // tokens of a chunk; a row's elements in LDS, 8 banks apart: 23 % of its cycles are conflicts (12: 42 %)
  static constexpr int PS = 3, PP = 3, PV = 3;       // parts of S, of the weighted products, of v
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
  // the largest size of a piece's values, as bits, in either half; whether one is no number
  __device__ static __forceinline__ uint32_t sizes(u32x4 v, uint32_t most) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu),
                                                                    __builtin_bit_cast(u16x2, most)));
    return most;
  }
  __device__ static __forceinline__ bool odd(uint32_t most) { return most >= 0x7f800000u || (most & 0xffffu) >= 0x7f80u; }
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
  __device__ static __forceinline__ uint32_t sizes(u32x4 v, uint32_t most) {
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, v[i] & 0x7fffffffu);
    return most;
  }
  __device__ static __forceinline__ bool odd(uint32_t most) { return most >= 0x7f800000u; }
};

// 2^c, with what fp32 cuts off of c: what a chunk keeps of a state enters it as
// often as there are chunks.  (exp2 of a double has some forty registers of
// constants, which the compiler held for the whole loop: 206 us instead of 160.)
__device__ __forceinline__ float power_of_two(double c) {
  const float hi = (float)c, e = __builtin_amdgcn_exp2f(hi);
  return __builtin_fmaf(e, (float)(c - hi) * 0.69314718f, e);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double add_dpp(double v) {
  const int64_t x = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return v + __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
// The sums up to each lane, and the last one's.
__device__ __forceinline__ double wave_scan(double v) {
  v = add_dpp<0x111, 0xf>(v);  // from the lane 1, 2, 4, 8 before it in its row of 16
  v = add_dpp<0x112, 0xf>(v);
  v = add_dpp<0x114, 0xf>(v);
  v = add_dpp<0x118, 0xf>(v);
  v = add_dpp<0x142, 0xa>(v);  // a row's last lane to the next row
  return add_dpp<0x143, 0xc>(v);  // lane 31 to the upper rows
}
__device__ __forceinline__ double last_lane(double v) {
  const int64_t x = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, 63), hi = __builtin_amdgcn_readlane((int)(x >> 32), 63);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}

constexpr int linear_waves(int D) { return D / 16; }

// STATES: the first of two launches, what runs add to a state.
// VEC: rows start on 16-byte addresses, and a chunk's lie within 32-bit offsets.
template <typename T, int D, bool STATES, bool VEC>
__global__ __launch_bounds__(64 * linear_waves(D)) __attribute__((amdgpu_waves_per_eu(4, 4))) void linear_chunk_kernel(
    LinearParams p) {
  typedef Core<T, D> At;
  typedef typename At::Frag Frag;
  constexpr int NW = linear_waves(D), THREADS = 64 * NW, MT = D / 16;
  constexpr int C = At::C, KS = At::KS, LD = At::LD, IT = C / 16, TPK = KS / 16, STEPS = D / KS, KSTEPS = C / KS;
  constexpr int E = 16 / sizeof(T), PIECES = C * D / E / THREADS;  // elements of 16 bytes; pieces of a thread
  // tiles of 16 rows i times steps of tokens j, those that some j <= i has: step
  // 0 of all, then step 1 of the later ones
  static_assert(KSTEPS == 2, "two steps to a chunk");
  constexpr int UNITS = 2 * IT - TPK;
  auto unit = [](int it, int ks) { return ks ? IT + it - TPK : it; };
  __shared__ __attribute__((aligned(16))) T sk[C * LD], sv[C * LD], sq[STATES ? 8 : C * LD];
  __shared__ Frag sp[STATES ? 1 : UNITS * At::PP * 64];
  // of this and the next chunk in turn: c_i in powers of two, scale 2^{c_i}, 2^{c_C - c_i}, 2^{c_C}
  __shared__ __attribute__((aligned(16))) double sum[2][C];
  __shared__ __attribute__((aligned(16))) float from[2][C], to[2][C];
  __shared__ float kept[2];
  __shared__ int odd_at;  // the latest chunk with a value that is no number

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  const int x = blockIdx.x, seg = blockIdx.y, j = blockIdx.z;  // kv head, run, query head of the group
  const int b = (int)fdiv(x, p.div_heads), h = x - b * p.kv_heads;
  const int n = clamp_len(p.count, b, p.tokens);
  const int first = seg * p.run, past = min(first + p.run, n);
  const int col0 = 16 * wave;
  float* const slots = p.ws + (int64_t)x * p.segments * (D * D);
  float* const decays = p.ws + (int64_t)gridDim.x * p.segments * (D * D) + (int64_t)x * p.segments;
  const int place = (wave * MT * 64 + lane) * 4;

  f32x4 S[MT];
  auto given = [&](const float* state) {  // by the caller
    const float* const at = state + (int64_t)x * D * D + At::channel(0, g) * D + col0 + r;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[mt][e] = state ? at[(At::channel(mt, 0) + e) * D] : 0.0f;
  };
  auto keep_slot = [&](int i) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) *(f32x4*)(slots + (int64_t)i * (D * D) + place + 256 * mt) = S[mt];
  };
  if (STATES) {
    // the last run's share is not needed: its place has the state to start from,
    // which may be overwritten by the second launch
    if (seg == p.segments - 1) {
      if (p.state) given(p.state), keep_slot(seg);
      return;
    }
    if (past <= first) return;
  } else {
    if (past <= first && seg > 0) return;
  }
  const bool last = j == 0 && past == n && p.state_out;  // its state is the last one

  const T* const k = (const T*)p.k.p + b * p.k.sb + h * p.k.sh;
  const T* const v = (const T*)p.v.p + b * p.v.sb + h * p.v.sh;
  const T* const q = (const T*)p.q.p + b * p.q.sb + ((int64_t)h * p.group + j) * p.q.sh;
  const float* const decay = p.decay + b * p.gb + h * p.gh;
  // a chunk of a tensor on its way to LDS; places behind the last token repeat it
  struct Stage {
    u32x4 piece[PIECES];
  };
  constexpr int ACROSS = D / E, ROWS = THREADS / ACROSS;  // pieces of a row; rows that the threads take at once
  const int row = tid / ACROSS, piece = tid % ACROSS * E;
  auto fetch = [&](const T* m, const TokensArg& a, int t0, Stage& to) {
    const T* const base = m + (int64_t)t0 * a.st;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int t = min(row + ROWS * i, past - 1 - t0);
      if constexpr (VEC) {
        to.piece[i] = *(const u32x4*)((const char*)base + (uint32_t)(t * (int)a.st + piece) * sizeof(T));
      } else {
        const T* const from = base + t * a.st + piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2) to.piece[i][e] = from[2 * e] | ((uint32_t)from[2 * e + 1] << 16);
          else to.piece[i][e] = __float_as_uint(from[e]);
        }
      }
    }
  };
  auto put = [&](const Stage& from, T* s) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) *(u32x4*)(s + (row + ROWS * i) * LD + piece) = from.piece[i];
  };
  // The results of a chunk, which lie where q did, to memory: whole rows, where a
  // wavefront's own columns would be 32 bytes of each.
  T* const out = (T*)p.o.p + b * p.o.sb + ((int64_t)h * p.group + j) * p.o.sh;
  auto take = [&](Stage& to) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) to.piece[i] = *(const u32x4*)(sq + (row + ROWS * i) * LD + piece);
  };
  auto give = [&](const Stage& from, int t0, int rows) {
    T* const base = out + (int64_t)t0 * p.o.st;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int t = row + ROWS * i;
      if (t >= rows) continue;
      if constexpr (VEC) {
        *(u32x4*)((char*)base + (uint32_t)(t * (int)p.o.st + piece) * sizeof(T)) = from.piece[i];
      } else {
        T* const to = base + t * p.o.st + piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2) to[2 * e] = (uint16_t)from.piece[i][e], to[2 * e + 1] = (uint16_t)(from.piece[i][e] >> 16);
          else to[e] = __uint_as_float(from.piece[i][e]);
        }
      }
    }
  };
  // The last wavefront makes the next chunk's weights from decays that it has
  // loaded a chunk before: the others would wait for them.
  double total = 0.0;  // of the run's log decays
  float ahead = 0.0f;
  auto fetch_decay = [&](int t0) {
    const float gt = decay[(int64_t)min(t0 + (lane & (C - 1)), past - 1) * p.gt];
    ahead = t0 + lane < past && lane < C ? gt : 0.0f;
  };
  auto weights = [&](int t0, int turn) {
    double c = wave_scan((ahead < -200.0f ? -200.0 : (double)ahead) * 1.4426950408889634);
    fetch_decay(t0 + C);
    const double all = last_lane(c);
    if (STATES) total += all;
    if (lane < C) {
      sum[turn][lane] = c;
      from[turn][lane] = p.scale * __builtin_amdgcn_exp2f((float)c);
      to[turn][lane] = __builtin_amdgcn_exp2f((float)(all - c));
    }
    const float a = power_of_two(all);
    if (lane == 0) kept[turn] = a;
  };

  Stage ks_, vs_, qs_;
  if (first < past) {
    if (wave == NW - 1) fetch_decay(first);  // ahead of what all workgroups ask for now
    fetch(k, p.k, first, ks_);
    fetch(v, p.v, first, vs_);
    if (!STATES) fetch(q, p.q, first, qs_);
    if (tid == 0) odd_at = -1;
  }
  if (STATES || !p.slots) {
    given(STATES ? nullptr : p.state);
  } else {
    // the state to start from and what the runs before leave of it, a slot ahead;
    // after the scan, this run's own
    f32x4 next[MT];
    auto load = [&](int i) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) next[mt] = *(const f32x4*)(slots + (int64_t)i * (D * D) + place + 256 * mt);
    };
    if (p.state || p.scan) load(p.scan ? seg : p.segments - 1);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) S[mt] = p.state || p.scan ? next[mt] : f32x4{};
    const int before = p.scan ? 0 : seg;
    if (before) load(0);
    for (int i = 0; i < before; ++i) {
      const float a = decays[i];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) S[mt] = S[mt] * a + next[mt];
      if (i + 1 < before) load(i + 1);
    }
  }
  if (first < past && wave == NW - 1) weights(first, 0);
  lds_barrier();
  // A chunk; the last one apart, so that the others have no branch with loads or
  // stores in it, behind which the compiler would wait for all of them.
  auto chunk = [&](int t0, int turn, auto last_one) {
    constexpr bool more = !decltype(last_one)::value;
    lds_barrier();  // the chunk before is done with LDS
    if (!more && past - t0 < C) {  // nothing from behind the last token enters the state
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (row + ROWS * i >= past - t0) vs_.piece[i] = u32x4{};
    }
    Stage done;
    if constexpr (!STATES) take(done);
    put(ks_, sk);
    put(vs_, sv);
    if constexpr (!STATES) {
      put(qs_, sq);
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) most = At::sizes(vs_.piece[i], most);
      if (At::odd(most)) odd_at = t0;
    }
    lds_barrier();
    if constexpr (!STATES) {
      if (t0 != first) give(done, t0 - C, C);
    }
    if constexpr (more) {
      fetch(k, p.k, t0 + C, ks_);
      fetch(v, p.v, t0 + C, vs_);
      if constexpr (!STATES) fetch(q, p.q, t0 + C, qs_);
    }
    if constexpr (STATES) {
      if (more && wave == NW - 1) weights(t0 + C, turn ^ 1);
    } else {
      const bool dirty = odd_at == t0;
      // k_j q_i with its decay: row i to a lane's r, tokens j in its registers
      for (int u = wave; u < UNITS; u += NW) {
        const int ks = u >= IT, it = ks ? u - IT + TPK : u;
        Frag qf[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) qf[s] = At::rows(sq, 16 * it + r, s, g);
        const double ci = sum[turn][16 * it + r];
        f32x4 w[TPK];
#pragma unroll
        for (int i = 0; i < TPK; ++i) {
          const int jt = ks * TPK + i;  // past `it` too: all masked
          w[i] = f32x4{};
#pragma unroll
          for (int s = 0; s < STEPS; ++s) w[i] = At::mma(At::rows(sk, 16 * jt + r, s, g), qf[s], w[i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tj = 16 * jt + 4 * g + e;
            const float f = __builtin_amdgcn_exp2f((float)(ci - sum[turn][tj])) * p.scale;
            w[i][e] = tj <= 16 * it + r ? f * w[i][e] : 0.0f;
          }
        }
        Frag f[At::PP];
        At::template parts<At::PP>(w, 1, f);
#pragma unroll
        for (int i = 0; i < At::PP; ++i) sp[(u * At::PP + i) * 64 + lane] = f[i];
      }
      if (more && wave == NW - 1) weights(t0 + C, turn ^ 1);
      lds_barrier();
      f32x4 o[IT] = {};  // channels col0 + 4 g .. + 3 of token 16 it + r
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        Frag f[At::PS];
        At::template parts<At::PS>(&S[s * TPK], 1, f);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const Frag a = At::rows(sq, 16 * it + r, s, g);
#pragma unroll
          for (int i = 0; i < At::PS; ++i) o[it] = At::mma(f[i], a, o[it]);
        }
      }
#pragma unroll
      for (int it = 0; it < IT; ++it) o[it] *= from[turn][16 * it + r];
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        // 0 times a later value that is no number would still be none: where a
        // row's tokens and later ones share a step, such values are left out and
        // added below
        const Frag f = At::values(sv, ks, col0, lane);
        Frag own = f;
        if (__builtin_expect(dirty, 0)) own = At::clean(f);
#pragma unroll
        for (int it = ks * TPK; it < IT; ++it)
#pragma unroll
          for (int i = 0; i < At::PP; ++i)
            o[it] = At::mma(it < (ks + 1) * TPK ? own : f, sp[(unit(it, ks) * At::PP + i) * 64 + lane], o[it]);
      }
      if (__builtin_expect(dirty, 0)) {
#pragma nounroll
        for (int t = 0; t < C; ++t) {
          float val[4];
          bool any = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) val[e] = Elem<T>::load(sv, t * LD + col0 + 4 * g + e), any |= odd_value(val[e]);
          if (!__any(any)) continue;
          // of part 0, row r, token t
          const int at = 16 / (int)sizeof(T) * (16 * ((t & 15) >> 2) + r) + 4 * (t % KS >> 4) + (t & 3);
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            if (it / TPK != t / KS) continue;
            float w = 0.0f;
#pragma unroll
            for (int i = 0; i < At::PP; ++i)
              w += Elem<T>::load(sp, (unit(it, it / TPK) * At::PP + i) * (1024 / (int)sizeof(T)) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (t <= 16 * it + r && odd_value(val[e])) o[it][e] += w * val[e];
          }
        }
      }
      lds_barrier();  // all are done with q: its place takes the result
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        T* const at = sq + (16 * it + r) * LD + col0 + 4 * g;
        if constexpr (sizeof(T) == 2) *(uint2*)at = make_uint2(pack_bf16(o[it][0], o[it][1]), pack_bf16(o[it][2], o[it][3]));
        else *(f32x4*)at = o[it];
      }
      if (!more && !last) return;  // nobody reads this state
    }

    const float a = kept[turn];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) S[mt] *= a;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      Frag f[At::PV];
      const f32x4 w0 = *(const f32x4*)(to[turn] + KS * ks + 4 * g), w1 = *(const f32x4*)(to[turn] + KS * ks + (KS - 16) + 4 * g);
      At::template weigh<At::PV>(At::values(sv, ks, col0, lane), w0, w1, f);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const Frag kt = At::keys(sk, ks, mt, lane);
#pragma unroll
        for (int i = 0; i < At::PV; ++i) S[mt] = At::mma(kt, f[i], S[mt]);
      }
    }
  };
  int t0 = first, turn = 0;
  for (; t0 + C < past; t0 += C, turn ^= 1) chunk(t0, turn, std::false_type());
  if (t0 < past) {
    chunk(t0, turn, std::true_type());
    if constexpr (!STATES) {
      Stage done;
      lds_barrier();
      take(done);
      give(done, t0, past - t0);
    }
  }
  if (STATES) {
    keep_slot(seg);
    if (tid == THREADS - 64) decays[seg] = power_of_two(total);
  } else if (last) {
    float* const at = p.state_out + (int64_t)x * D * D + At::channel(0, g) * D + col0 + r;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 4; ++e) at[(At::channel(mt, 0) + e) * D] = S[mt][e];
  }
}

// What runs add to a state into what each starts from, in place: a thread has four
// values of a head's state.
__global__ __launch_bounds__(256) void linear_scan_kernel(LinearParams p, int size) {
  constexpr int AHEAD = 8;
  const int x = blockIdx.y, at = (blockIdx.x * 256 + threadIdx.x) * 4;
  float* const slots = p.ws + (int64_t)x * p.segments * size + at;
  const float* const decays = p.ws + (int64_t)gridDim.y * p.segments * size + (int64_t)x * p.segments;
  const int last = p.segments - 1;
  f32x4 S = p.state ? *(const f32x4*)(slots + (int64_t)last * size) : f32x4{};
  for (int i = 0; i <= last; i += AHEAD) {
    f32x4 u[AHEAD];
    float a[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      u[j] = *(const f32x4*)(slots + (int64_t)min(i + j, last) * size);
      a[j] = decays[min(i + j, last)];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (i + j <= last) {
        *(f32x4*)(slots + (int64_t)(i + j) * size) = S;
        S = S * a[j] + u[j];
      }
  }
}

template <typename T, int D, bool VEC>
hipError_t launch(const LinearParams& p, hipStream_t s) {
  const uint32_t heads = p.batch * p.kv_heads;
  const dim3 block(64 * linear_waves(D));
  if (p.slots) {
    hipLaunchKernelGGL((linear_chunk_kernel<T, D, true, VEC>), dim3(heads, p.segments), block, 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.scan) {
      hipLaunchKernelGGL(linear_scan_kernel, dim3(D * D / 1024, heads), dim3(256), 0, s, p, D * D);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  hipLaunchKernelGGL((linear_chunk_kernel<T, D, false, VEC>), dim3(heads, p.segments, p.group), block, 0, s, p);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch(const LinearParams& p, hipStream_t s) {
  const int64_t most = (int64_t(1) << 31) / 256 - D;  // 64 rows of 4 bytes an element
  const bool vec = p.q.vec && p.k.vec && p.v.vec && p.o.vec && p.q.st < most && p.k.st < most && p.v.st < most && p.o.st < most;
  return vec ? launch<T, D, true>(p, s) : launch<T, D, false>(p, s);
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
