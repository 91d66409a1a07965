// The 4-bit cache written and read back (format: fluid_attention.h).
//
// Writing, a wavefront takes one octet of tokens of one kv head, a group of 32
// channels of K or V to each half of it at a time: lane 4 L + q holds the
// eight channels 8 q .. +7 (16 bytes of bf16) of the octet's token
// nibble_element(L).  The group's extremes are two steps within a quad of
// lanes; a lane's eight nibbles are just one word of K, and an 8 x 8 transpose
// of nibbles over the lanes that share q, in three exchanges, makes the words
// of V.  Reading, it takes 32 tokens and holds them as attention does.
//
// Each value is read once and 5 bits of it written, or the reverse.  Reading
// is bound by memory: 8192 tokens of 32 heads of 128 to bf16, 176 MB, in 39 us
// (4.5 TB/s; a copy of 4 GiB has 4.7).  Non-temporal stores made the reads of
// 512 to 1024 tokens 10 % faster and the attention that follows slower (512
// queries over 8192 tokens and 32 heads, with the read: 161 us, 189 with them).
// Writing has some 20 vector instructions a value, 84 % of the cycles of the 13.4
// us that 2048 tokens (44 MB) take; all wavefronts of so many fit the GPU at once,
// so loads and arithmetic overlap little.  One token or 16 take 5 to 6 us: the
// launch and a chain of dependent loads (lengths; the page, beside the values to
// write; the words to read, or those that keep some of their nibbles).
#include "kv_tile.h"
#include "launch_attn.h"

namespace fluid {

namespace {

// Transpose of the 8 x 8 matrix whose row L is the word of lane L (bits 2..4
// of the lane), columns its nibbles.
__device__ __forceinline__ uint32_t transpose_nibbles(uint32_t w, int L) {
  uint32_t o = __shfl_xor(w, 16);
  w = L & 4 ? (w & 0xffff0000u) | (o >> 16) : (w & 0x0000ffffu) | (o << 16);
  o = __shfl_xor(w, 8);
  w = L & 2 ? (w & 0xff00ff00u) | ((o >> 8) & 0x00ff00ffu) : (w & 0x00ff00ffu) | ((o & 0x00ff00ffu) << 8);
  o = __shfl_xor(w, 4);
  return L & 1 ? (w & 0xf0f0f0f0u) | ((o >> 4) & 0x0f0f0f0fu) : (w & 0x0f0f0f0fu) | ((o & 0x0f0f0f0fu) << 4);
}

// The run of `span` tokens (8 or 32, at a multiple of it) and the head that a
// wavefront works on.
struct Run {
  int b, h;
  int64_t first, start;  // tokens: the run's, the call's
  int n;                 // tokens of the call
  int slot;              // the run's place in its page
  uint8_t* block;        // of the (page, head)

  // false: none of the call's tokens is here
  __device__ __forceinline__ bool locate(const KvIoParams& p, int64_t item, int span) {
    if (item >= p.items) return false;
    int x = (int)fdiv((uint32_t)item, p.div_heads);
    h = (int)item - x * p.c.kv_heads;
    b = (int)fdiv((uint32_t)x, p.div_runs);
    const int o = x - b * p.runs;
    start = uniform_load(p.start, b);
    n = clamp_len(p.count, b, p.tokens);
    first = (start & -(int64_t)span) + span * (int64_t)o;  // floor, negative starts too
    return n != 0 && first >= 0 && first < p.c.capacity && first < start + n;
  }
  // false: the page holds no tokens; block is then page 0's
  __device__ __forceinline__ bool place(const KvIoParams& p) {
    const int page = uniform_load(p.c.pages, b * p.c.table_stride + (first >> p.c.log_page));
    const bool held = (uint32_t)page < (uint32_t)p.c.n_pages;
    slot = (int)first & ((1 << p.c.log_page) - 1);
    block = p.c.pool + ((int64_t)(held ? page : 0) * p.c.kv_heads + h) * p.c.block;
    return held;
  }
  // row of the call's tensors that holds token t of the run, if it is one
  __device__ __forceinline__ bool row(int t, int64_t& r) const {
    r = first + t - start;
    return r >= 0 && r < n;
  }
};

__device__ __forceinline__ float clamped(float x) { return fminf(fmaxf(x, -kLimit), kLimit); }
// what eight nibbles' 1.5 2^23 + 16 add to a word, modulo 2^32
constexpr uint32_t kMagicWord = 0x4B400010u * 0x11111111u;

// Wavefront index of the launch.
__device__ __forceinline__ int64_t wave_index() {
  return (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_write_kernel(KvIoParams p) {
  constexpr int G = D / 32;
  Run run;
  if (!run.locate(p, wave_index(), 8)) return;
  const int lane = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1, q = lane & 3, L = lane >> 2, t = nibble_element(L);
  int64_t row;
  const bool within = run.row(t, row);
  // the values are on their way while the page is looked up, and the words of
  // V that keep some of their nibbles while the values are
  // parts 0 .. G - 1 are the groups of K, G .. 2 G - 1 those of V, two at a
  // time; lanes without a token of the call read one that is
  const int64_t from = min(max(row, (int64_t)0), (int64_t)run.n - 1);
  const T* const kt = (const T*)p.k.p + run.b * p.k.sb + run.h * p.k.sh + (from * p.k.st + 8 * q);
  const T* const vt = (const T*)p.v.p + run.b * p.v.sb + run.h * p.v.sh + (from * p.v.st + 8 * q);
  Eight<T> raw[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const T* const at = G == 1 ? (half ? vt : kt) : 2 * i < G ? kt + 32 * (2 * i + half) : vt + 32 * (2 * i - G + half);
    raw[i].load(at, 2 * i < G && !(G == 1 && half) ? p.k.vec : p.v.vec);
  }
  const bool mine = run.place(p) && within;
  // lane 4 L + q votes on the token that nibble L holds: a half's 32 votes
  // are the mask of the nibbles of V to change
  const uint32_t mask = (uint32_t)__ballot(mine);
  const int P = 1 << p.c.log_page, slot = run.slot + t;
  uint32_t* const base = (uint32_t*)run.block;
  uint32_t* const words = base + P * (D / 8 + G) + (slot >> 3) * D + 8 * q + t;  // of V, channel 8 q + t of a group
  uint32_t old[G] = {};
  if (mask != 0xffffffffu) {
#pragma unroll
    for (int i = 0; i < G; ++i)
      if (2 * i + half >= G) old[i] = words[32 * ((2 * i + half) % G)];
  }
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int part = 2 * i + half, g = part % G;
    float x[8];
    raw[i].floats(x);
    float lo = x[0], hi = x[0], odd = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      odd = __builtin_fmaf(x[e], 0.0f, odd);  // NaN from an infinity or a NaN on
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
    }
    lo = quad_min(lo);
    hi = quad_max(hi);
    odd += dpp<0xB1>(odd);
    odd += dpp<0x4E>(odd);
    if (__builtin_expect(__ballot(!(lo >= -kLimit && hi <= kLimit)) != 0, 0)) {
      lo = clamped(lo);
      hi = clamped(hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = clamped(x[e]);
    }
    // (hi - lo) / 15 and below (x - b) / s by the reciprocal and one
    // correction, which rounds as the division does where the reciprocal is
    // the nearest fp32 value
    const float span = hi - lo, s0 = span * (1.0f / 15.0f);
    _Float16 sh = half_of(__builtin_fmaf(__builtin_fmaf(-s0, 15.0f, span), 1.0f / 15.0f, s0));
    if (odd != odd) sh = (_Float16)0.0f;
    const float s = (float)sh;
    _Float16 bh = half_of(lo - 16.0f * s);
    const float b = (float)bh;
    if (odd != odd) bh = __builtin_bit_cast(_Float16, (uint16_t)0x7e00);
    const uint32_t s16 = __builtin_bit_cast(uint16_t, sh), b16 = __builtin_bit_cast(uint16_t, bh);
    // Added to 1.5 2^23 the quotient is rounded to a whole number, 16 + n, in
    // the low bits; the words are summed with what lies above them, a constant.
    const float r = s > 0.0f ? 1.0f / s : 0.0f;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = x[e] - b, q0 = d * r;
      const float qt = __builtin_fmaf(__builtin_fmaf(-q0, s, d), r, q0);
      const float n = fminf(fmaxf(qt, 16.0f), 31.0f) + 12582912.0f;
      w += __float_as_uint(n) << (4 * ((e >> 1) + 4 * (e & 1)));
    }
    w -= kMagicWord;
    if (part < G) {
      if (mine) {
        base[slot * (D / 8) + q * G + g] = w;
        if (q == 0) base[P * (D / 8) + slot * G + g] = s16 | b16 << 16;
      }
    } else {
      w = transpose_nibbles(w, L);  // now of channel 8 q + t
      if (mask != 0) words[32 * g] = (old[i] & ~mask) | (w & mask);
      if (mine && q == 0) {
        uint16_t* const pair = (uint16_t*)(base + P * (D / 4 + G)) + ((slot >> 3) * G + g) * 16 + t;
        pair[0] = (uint16_t)s16;
        pair[8] = (uint16_t)b16;
      }
    }
  }
}

// N neighbouring elements from f16.
template <typename T, int N>
__device__ __forceinline__ void store_values(T* to, bool vec, const _Float16* v) {
  if (vec) {
    if constexpr (sizeof(T) == 2) {
      typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
      if constexpr (N == 2) {
        *(uint32_t*)to = pack_bf16((float)v[0], (float)v[1]);
      } else {
        words w;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16((float)v[2 * i], (float)v[2 * i + 1]);
        *(words*)to = w;
      }
    } else {
      typedef float floats __attribute__((ext_vector_type(N > 4 ? 4 : N)));
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        floats f;
#pragma unroll
        for (int j = 0; j < (N > 4 ? 4 : N); ++j) f[j] = (float)v[i + j];
        *(floats*)(to + i) = f;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) Elem<T>::store(to, i, (float)v[i]);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvIoParams p) {
  using Tile = KvTile<D>;
  constexpr int G = Tile::G, WPL = Tile::WPL, NC = Tile::NC;
  Run run;
  if (!run.locate(p, wave_index(), kKvTile) || !run.place(p)) return;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, P = 1 << p.c.log_page;
  const Magic mg;
  Tile tile;
  tile.load_k(run.block, P, run.slot, Tile::lane_offsets(lane));
  tile.load_v(run.block, P, run.slot, Tile::lane_offsets(lane));
  T* const kt = (T*)p.k.p + run.b * p.k.sb + run.h * p.k.sh;
  T* const vt = (T*)p.v.p + run.b * p.v.sb + run.h * p.v.sh;
  int64_t row;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!run.row(8 * (m >> 2) + (m & 3) + 4 * i, row)) continue;
#pragma unroll
    for (int j = 0; j < G; ++j) {
      const f16x8 v = word_values(mg, tile.kw[i][j], tile.kp[i][j]);
      store_values<T, 8>(kt + row * p.k.st + 32 * j + 8 * g, p.k.vec, (const _Float16*)&v);
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    f16x8 v[WPL];  // of a channel, eight tokens
    f16x2 vs[4], vb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      vs[i] = __builtin_bit_cast(f16x2, tile.vs[c][i]);
      vb[i] = __builtin_bit_cast(f16x2, tile.vb[c][i]);
    }
#pragma unroll
    for (int j = 0; j < WPL; ++j) v[j] = word_values(mg, tile.vw[c][j], vs, vb);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!run.row(8 * g + e, row)) continue;
      _Float16 of[WPL];
#pragma unroll
      for (int j = 0; j < WPL; ++j) of[j] = v[j][e];
      store_values<T, WPL>(vt + row * p.v.st + 64 * c + WPL * m, p.v.vec, of);
    }
  }
}

template <typename T>
hipError_t launch(const KvIoParams& p, int D, bool write, hipStream_t s) {
  const dim3 grid((uint32_t)((p.items + 3) / 4)), block(256);
#define FLUID_KV_D(N)                                                              \
  case N:                                                                          \
    if (write) hipLaunchKernelGGL((kv_write_kernel<T, N>), grid, block, 0, s, p); \
    else hipLaunchKernelGGL((kv_read_kernel<T, N>), grid, block, 0, s, p);        \
    break;
  switch (D) {
    FLUID_KV_D(32)
    FLUID_KV_D(64)
    FLUID_KV_D(128)
  }
#undef FLUID_KV_D
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_io(const KvIoParams& p, int dtype, int head_dim, bool write, hipStream_t s) {
  return dtype == DT_BF16 ? launch<uint16_t>(p, head_dim, write, s) : launch<float>(p, head_dim, write, s);
}

}  // namespace fluid
