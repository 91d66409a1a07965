// The 4-bit cache written and read back (format: fluid_attention.h).
//
// A half-wavefront owns one octet of tokens and one group of 32 channels, of
// K or of V: lane 4 L + q holds the eight channels 8 q .. +7 (16 bytes of
// bf16) of the octet's token nibble_element(L).  The group's extremes are two
// steps within a quad of lanes; a lane's eight nibbles are just one word of
// K, and an 8 x 8 transpose of nibbles over the lanes that share q, in three
// exchanges, makes the words of V.  Bound by memory: each value is read once
// and 5 bits of it written, or the reverse.
#include "dev_attn.h"
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

// What a half-wavefront works on: which octet, group and head, and where.
template <int D>
struct Unit {
  static constexpr int G = D / 32;
  int b, h, g, L, q, t;
  bool is_v, ok, mine;  // ok: the octet has a place; mine: this lane's token is one of the call's
  int64_t row;          // of the call's tensors
  uint8_t* base;        // of the (page, head) block
  int slot, P;          // the token's place in the page, tokens a page

  __device__ __forceinline__ Unit(const KvIoParams& p) {
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    int64_t item = unit / (2 * G);
    const int part = (int)(unit - item * (2 * G));
    is_v = part >= G;
    g = is_v ? part - G : part;
    q = lane & 3;
    L = lane >> 2;
    t = nibble_element(L);
    ok = item < p.items;
    mine = false;
    if (!ok) return;
    h = (int)(item % p.c.kv_heads);
    item /= p.c.kv_heads;
    const int o = (int)(item % p.octets);
    b = (int)(item / p.octets);
    const int64_t start = p.start[b];
    const int n = clamp_len(p.count, b, p.tokens);
    const int64_t first = (start & ~(int64_t)7) + 8 * (int64_t)o;  // floor, negative starts too
    ok = first >= 0 && first < p.c.capacity && first < start + n;
    if (!ok) return;
    P = 1 << p.c.log_page;
    const int page = p.c.pages[b * p.c.table_stride + (first >> p.c.log_page)];
    ok = page >= 0 && page < p.c.n_pages;
    if (!ok) return;
    row = first + t - start;
    mine = row >= 0 && row < n;
    slot = (int)(first & (P - 1)) + t;
    base = p.c.pool + ((int64_t)page * p.c.kv_heads + h) * p.c.block;
  }
  __device__ __forceinline__ uint32_t* k_word() const { return (uint32_t*)base + slot * (D / 8) + q * G + g; }
  __device__ __forceinline__ uint32_t* k_pair() const { return (uint32_t*)base + P * (D / 8) + slot * G + g; }
  // after the transpose lane (L, q) has the word of channel 8 q + t
  __device__ __forceinline__ uint32_t* v_word() const {
    return (uint32_t*)base + P * (D / 8 + G) + (slot >> 3) * D + 32 * g + 8 * q + t;
  }
  __device__ __forceinline__ _Float16* v_pair() const {
    return (_Float16*)((uint32_t*)base + P * (D / 8 + G + D / 8)) + ((slot >> 3) * G + g) * 16 + t;
  }
};

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_write_kernel(KvIoParams p) {
  // lo - 16 s is rounded to fp32 before it is rounded to f16: a fused form
  // that rounds once gives another b for one group in some 20000
#pragma clang fp contract(off)
  const Unit<D> u(p);
  if (!u.ok) return;  // whole half-wavefronts: the exchanges below stay within one
  const TokensArg& a = u.is_v ? p.v : p.k;
  Eight<T> raw = {};
  if (u.mine) raw.load((const T*)a.p + u.b * a.sb + u.row * a.st + u.h * a.sh + 32 * u.g + 8 * u.q, a.vec);
  float x[8];
  raw.floats(x);
  float lo = 16384.0f, hi = -16384.0f, odd = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (!(fabsf(x[i]) <= 3.402823466e38f)) odd = 1.0f;
    x[i] = fminf(fmaxf(x[i], -16384.0f), 16384.0f);
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
  lo = quad_min(lo);
  hi = quad_max(hi);
  odd = quad_max(odd);
  _Float16 sh = (_Float16)((hi - lo) / 15.0f);
  if (odd != 0.0f) sh = (_Float16)0.0f;
  const float s = (float)sh;
  _Float16 bh = (_Float16)(lo - 16.0f * s);
  const float b = (float)bh;
  if (odd != 0.0f) bh = __builtin_bit_cast(_Float16, (uint16_t)0x7e00);
  // (x - b) / s by the reciprocal and one correction, which rounds as the
  // division does: s has 11 bits, so its fp32 reciprocal is the nearest one
  const float r = 1.0f / s;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float d = x[e] - b, q0 = d * r;
    const float qt = __builtin_fmaf(__builtin_fmaf(-q0, s, d), r, q0);
    const float n = fminf(fmaxf(__builtin_rintf(qt) - 16.0f, 0.0f), 15.0f);
    w |= (s > 0.0f ? (uint32_t)n : 0u) << (4 * ((e >> 1) + 4 * (e & 1)));
  }
  if (!u.is_v) {
    if (u.mine) {
      *u.k_word() = w;
      if (u.q == 0) *u.k_pair() = __builtin_bit_cast(uint16_t, sh) | ((uint32_t)__builtin_bit_cast(uint16_t, bh) << 16);
    }
    return;
  }
  // lane 4 L + q votes on the token that nibble L holds: the half's 32 votes
  // are the mask of the nibbles to change
  const uint64_t votes = __ballot(u.mine);
  const uint32_t mask = (uint32_t)(votes >> (threadIdx.x & 32));
  w = transpose_nibbles(w, u.L);
  uint32_t* const to = u.v_word();
  *to = mask == 0xffffffffu ? w : (*to & ~mask) | (w & mask);
  if (u.mine && u.q == 0) {
    u.v_pair()[0] = sh;
    u.v_pair()[8] = bh;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvIoParams p) {
  const Unit<D> u(p);
  if (!u.ok) return;
  uint32_t w, pair;
  if (!u.is_v) {
    w = *u.k_word();
    pair = *u.k_pair();
  } else {
    w = transpose_nibbles(*u.v_word(), u.L);
    const uint16_t* vp = (const uint16_t*)u.v_pair();
    pair = vp[0] | ((uint32_t)vp[8] << 16);
  }
  if (!u.mine) return;
  const f16x8 v = word_values(Magic(), w, pair);
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  const TokensArg& a = u.is_v ? p.v : p.k;
  store8((T*)a.p + u.b * a.sb + u.row * a.st + u.h * a.sh + 32 * u.g + 8 * u.q, a.vec, x);
}

template <typename T>
hipError_t launch(const KvIoParams& p, int D, bool write, hipStream_t s) {
  const int64_t units = p.items * (D / 16);
  const dim3 grid((uint32_t)((units + 7) / 8)), block(256);
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
