// Operands of the products with matrices in 4 bits.
//
// A nibble in bits 3 .. 6 of a bf16 with the exponent of 16 reads 16 + n, exact,
// so a word becomes an operand in eight instructions; a group's products with x
// are summed in fp32, and so are x's own (a product with ones): the group adds
// s sum x (16 + n) + b sum x.  No weight is rounded.  A lane's words are one row's,
// so it needs that row's pair alone.
#pragma once

#include "../attn/dev_attn.h"
#include "params.h"

namespace fluid {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Channels of x as they are loaded, and as operands whose sum they are; a word's
// eight levels as the other operand, n + OFFSET.
template <typename T>
struct Rows;
template <>
struct Rows<uint16_t> {
  static constexpr int N = 1;
  static constexpr float OFFSET = 16.0f;
  typedef uint32_t unaligned __attribute__((ext_vector_type(4), aligned(2)));
  u32x4 raw;
  __device__ __forceinline__ void load(const uint16_t* x) { raw = *(const unaligned*)x; }
  __device__ __forceinline__ void load(const uint16_t* x, int left) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      raw[i] = (2 * i < left ? x[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)x[2 * i + 1] << 16 : 0u);
  }
  // without the first n channels, zeros behind the others
  __device__ __forceinline__ void drop(int n) {
    if (n & 1) raw = u32x4{raw[0] >> 16 | raw[1] << 16, raw[1] >> 16 | raw[2] << 16, raw[2] >> 16 | raw[3] << 16, raw[3] >> 16};
    if (n & 2) raw = u32x4{raw[1], raw[2], raw[3], 0};
    if (n & 4) raw = u32x4{raw[2], raw[3], 0, 0};
    if (n >= 8) raw = u32x4{};
  }
  // in LDS
  static constexpr int PLANES = 1;
  __device__ __forceinline__ void put(u32x4* at, int plane) const { at[0] = raw; }
  __device__ __forceinline__ void get(const u32x4* at, int plane) { raw = at[0]; }
  __device__ __forceinline__ void parts(u32x4 p[N]) const { p[0] = raw; }
  __device__ static __forceinline__ u32x4 levels(uint32_t w) {
    constexpr uint32_t mask = 0x00780078, sixteen = 0x41804180;
    return u32x4{((w << 3) & mask) | sixteen, ((w >> 1) & mask) | sixteen, ((w >> 5) & mask) | sixteen,
                 ((w >> 9) & mask) | sixteen};
  }
};
template <>
struct Rows<float> {
  static constexpr int N = 3;
  // about zero, so that a group's sums are no larger than they need be: with 16 + n
  // the error of 4096 channels was 2.5 times that of an fp32 product
  static constexpr float OFFSET = -8.0f;
  typedef float unaligned __attribute__((ext_vector_type(4), aligned(4)));
  f32x4 raw[2];
  __device__ __forceinline__ void load(const float* x) {
    raw[0] = ((const unaligned*)x)[0], raw[1] = ((const unaligned*)x)[1];
  }
  __device__ __forceinline__ void load(const float* x, int left) {
#pragma unroll
    for (int e = 0; e < 8; ++e) raw[e >> 2][e & 3] = e < left ? x[e] : 0.0f;
  }
  __device__ __forceinline__ void drop(int n) {
    if (n & 1) {
      raw[0] = f32x4{raw[0][1], raw[0][2], raw[0][3], raw[1][0]};
      raw[1] = f32x4{raw[1][1], raw[1][2], raw[1][3], 0.0f};
    }
    if (n & 2) {
      raw[0] = f32x4{raw[0][2], raw[0][3], raw[1][0], raw[1][1]};
      raw[1] = f32x4{raw[1][2], raw[1][3], 0.0f, 0.0f};
    }
    if (n & 4) raw[0] = raw[1], raw[1] = f32x4{};
    if (n >= 8) raw[0] = raw[1] = f32x4{};
  }
  static constexpr int PLANES = 2;
  __device__ __forceinline__ void put(u32x4* at, int plane) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) at[i * plane] = __builtin_bit_cast(u32x4, raw[i]);
  }
  __device__ __forceinline__ void get(const u32x4* at, int plane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) raw[i] = __builtin_bit_cast(f32x4, at[i * plane]);
  }
  // the first two parts are cut off, so that what is left is exact
  __device__ __forceinline__ void parts(u32x4 p[N]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = raw[i >> 1][2 * (i & 1)], b = raw[i >> 1][2 * (i & 1) + 1];
      const uint32_t ah = __float_as_uint(a) & 0xffff0000u, bh = __float_as_uint(b) & 0xffff0000u;
      const float a1 = a - __uint_as_float(ah), b1 = b - __uint_as_float(bh);
      const uint32_t am = __float_as_uint(a1) & 0xffff0000u, bm = __float_as_uint(b1) & 0xffff0000u;
      p[0][i] = (ah >> 16) | bh;
      p[1][i] = (am >> 16) | bm;
      p[2][i] = pack_bf16(a1 - __uint_as_float(am), b1 - __uint_as_float(bm));
    }
  }
  __device__ static __forceinline__ u32x4 levels(uint32_t w) {
    u32x4 l = Rows<uint16_t>::levels(w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = __uint_as_float(l[i] << 16) - 24.0f, hi = __uint_as_float(l[i] & 0xffff0000u) - 24.0f;
      l[i] = (__float_as_uint(lo) >> 16) | __float_as_uint(hi);  // exact: the lower halves are zero
    }
    return l;
  }
};

// How eight channels of a row of x are loaded: one by one (rows of fewer than eight);
// at once, the row's last ones from where they end with it; or, where rows start at
// odd halves of a word, as the words that hold them (16 bytes at such an address took
// 8 rows of 4095 channels from 5 to 14 us).
enum Load { kOneByOne, kAtOnce, kByWords };

template <typename T, Load HOW>
struct Piece : Rows<T> {
  __device__ __forceinline__ void fetch(const T* row, int ch, int k) {
    if constexpr (HOW == kOneByOne) this->load(row + ch, k - ch);
    else this->load(row + min(ch, k - 8));
  }
  // before use; last: the block ends behind the row
  __device__ __forceinline__ void settle(int ch, int k, bool last) {
    if (HOW != kOneByOne && last) this->drop(max(ch - (k - 8), 0));
  }
};
template <>
struct Piece<uint16_t, kByWords> : Rows<uint16_t> {
  uint32_t end, shift;
  __device__ __forceinline__ void fetch(const uint16_t* row, int ch, int k) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(4)));
    const uintptr_t at = (uintptr_t)(row + min(ch, k - 8));
    raw = *(const words*)(at & ~uintptr_t(3));
    end = *(const uint32_t*)((at + 14) & ~uintptr_t(3));  // the word of the last channel
    shift = (at & 2) * 8;
  }
  __device__ __forceinline__ void settle(int ch, int k, bool last) {
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = __builtin_amdgcn_alignbit(i < 3 ? raw[i + 1] : end, raw[i], shift);
    if (last) drop(max(ch - (k - 8), 0));
  }
};
template <typename T>
inline bool by_words(const W4Params& p) {
  return sizeof(T) == 2 && ((uintptr_t)p.x % 4 || p.xs % 2);
}

// A group's sums of x times levels, and of x, into y.
template <typename T>
__device__ __forceinline__ void add_group(f16x2 sb, f32x4 part, f32x4 all, f32x4& y) {
  const float s = (float)sb[0], b = __builtin_fmaf(16.0f - Rows<T>::OFFSET, s, (float)sb[1]);
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = __builtin_fmaf(s, part[e], __builtin_fmaf(b, all[e], y[e]));
}

// Row m, output col: y, with the gate's product z and the residual.
template <typename T>
__device__ __forceinline__ void finish(const W4Params& p, int m, int col, float y, float z, bool gate) {
  if (gate) y *= z / (1.0f + expf(-z));
  if (p.add) y += Elem<T>::load((const T*)p.add + m * p.as, col);
  Elem<T>::store((T*)p.out + m * p.os, col, y);
}

// A lane's pairs of its row in one block.
template <int GROUPS>
__device__ __forceinline__ void load_pairs(const uint8_t* at, f16x2 sb[GROUPS]) {
  if constexpr (GROUPS == 4) *(u32x4*)sb = *(const u32x4*)at;
  else if constexpr (GROUPS == 2) *(uint2*)sb = *(const uint2*)at;
  else sb[0] = *(const f16x2*)at;
}

}  // namespace fluid
