// The cache's words of 32 tokens of one kv head, as a wavefront holds them.
//
// Lane 16 g + m has, of K, the nibbles of channels 8 g .. +7 of every group of
// tokens 8 (m / 4) + m % 4 and + 4, and of V those of octet g's eight tokens
// for NC runs of WPL channels from 4 m (2 m with 32 channels).
#pragma once

#include "dev_attn.h"

namespace fluid {

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t w[N]) {
  typedef uint32_t vec __attribute__((ext_vector_type(N)));
  if constexpr (N == 1) {
    w[0] = __builtin_nontemporal_load((const uint32_t*)p);
  } else {
    const vec v = __builtin_nontemporal_load((const vec*)p);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = v[i];
  }
}

// The cache's words of one tile that a lane needs.
template <int D>
struct KvTile {
  static constexpr int G = D / 32, WPL = D == 32 ? 2 : 4, NC = D == 32 ? 1 : D / 64;
  uint32_t kw[2][G], kp[2][G];
  uint32_t vw[NC][WPL], vs[NC][4], vb[NC][4];

  // blk, P and slot are the same for all lanes; what a lane adds to the four
  // parts' starts is not, but the same for every tile
  struct Lane { uint32_t k, kp, v, vp; };
  __device__ static __forceinline__ Lane lane_offsets(int lane) {
    const int m = lane & 15, g = lane >> 4, t = 8 * (m >> 2) + (m & 3);
    return {(uint32_t)(t * (D / 2) + g * (4 * G)), (uint32_t)(t * (4 * G)), (uint32_t)(g * (4 * D) + 4 * WPL * m),
            (uint32_t)(g * (32 * G) + (D == 32 ? 0 : 32 * (m >> 3)))};
  }
  __device__ __forceinline__ void load_k(const uint8_t* blk, int P, int slot, const Lane& at) {
    const uint8_t* const k = blk + slot * (D / 2);
    const uint8_t* const kpairs = blk + P * (D / 2) + slot * (4 * G);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_words<G>(k + at.k + 4 * i * (D / 2), kw[i]);
      load_words<G>(kpairs + at.kp + 4 * i * (4 * G), kp[i]);
    }
  }
  __device__ __forceinline__ void load_v(const uint8_t* blk, int P, int slot, const Lane& at) {
    const uint8_t* const v = blk + P * (D / 2 + 4 * G) + slot * (D / 2);
    const uint8_t* const vpairs = blk + P * (D + 4 * G) + slot * (4 * G);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      load_words<WPL>(v + at.v + 256 * c, vw[c]);
      load_words<4>(vpairs + at.vp + 64 * c, vs[c]);
      load_words<4>(vpairs + at.vp + 64 * c + 16, vb[c]);
    }
  }
};

}  // namespace fluid
