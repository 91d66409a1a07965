// Device helpers of the cache and attention kernels.
#pragma once

#include "../gpu/dev.h"
#include "params.h"

namespace fluid {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A running maximum before the first score: none is below it, so a row that sees
// tokens gives weight to some.
constexpr float kLow = -3.402823466e38f;

// A weight is 2 to the power of score * scale - maximum, fused: the product's
// rounding, which the maximum has, is left out of it.  That is at most 1/8 up to
// here, but 2^(m - 24) at 2^m: maxima from 2^31 on would make infinite weights, so
// rows past this bound have their products rounded first.
constexpr float kFusedMost = 4194304.0f;
__device__ __forceinline__ bool past_fused(float m) { return (fabsf(m) > kFusedMost) & (m != kLow); }

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
// over the four lanes of a quad
__device__ __forceinline__ float quad_min(float v) {
  v = fminf(v, dpp<0xB1>(v));
  return fminf(v, dpp<0x4E>(v));
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  return fmaxf(v, dpp<0x4E>(v));
}

// Element of a word that its nibble i holds (the inverse of
// e -> (e >> 1) + 4 (e & 1)): nibbles i and i + 4 are neighbours, so that an
// AND-OR makes a pair of f16 of them.
__device__ __forceinline__ int nibble_element(int i) { return ((i & 3) << 1) | (i >> 2); }

// The two constants that make f16 of nibbles.  They are opaque to the compiler
// so that each stays in a register: an AND-OR of literals is two instructions.
struct Magic {
  uint32_t mask, sixteen;
  __device__ __forceinline__ Magic() {
    asm("s_mov_b32 %0, 0x03c003c0" : "=s"(mask));
    asm("v_mov_b32 %0, 0x4c004c00" : "=v"(sixteen));
  }
};
// The values of a word's elements 2 i and 2 i + 1 as one f16 pair: the two
// nibbles moved to bits 6..9 of their halves and given the exponent of 16
// read as 16 + n, and one fused multiply-add finishes b + s (16 + n).
template <int I>
__device__ __forceinline__ f16x2 nibble_pair(const Magic& mg, uint32_t w, f16x2 s, f16x2 b) {
  const uint32_t x = I == 0 ? w << 6 : I == 1 ? w << 2 : I == 2 ? w >> 2 : w >> 6;
  const f16x2 n = __builtin_bit_cast(f16x2, (x & mg.mask) | mg.sixteen);
  return __builtin_elementwise_fma(n, s, b);
}
// A word's eight values, one (s, b) for all (K) or a pair per two (V).
__device__ __forceinline__ f16x8 word_values(const Magic& mg, uint32_t w, const f16x2 s[4], const f16x2 b[4]) {
  union { f16x2 h[4]; f16x8 v; } u;
  u.h[0] = nibble_pair<0>(mg, w, s[0], b[0]);
  u.h[1] = nibble_pair<1>(mg, w, s[1], b[1]);
  u.h[2] = nibble_pair<2>(mg, w, s[2], b[2]);
  u.h[3] = nibble_pair<3>(mg, w, s[3], b[3]);
  return u.v;
}
__device__ __forceinline__ f16x8 word_values(const Magic& mg, uint32_t w, uint32_t pair) {
  const f16x2 p = __builtin_bit_cast(f16x2, pair);
  const f16x2 s = {p[0], p[0]}, b = {p[1], p[1]};
  const f16x2 ss[4] = {s, s, s, s}, bb[4] = {b, b, b, b};
  return word_values(mg, w, ss, bb);
}

// Eight neighbouring elements; vec: the address is 16-byte aligned.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p, bool vec) {
    if (vec) {
      a = ((const f32x4*)p)[0];
      b = ((const f32x4*)p)[1];
    } else {
      a = f32x4{p[0], p[1], p[2], p[3]};
      b = f32x4{p[4], p[5], p[6], p[7]};
    }
  }
  __device__ __forceinline__ void floats(float x[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
};
template <>
struct Eight<uint16_t> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const uint16_t* p, bool vec) {
    if (vec) {
      const uint4 a = *(const uint4*)p;
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
    }
  }
  __device__ __forceinline__ void floats(float x[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
};
template <typename T>
__device__ __forceinline__ void store8(T* p, bool vec, const float x[8]);
template <>
__device__ __forceinline__ void store8<float>(float* p, bool vec, const float x[8]) {
  if (vec) {
    ((f32x4*)p)[0] = f32x4{x[0], x[1], x[2], x[3]};
    ((f32x4*)p)[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = x[i];
  }
}
template <>
__device__ __forceinline__ void store8<uint16_t>(uint16_t* p, bool vec, const float x[8]) {
  if (vec) {
    *(uint4*)p = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = f32_to_bf16(x[i]);
  }
}

// over a wavefront, the same for all lanes
__device__ __forceinline__ int wave_total(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // from the lane 1, 2, 4, 8 before it in its row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // a row's last lane to the next row
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to the upper rows
  return __builtin_amdgcn_readlane(v, 63);
}

// A value that all lanes read, by a scalar load: the lengths and page tables
// are not written while a kernel runs.
__device__ __forceinline__ int uniform_load(const int32_t* p, int64_t i) {
  return ((const __attribute__((address_space(4))) int32_t*)p)[i];
}
__device__ __forceinline__ int clamp_len(const int32_t* len, int b, int most) {
  return len ? min(max(uniform_load(len, b), 0), most) : most;
}

// The tiles of `tile` tokens that rows at positions p_min .. p_max (of n
// tokens) have to visit, numbered without gaps: first those of the sinks
// before the window, then those from the window's start to the last token
// seen.
struct TileRange {
  int sink_tiles, first, count;
  __device__ __forceinline__ int tile(int u) const { return u < sink_tiles ? u : first + (u - sink_tiles); }
};
__device__ __forceinline__ TileRange tile_range(const AttnParams& p, int p_min, int p_max, int n, int tile) {
  int hi = n, lo = 0, s = 0;
  if (p.causal) hi = min(hi, p_max + 1);
  else if (p.window > 0) hi = min(hi, p_max + p.window);
  if (p.window > 0) {
    lo = max(0, p_min - p.window + 1);
    s = max(0, min(p.sinks, p.causal ? hi : n));
  }
  const int a = (s + tile - 1) / tile;
  TileRange r;
  if (hi <= lo) {
    r.first = 0;
    r.sink_tiles = r.count = a;
  } else {
    r.first = lo / tile;
    r.sink_tiles = min(a, r.first);
    r.count = r.sink_tiles + max((hi + tile - 1) / tile, a) - r.first;
  }
  return r;
}

// The tokens that the row at position `pos` sees: lo .. lo + span - 1 and those
// below sinks.
struct Sight {
  int lo, span, sinks;
  __device__ __forceinline__ bool sees(int t) const { return (uint32_t)(t - lo) < (uint32_t)span | t < sinks; }
};
__device__ __forceinline__ Sight sight(const AttnParams& p, int pos, int n) {
  int hi = n;
  Sight s = {0, 0, 0};
  if (p.causal) hi = min(hi, pos + 1);
  else if (p.window > 0) hi = min(hi, pos + p.window);
  if (p.window > 0) {
    s.lo = max(0, pos - p.window + 1);
    s.sinks = min(p.sinks, p.causal ? hi : n);
  }
  s.span = max(0, hi - s.lo);
  return s;
}

// One tile of rows of one kv head, and the tiles of tokens it visits.
struct Item {
  int b, h, rt;
  int n, rows, p0;  // tokens; rows of the kv head; position of row 0's query
  int r0, r1;
  TileRange range;
  __device__ __forceinline__ void sequence(const AttnParams& p, int b_) {
    b = b_;
    n = clamp_len(p.kv_len, b, p.kv_tokens);
    const int ql = clamp_len(p.q_len, b, p.q_tokens);
    rows = ql * p.group;
    p0 = n - ql;
  }
  __device__ __forceinline__ int p_min(const AttnParams& p) const { return p0 + (int)fdiv(r0, p.div_group); }
  __device__ __forceinline__ int p_max(const AttnParams& p) const { return p0 + (int)fdiv(r1 - 1, p.div_group); }
  // The row tile rt of the sequence; false if it has no rows.
  __device__ __forceinline__ bool tile(const AttnParams& p, int rt_) {
    rt = rt_;
    r0 = rt * p.row_tile;
    r1 = min(r0 + p.row_tile, rows);
    if (r0 >= rows) return false;
    range = tile_range(p, p_min(p), p_max(p), n, p.token_tile);
    return true;
  }
};

// What a workgroup works on: a run of an item's steps.  With p.splits shares
// to an item each has p.chunk steps, or as many more as an item that proves
// longer than the host expected needs; one that is shorter leaves the last
// shares idle.  An item in one share is written by its workgroup, the others
// are put together by the join.
struct Share {
  Item item;
  int index, split;  // of the item and of its share
  int shares;        // that the item has
  int first, end;    // steps

  __device__ __forceinline__ void steps(const AttnParams& p) {
    const int per = max(p.chunk, (int)fdiv(item.range.count + p.splits - 1, p.div_splits));
    shares = max(1, (item.range.count + per - 1) / per);
    first = split * per;
    end = min(first + per, item.range.count);
  }
  // The k-th longest row tile of the heads head0, head0 + rank_step, .., one
  // share each: by the position it starts at in units of a tile's rows, or by
  // the sequence's length where no mask cuts it off.  Lane i counts those of the
  // i-th head.  Workgroups go to the rank_units compute
  // units in turn, so where each gets two at most the second ones come from the
  // shortest on, and a unit with a long one has a short one beside it.
  __device__ __forceinline__ bool by_length(const AttnParams& p, int head0, int k) {
    const int lane = threadIdx.x & 63, log_tile = __builtin_ctz(p.row_tile);
    int n = p.kv_tokens, queries = p.q_tokens, tiles = 0, low = 0;
    if (lane < p.rank_heads) {
      const int b = (int)fdiv(head0 + p.rank_step * lane, p.div_heads);
      if (p.kv_len) n = min(max(p.kv_len[b], 0), n);
      if (p.q_len) queries = min(max(p.q_len[b], 0), queries);
      tiles = (queries * p.group + p.row_tile - 1) >> log_tile;
      const int64_t at = p.causal ? ((int64_t)max(n - queries, 0) * p.group) >> log_tile
                                  : (int64_t)(n >> log_tile) * p.row_tiles;
      low = (int)min(at, (int64_t)kMostLevels);
    }
    // how many start at x or later
    auto from = [&](int x) { return wave_total(min(max(low + tiles - x, 0), tiles)); };
    const int all = from(0);
    if (k >= all) return false;
    if (all <= 2 * p.rank_units && k >= p.rank_units) k = all - 1 - (k - p.rank_units);
    int x = 0, end = p.levels - 1;
    while (x < end) {
      const int mid = (x + end) >> 1;
      if (from(mid + 1) <= k) end = mid;
      else x = mid + 1;
    }
    k -= from(x + 1);
    const bool has = low <= x && x < low + tiles;
    const int before = __popcll(__ballot(has) & ((uint64_t(1) << lane) - 1));
    const int i = __builtin_ctzll(__ballot(has && before == k)), head = head0 + p.rank_step * i;
    item.b = (int)fdiv(head, p.div_heads);
    item.h = head - item.b * p.kv_heads;
    item.n = __builtin_amdgcn_readlane(n, i);
    const int ql = __builtin_amdgcn_readlane(queries, i), rt = x - __builtin_amdgcn_readlane(low, i);
    item.rows = ql * p.group;
    item.p0 = item.n - ql;
    index = head * p.row_tiles + (p.row_tiles - 1 - rt);
    split = 0;
    item.tile(p, rt);
    steps(p);
    return true;
  }
  // false: nothing to do
  __device__ __forceinline__ bool find(const AttnParams& p, int block) {
    // Workgroups go to the eight XCDs, which have an L2 each, in turn.  Heads
    // are dealt to them likewise where that comes out even, so that a head's
    // keys are read into one L2 and the sequences of a ragged batch are spread
    // over all.
    if (p.rank_heads) return p.by_xcd ? by_length(p, block & 7, block >> 3) : by_length(p, 0, block);
    if (p.by_xcd) {
      const int j = block >> 3, head = (int)fdiv(j, p.div_head), of = p.row_tiles * p.splits;
      block = ((block & 7) + 8 * head) * of + (j - head * of);
    }
    index = (int)fdiv(block, p.div_splits);
    split = block - index * p.splits;
    const int x = (int)fdiv(index, p.div_tiles), b = (int)fdiv(x, p.div_heads);
    item.sequence(p, b);
    item.h = x - b * p.kv_heads;
    // row tiles from the last: with a causal mask the longest start first
    if (!item.tile(p, p.row_tiles - 1 - (index - x * p.row_tiles))) return false;
    steps(p);
    return split < shares;
  }
  __device__ __forceinline__ bool whole() const { return shares == 1; }
  __device__ __forceinline__ float* slot(const AttnParams& p, int head_dim) const {
    return p.ws + ((int64_t)index * p.splits + split) * (p.row_tile * (head_dim + 2));
  }
};

}  // namespace fluid
