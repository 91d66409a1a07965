// Launch parameters of the cache and attention kernels (host and device).
#pragma once

#include <stdint.h>

#include "../host/kparams.h"

namespace fluid {

// A tensor of tokens: base and strides in elements; vec: every row starts on
// a 16-byte address.
struct TokensArg {
  void* p;
  int64_t sb, st, sh;
  int32_t vec;
};

struct KvArgs {
  uint8_t* pool;
  const int32_t* pages;
  int64_t table_stride;
  int64_t block;  // bytes of one page of one kv head
  int32_t n_pages, log_page, kv_heads;
  int32_t capacity;  // tokens a row of the table can name
};

struct KvIoParams {
  KvArgs c;
  TokensArg k, v;
  const int32_t* start;
  const int32_t* count;
  int32_t tokens;
  int32_t runs;    // runs of 8 (write) or 32 (read) tokens that T rows at any start can touch
  int64_t items;   // batch * runs * kv_heads, a wavefront each
  FastDiv div_heads, div_runs;
};

// Rows are the (query, head of the group) pairs of one kv head, query slowest.
struct AttnParams {
  KvArgs c;        // kv_attention only
  TokensArg q, k, v, o;
  const int32_t* q_len;
  const int32_t* kv_len;
  int32_t batch, q_tokens, kv_tokens, kv_heads, group;
  int32_t causal, window, sinks;
  float cs;          // scale * log2(e)
  int32_t row_tile, token_tile;  // rows and tokens of a workgroup's step
  int32_t row_tiles;             // tiles of rows of one kv head
  int32_t waves;   // kv_attention: wavefronts of a workgroup
  int32_t teams;   // attention: teams of four wavefronts to a workgroup
  int32_t splits;  // most shares of an item, a workgroup each
  int32_t chunk;   // steps of a share
  FastDiv div_group, div_tiles, div_heads, div_splits;
  int32_t by_xcd;     // 1: a kv head's workgroups on one XCD
  int32_t rank_heads;  // > 0: row tiles from the longest on, of so many heads together
  int32_t rank_step, rank_units;  // from one of the heads to the next; compute units they have
  int32_t levels;      // past the last place that a row tile can start at
  FastDiv div_head;   // by a kv head's workgroups
  float* ws;       // splits > 1: [item][split] of row_tile maxima, sums and rows of partial sums
};

// Queries and keys (the second ones, if any) turned by their positions.
struct RotaryParams {
  TokensArg x[2], y[2];
  int32_t heads[2];
  const uint64_t* turns;
  const int32_t* start;
  const int32_t* positions;
  int64_t position_stride;
  const int32_t* count;
  int32_t batch, tokens, head_dim, dim;
  int32_t interleaved, inverse, tail;  // tail: channels behind dim are copied
  float amplitude;
  int32_t vec;           // channels at a time, a power of two, 16 bytes of them at most
  int32_t units, pairs;  // of a head: in all, of turned ones
  int32_t head_threads;  // that share a token's heads
  uint32_t items;        // threads
  FastDiv div_units, div_heads, div_tokens;
};

// Linear attention: a state per kv head.
struct LinearParams {
  TokensArg q, k, v, o;
  const float* decay;
  int64_t gb, gt, gh;
  const float* state;  // may be state_out
  float* state_out;
  const int32_t* count;
  int32_t batch, tokens, kv_heads, group;
  float scale;
  FastDiv div_heads;
  int32_t segments;  // runs of tokens that workgroups of their own take; 0: token after token
  int32_t run;       // tokens of a run, whole chunks
  int32_t slots;     // 1: a first launch leaves states in ws
  int32_t scan;      // 1: a launch between them makes the runs' first states
  float* ws;         // [kv head][run] states, then what runs keep of one
};

// tokens of a chunk of linear attention
constexpr int linear_chunk(int dtype) { return dtype == DT_BF16 ? 64 : 32; }

// tokens of a step over the 4-bit cache, and over bf16 and fp32 keys and values
constexpr int kKvTile = 32, kBf16Tile = 64, kF32Tile = 32;

// Bound on the places, in row tiles, by which long rows are told from short ones.
constexpr int kMostLevels = 1 << 24;

// Wavefronts of a workgroup that has an item's tokens to itself: as many as the
// registers of a compute unit hold.
constexpr int kv_waves(int head_dim) { return head_dim == 128 ? 8 : 16; }

}  // namespace fluid
