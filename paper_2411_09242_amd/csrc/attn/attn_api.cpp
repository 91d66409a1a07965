// Entry points of fluid_attention.h: argument checks and launch sizes.
#include "fluid_attention.h"

#include <algorithm>
#include <cstdint>

#include "../host/handles.h"
#include "../host/kparams.h"
#include "backend.h"
#include "check_tokens.h"

namespace fluid {

namespace {

int64_t block_bytes(const fluid_kv_cache* c) { return int64_t(5) * c->head_dim * c->page_tokens / 4; }

KvArgs check_cache(const fluid_kv_cache* c) {
  require(c != nullptr, "cache: NULL description");
  require(c->n_pages >= 1 && c->kv_heads >= 1 && c->batch >= 1 && c->max_pages >= 1,
          "cache: n_pages, kv_heads, batch and max_pages must be at least 1");
  check_head_dim(c->head_dim);
  int log = 5;
  while (log < 10 && (1 << log) != c->page_tokens) ++log;
  require((1 << log) == c->page_tokens, "cache: page_tokens must be a power of two, 32 .. 1024");
  require(int64_t(c->max_pages) * c->page_tokens <= kMostTokens, "cache: a table row names more than 2^30 tokens");
  require(c->table_stride >= c->max_pages && c->table_stride <= (int64_t(1) << 40), "cache: table_stride below max_pages");
  KvArgs a{};
  a.table_stride = c->table_stride;
  a.block = block_bytes(c);
  a.n_pages = c->n_pages;
  a.log_page = log;
  a.kv_heads = c->kv_heads;
  a.capacity = c->max_pages * c->page_tokens;
  return a;
}
KvArgs check_pool(const fluid_kv_cache* c, const void* pool, const int32_t* pages) {
  KvArgs a = check_cache(c);
  require(pool != nullptr && pages != nullptr, "cache: NULL pool or page table");
  require((uintptr_t)pool % 16 == 0, "cache: the pool must be 16-byte aligned");
  a.pool = (uint8_t*)const_cast<void*>(pool);
  a.pages = pages;
  return a;
}

void kv_io(const fluid_kv_cache* cache, const void* pool, const int32_t* pages, const fluid_tokens* kd, const void* k,
           const fluid_tokens* vd, const void* v, const int32_t* start, const int32_t* count, void* stream, bool write) {
  KvIoParams p{};
  p.c = check_pool(cache, pool, pages);
  p.k = tokens_data(kd, k, "k");
  p.v = tokens_data(vd, v, "v");
  require(start != nullptr, "start: NULL");
  require(kd->dtype == vd->dtype && kd->tokens == vd->tokens, "k and v must have one dtype and as many tokens");
  for (const fluid_tokens* d : {kd, vd})
    require(d->batch == cache->batch && d->heads == cache->kv_heads && d->head_dim == cache->head_dim,
            "k and v must have the cache's batch, kv_heads and head_dim");
  if (!write) {
    check_apart(kd, "k");
    check_apart(vd, "v");
  }
  p.start = start;
  p.count = count;
  p.tokens = kd->tokens;
  const int span = write ? 8 : kKvTile;
  p.runs = (kd->tokens + span - 2) / span + 1;
  p.items = product({cache->batch, p.runs, cache->kv_heads});  // a wavefront each
  require(p.items <= kMostThreads / 64 - 3, "k, v: too large for one launch");  // four to a workgroup
  p.div_heads = make_fastdiv(cache->kv_heads);
  p.div_runs = make_fastdiv(p.runs);
  run_kv_io(p, kd->dtype, cache->head_dim, write, stream);
}

// How an attention is cut into workgroups: items (a tile of rows of one kv
// head) times splits, which share the item's steps (tiles of tokens): as many
// as make `slots` workgroups in all, the number that the GPU runs at once, but
// shares of at least `least` steps.
void plan_shares(AttnParams& p, int64_t visible, int64_t slots, int64_t least) {
  p.row_tiles = (int32_t)((int64_t(p.q_tokens) * p.group + p.row_tile - 1) / p.row_tile);
  const int64_t items = product({p.batch, p.kv_heads, p.row_tiles});
  require(items <= kMostThreads / 64 && product({p.batch, p.kv_heads, p.q_tokens, p.group}) < int64_t(1) << 31,
          "q: too large for one launch");
  const int64_t steps = visible / p.token_tile + 1;
  // a row's shares are put together by one workgroup: 507 of them took 4 us more than 254
  const int64_t splits = std::max<int64_t>(1, std::min({slots / items, steps / least, (int64_t)256}));
  p.chunk = (int32_t)((steps + splits - 1) / splits);
  p.splits = (int32_t)((steps + p.chunk - 1) / p.chunk);
  p.div_group = make_fastdiv(p.group);
  p.div_tiles = make_fastdiv(p.row_tiles);
  p.div_heads = make_fastdiv(p.kv_heads);
  p.div_splits = make_fastdiv(p.splits);
}
void check_launch(const AttnParams& p, int threads) {
  require(product({p.batch, p.kv_heads, p.row_tiles, p.splits, threads}) <= kMostThreads, "q: too large for one launch");
}
uint64_t workspace_of(const AttnParams& p, int head_dim) {
  return p.splits == 1 ? 0 : uint64_t(p.batch) * p.kv_heads * p.row_tiles * p.splits * p.row_tile * (head_dim + 2) * 4;
}
void set_workspace(AttnParams& p, int head_dim, void* ws, uint64_t bytes) {
  const uint64_t need = workspace_of(p, head_dim);
  if (need == 0) return;
  if (ws == nullptr || bytes < need)
    fail(FLUID_E_ARENA_TOO_SMALL, "workspace: " + std::to_string(need) + " bytes needed, " +
                                      std::to_string(ws ? bytes : 0) + " given");
  require((uintptr_t)ws % 256 == 0, "workspace: must be 256-byte aligned");
  p.ws = (float*)ws;
}

AttnParams check_opts(const fluid_attention_opts* o, const fluid_tokens* qd, int kv_heads) {
  require(o != nullptr, "opts: NULL");
  // times log2(e) it still is a number; a NaN fails both
  require(o->scale > 0.0f && o->scale <= 0x1p127f, "opts: scale must be positive and at most 2^127");
  require(o->causal == 0 || o->causal == 1, "opts: causal must be 0 or 1");
  require(o->window >= 0 && o->sinks >= 0, "opts: window and sinks must not be negative");
  require(qd->heads % kv_heads == 0, "q: heads must be a multiple of kv_heads");
  AttnParams p{};
  p.batch = qd->batch;
  p.q_tokens = qd->tokens;
  p.kv_heads = kv_heads;
  p.group = qd->heads / kv_heads;
  require(int64_t(p.q_tokens) * p.group <= kMostTokens, "q: more than 2^30 rows to a kv head");
  p.causal = o->causal;
  p.window = (int32_t)std::min<int64_t>(o->window, kMostTokens);
  p.sinks = o->sinks;
  p.cs = o->scale * 1.4426950408889634f;
  return p;
}
void check_out(const fluid_tokens* qd, const fluid_tokens* od) {
  require(od->dtype == qd->dtype && od->batch == qd->batch && od->tokens == qd->tokens && od->heads == qd->heads &&
              od->head_dim == qd->head_dim,
          "out must have q's dtype and shape");
}
// Tokens that a tile of rows can see, of `most`.
int64_t visible_of(const AttnParams& p, int64_t most, int64_t queries) {
  if (p.window == 0) return most;
  return std::min(most, int64_t(p.window) * (p.causal ? 1 : 2) + queries + p.sinks);
}

// kv_max bounds the split alone; a cache that proves longer is shared in
// larger chunks.
AttnParams plan_kv_attention(const fluid_kv_cache* cache, const fluid_attention_opts* opts, int32_t kv_max,
                             const fluid_tokens* qd) {
  AttnParams p = check_opts(opts, qd, cache->kv_heads);
  require(opts->causal == 1, "opts: attention over the cache is causal");
  require(kv_max >= 1, "kv_max must be at least 1");
  require(qd->batch == cache->batch && qd->head_dim == cache->head_dim, "q must have the cache's batch and head_dim");
  p.kv_tokens = cache->max_pages * cache->page_tokens;
  p.row_tile = int64_t(p.q_tokens) * p.group <= 16 ? 16 : 32;
  p.token_tile = kKvTile;
  const int64_t visible =
      visible_of(p, std::min(kv_max, p.kv_tokens), std::min(p.q_tokens, p.row_tile / p.group + 1));
  // one round of the three workgroups that fit a compute unit: 131072 tokens of
  // 8 heads take 42.8 us with 768 workgroups, 47.1 with twice and 53.7 with
  // three times as many; 16 sequences of 1000 tokens and 32 heads 18.5 us with
  // 512 and 24.9 with 1024.  With 32 rows to a workgroup two fit, and one is as
  // fast (16000 tokens of 16 heads, 16 rows each: 20.7 us, 23.5 with two).
  plan_shares(p, visible, p.row_tile == 16 ? 768 : 256, 8);
  p.waves = 4;
  // Few tokens are left to one larger workgroup, which saves the join: up to
  // four steps to a wavefront.  1024 tokens of 32 heads of 128: 9.7 us in one
  // launch, 12.5 in two; 2048 tokens 15.1 and 12.0.
  const int many = kv_waves(qd->head_dim);
  if (p.row_tile == 16 && p.splits > 1 && visible / p.token_tile < 4 * many) {
    plan_shares(p, visible, 1, 1);
    p.waves = many;
  }
  check_launch(p, 64 * p.waves);
  return p;
}
AttnParams plan_attention(const fluid_attention_opts* opts, const fluid_tokens* qd, const fluid_tokens* kd) {
  AttnParams p = check_opts(opts, qd, kd->heads);
  require(qd->dtype == kd->dtype && qd->batch == kd->batch && qd->head_dim == kd->head_dim,
          "q and k must have one dtype, batch and head_dim");
  p.kv_tokens = kd->tokens;
  p.row_tile = 128;
  p.token_tile = qd->dtype == FLUID_BF16 ? kBf16Tile : kF32Tile;
  const int64_t visible = visible_of(p, p.kv_tokens, std::min(p.q_tokens, p.row_tile / p.group + 1));
  // One round of workgroups, one to a compute unit.  512 queries of 32 heads
  // behind 7680 tokens, bf16: 121 us in 128 workgroups, 80 in 256 or 512, 91 in
  // 1024; 64 queries behind 4032: 64 us in 16, 19 in 256, 23 in 512; fp32: 437,
  // 48 and 60.  A short loop is not worth a second launch: bf16, 512 queries of
  // 12 heads over 512 tokens 11.2 us in one, 13.3 in two; fp32, 4 x 130 tokens
  // of 8 heads 13.0 and 15.4 (4 x 180: 14.2 and 13.9; 512 of 12 heads 28.5 and 18.3).
  const bool bf16 = qd->dtype == FLUID_BF16, brief = visible <= (bf16 ? 512 : 160);
  plan_shares(p, visible, brief ? 1 : 256, 2);
  // Two teams where that still is one round of workgroups, but not to join a
  // single step, or two short ones, of 32 tokens: 16 bf16 tokens of 8 heads 6.5 us
  // with one team, 7.8 with two; 100 tokens (two steps) 7.8 and 7.3; fp32, a
  // query each over 50 tokens 8.1 and 8.5.  fp32 with 128 channels has no room
  // for a second team's stages.
  const int64_t heads = int64_t(p.batch) * p.kv_heads, groups = heads * p.row_tiles * p.splits;
  p.teams = groups <= 256 && p.chunk > (bf16 ? 1 : 2) && (bf16 || qd->head_dim < 128) ? 2 : 1;
  p.by_xcd = heads % 8 == 0;
  // More than one workgroup to a compute unit: the longest rows first, whatever
  // their head, where a wavefront's lanes can hold an XCD's heads, or all of
  // them where they are not dealt to XCDs.  2048 causal queries of 32 heads of
  // 128 take 55.0 us, head after head 65.1; of 64 heads 94.9 and 117.2; 8192 of
  // 32 heads 554 and 558, 4096 of 12 heads 90.6 and 113; 16 ragged sequences of
  // up to 700 tokens 50.7 and 55.2, of up to 500 in both directions 20.5 and 28.7.
  p.rank_step = p.by_xcd ? 8 : 1;
  p.rank_units = p.by_xcd ? 32 : 256;
  const int64_t places = int64_t(p.kv_tokens) * (p.causal ? p.group : p.row_tiles) / p.row_tile;
  p.levels = (int32_t)std::min<int64_t>(places, kMostLevels) + p.row_tiles + 1;
  if (p.splits == 1 && groups > 256 && heads / p.rank_step <= 64) p.rank_heads = (int32_t)(heads / p.rank_step);
  p.div_head = make_fastdiv(p.row_tiles * p.splits);
  check_launch(p, 256 * p.teams);
  return p;
}

}  // namespace

}  // namespace fluid

using namespace fluid;

extern "C" {

fluid_status fluid_kv_pool_bytes(const fluid_kv_cache* cache, uint64_t* bytes) {
  return call_guarded([&] {
    check_cache(cache);
    require(bytes != nullptr, "bytes: NULL");
    const int64_t n = product({cache->n_pages, cache->kv_heads, block_bytes(cache)});
    require(n < int64_t(1) << 62, "cache: too large");
    *bytes = n;
  });
}

fluid_status fluid_kv_write(const fluid_kv_cache* cache, void* pool, const int32_t* pages, const fluid_tokens* kd,
                            const void* k, const fluid_tokens* vd, const void* v, const int32_t* start,
                            const int32_t* count, void* hip_stream) {
  return call_guarded([&] { kv_io(cache, pool, pages, kd, k, vd, v, start, count, hip_stream, true); });
}

fluid_status fluid_kv_read(const fluid_kv_cache* cache, const void* pool, const int32_t* pages, const fluid_tokens* kd,
                           void* k, const fluid_tokens* vd, void* v, const int32_t* start, const int32_t* count,
                           void* hip_stream) {
  return call_guarded([&] { kv_io(cache, pool, pages, kd, k, vd, v, start, count, hip_stream, false); });
}

fluid_status fluid_kv_attention_workspace(const fluid_kv_cache* cache, const fluid_attention_opts* opts,
                                          int32_t kv_max, const fluid_tokens* qd, uint64_t* bytes) {
  return call_guarded([&] {
    check_cache(cache);
    tokens_arg(qd, nullptr, "q");
    require(bytes != nullptr, "bytes: NULL");
    *bytes = workspace_of(plan_kv_attention(cache, opts, kv_max, qd), cache->head_dim);
  });
}

fluid_status fluid_kv_attention(const fluid_kv_cache* cache, const void* pool, const int32_t* pages,
                                const fluid_attention_opts* opts, int32_t kv_max, const fluid_tokens* qd,
                                const void* q, const int32_t* q_len, const int32_t* kv_len, const fluid_tokens* od,
                                void* out, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  return call_guarded([&] {
    const KvArgs c = check_pool(cache, pool, pages);
    const TokensArg qa = tokens_data(qd, q, "q"), oa = tokens_data(od, out, "out");
    check_out(qd, od);
    require(kv_len != nullptr, "kv_len: NULL");
    AttnParams p = plan_kv_attention(cache, opts, kv_max, qd);
    check_apart(od, "out");
    p.c = c;
    p.q = qa;
    p.o = oa;
    p.q_len = q_len;
    p.kv_len = kv_len;
    set_workspace(p, cache->head_dim, workspace, workspace_bytes);
    run_kv_attention(p, qd->dtype, cache->head_dim, hip_stream);
  });
}

fluid_status fluid_attention_workspace(const fluid_attention_opts* opts, const fluid_tokens* qd,
                                       const fluid_tokens* kd, uint64_t* bytes) {
  return call_guarded([&] {
    tokens_arg(qd, nullptr, "q");
    tokens_arg(kd, nullptr, "k");
    require(bytes != nullptr, "bytes: NULL");
    *bytes = workspace_of(plan_attention(opts, qd, kd), qd->head_dim);
  });
}

fluid_status fluid_attention(const fluid_attention_opts* opts, const fluid_tokens* qd, const void* q,
                             const fluid_tokens* kd, const void* k, const fluid_tokens* vd, const void* v,
                             const int32_t* q_len, const int32_t* kv_len, const fluid_tokens* od, void* out,
                             void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  return call_guarded([&] {
    const TokensArg qa = tokens_data(qd, q, "q"), ka = tokens_data(kd, k, "k"), va = tokens_data(vd, v, "v"),
                    oa = tokens_data(od, out, "out");
    check_out(qd, od);
    require(kd->dtype == vd->dtype && kd->batch == vd->batch && kd->tokens == vd->tokens && kd->heads == vd->heads &&
                kd->head_dim == vd->head_dim,
            "k and v must have one dtype and shape");
    AttnParams p = plan_attention(opts, qd, kd);
    check_apart(od, "out");
    p.q = qa;
    p.k = ka;
    p.v = va;
    p.o = oa;
    p.q_len = q_len;
    p.kv_len = kv_len;
    set_workspace(p, qd->head_dim, workspace, workspace_bytes);
    run_attention(p, qd->dtype, qd->head_dim, hip_stream);
  });
}

}  // extern "C"
