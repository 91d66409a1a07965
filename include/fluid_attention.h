/*
 * fluid_attention.h -- token-by-token generation next to the planned graphs
 * of fluid.h: a paged key/value cache held in 4 bits, the attention that
 * reads it, and attention over ordinary keys and values with a sliding window
 * and a few first tokens that stay visible.
 *
 * Conventions are those of fluid.h: every call returns a fluid_status and
 * nothing throws across the ABI (fluid_last_error() has the cause), arguments
 * are validated before any HIP call, all device memory (pool, tensors, page
 * table, lengths, workspace) is the caller's, nothing is allocated, and a
 * call only enqueues kernels on `hip_stream`, so it can be captured in a HIP
 * graph.  The calling thread's current device has to be the stream's and the
 * memory's.  Nothing is kept between calls.  The host-only library validates
 * alike and then returns FLUID_E_UNSUPPORTED.
 *
 * Tensors of tokens are [batch, tokens, heads, head_dim] with any strides and
 * contiguous channels (fluid_tokens).  Lengths, starts and page tables are
 * int32 in device memory, read when the kernels run; what they hold cannot be
 * refused, so each declaration says what out-of-range values do.
 */
#ifndef FLUID_ATTENTION_H
#define FLUID_ATTENTION_H

#include "fluid.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A tensor of tokens.  Channels are contiguous; stride holds the distance in
 * elements between sequences, tokens and heads (not negative; 0 repeats an
 * input; an output's are at least head_dim, and its elements must not
 * overlap).  head_dim is 32, 64 or 128; batch, tokens and heads are at least 1
 * (a sequence's own lengths may be 0).  Rows that start on 16-byte addresses
 * are fastest; others are read and written element by element. */
typedef struct {
  int32_t dtype; /* FLUID_F32 or FLUID_BF16 */
  int32_t batch, tokens, heads, head_dim;
  int64_t stride[3];
} fluid_tokens;

/* Geometry of a paged cache.
 *
 * Every group of 32 channels of one token is held as 32 nibbles n and a pair
 * of float16 (s, b); nibble n stands for f16(b + s (16 + n)), rounded once.
 * With c = x clamped to [-16384, 16384], lo and hi the group's least and
 * largest c:
 *     s = f16((hi - lo) / 15)   b = f16(lo - 16 s)
 *     n = s > 0 ? clamp(rint((c - b) / s) - 16, 0, 15) : 0
 * in fp32, ties to even.  A group that holds an infinity or a NaN reads back
 * as NaN in all its 32 channels.  Groups whose values are all below 2^-14
 * lose precision with the float16 pair.  Values of pairs made so are within
 * float16; attention may take a group whose values at nibbles 0 and 15 are not
 * for NaN.  The pool need not be cleared: no call uses what was not written,
 * but for tokens that a length says are there.
 *
 * pool: [n_pages][kv_heads][block], block = 5 * head_dim * page_tokens / 4
 * bytes, 16-byte aligned.  A block holds page_tokens P of one kv head, with
 * G = head_dim / 32 (32-bit little-endian words):
 *     K nibbles  P rows of head_dim / 8 words: word o * G + j holds channels
 *                32 j + 8 o .. +7 of the token
 *     K pairs    P rows of G words: s in the low half, b in the high half
 *     V nibbles  P / 8 rows of head_dim words: word d holds channel d of
 *                8 consecutive tokens
 *     V pairs    P / 8 rows of G times (8 float16 s, 8 float16 b)
 * element e of a word is its nibble (e >> 1) + 4 (e & 1).
 *
 * pages: int32 [batch][max_pages], rows table_stride apart: the page that
 * holds tokens i * page_tokens .. of the sequence.  An entry outside
 * [0, n_pages) holds no tokens: nothing is written to it, kv_read leaves its
 * rows as they are and attention does not see its tokens.  So a page that a
 * window has left behind can be given back.  Sequences may share pages that
 * are only read; a page that a call writes to must be in one row alone. */
typedef struct {
  int32_t n_pages, page_tokens; /* page_tokens: 32, 64, 128, 256, 512 or 1024 */
  int32_t kv_heads, head_dim;   /* head_dim: 32, 64 or 128 */
  int32_t batch, max_pages;
  int64_t table_stride; /* >= max_pages */
} fluid_kv_cache;

/* Which tokens a query sees, and the factor on q . k.  The query of row i of
 * a sequence sits at position p = kv_len - q_len + i; it sees the tokens
 * j < kv_len with
 *     j <= p                              if causal
 *     |p - j| < window  or  j < sinks     if window > 0
 * A row that sees no token gets zeros, and so does one whose scores are all
 * minus infinity.  A token that a row does not see contributes nothing to it,
 * whatever its key and value hold.  Scores times log2(e) are held in fp32: past
 * 2.3e38 a score is infinite. */
typedef struct {
  float scale; /* positive, at most 2^127 */
  int32_t causal;
  int32_t window; /* 0: none */
  int32_t sinks;  /* first tokens that stay visible beside the window */
} fluid_attention_opts;

/* Bytes of the cache's pool.  Errors: FLUID_E_INVALID (geometry). */
fluid_status fluid_kv_pool_bytes(const fluid_kv_cache* cache, uint64_t* bytes);

/* Quantise tokens k, v [batch, T, kv_heads, head_dim] into the cache.  Row i
 * of sequence b becomes token start[b] + i for i < min(count[b], T); count
 * NULL writes all T rows.  Positions past the table's row, or negative, are
 * left out.  Tokens beside the written ones keep their values, also where
 * they share a word with them.  Errors: FLUID_E_INVALID (NULL argument but
 * count, geometry, shapes or dtypes that disagree, misaligned pool). */
fluid_status fluid_kv_write(const fluid_kv_cache* cache, void* pool, const int32_t* pages, const fluid_tokens* kd,
                            const void* k, const fluid_tokens* vd, const void* v, const int32_t* start,
                            const int32_t* count, void* hip_stream);

/* The values of tokens start[b] .. start[b] + min(count[b], T) - 1 into rows
 * 0 .. of k, v; other rows are left as they are.  count NULL: T.  Errors as
 * fluid_kv_write. */
fluid_status fluid_kv_read(const fluid_kv_cache* cache, const void* pool, const int32_t* pages, const fluid_tokens* kd,
                           void* k, const fluid_tokens* vd, void* v, const int32_t* start, const int32_t* count,
                           void* hip_stream);

/* Attention of q [batch, T, heads, head_dim] over the cache, heads a multiple
 * of kv_heads (query head h reads kv head h / (heads / kv_heads)), out of q's
 * shape and dtype; opts->causal must be 1.  Sequence b has q_len[b] queries
 * (NULL: T; clamped to [0, T]) and kv_len[b] tokens (clamped to [0, the
 * table's row]), its newest being the queries' own.  Rows from q_len[b] on
 * are left as they are.  kv_max: the largest kv_len the caller expects
 * (>= 1); it sizes the split of long caches over the GPU.  Results are right for
 * any kv_len, but the split is in equal shares of kv_max: caches far shorter are
 * shared by few workgroups, and slower than with a kv_max near their length.
 * workspace: 256-byte aligned device memory of at least the bytes
 * fluid_kv_attention_workspace returns for the same arguments (0: NULL will do),
 * for this call alone while it runs.  Arithmetic: products on the f16 matrix
 * cores with fp32 sums, softmax in fp32.  bf16: a query's channels below 2^-14 of
 * its largest are rounded to 2^-25 of that, and a weight to f16 (11 bits) for its
 * product with the value.  fp32: queries and weights are two f16 parts each,
 * within 2^-22 of themselves and queries within 2^-25 of the row's largest: up to
 * four times an fp32 rounding.  Errors: FLUID_E_INVALID; FLUID_E_ARENA_TOO_SMALL
 * (workspace). */
fluid_status fluid_kv_attention_workspace(const fluid_kv_cache* cache, const fluid_attention_opts* opts,
                                          int32_t kv_max, const fluid_tokens* qd, uint64_t* bytes);
fluid_status fluid_kv_attention(const fluid_kv_cache* cache, const void* pool, const int32_t* pages,
                                const fluid_attention_opts* opts, int32_t kv_max, const fluid_tokens* qd,
                                const void* q, const int32_t* q_len, const int32_t* kv_len, const fluid_tokens* od,
                                void* out, void* workspace, uint64_t workspace_bytes, void* hip_stream);

/* Attention of q [batch, T, heads, head_dim] over k, v [batch, N, kv_heads,
 * head_dim], all of one dtype.  Lengths as above (NULL: T and N; kv_len is
 * clamped to [0, N]); rows of k and v from kv_len[b] on are not used.
 * Arithmetic: on the bf16 matrix cores with fp32 sums, softmax in fp32.  bf16:
 * a weight is rounded to bf16 for its product with the value, and so summed.
 * fp32: operands are three bf16 parts each, which leaves the error of an fp32
 * product; a row's sums run before their division, with weights of up to 2^8, and
 * overflow to infinity for values near fp32's largest.  Workspace and errors as
 * fluid_kv_attention. */
fluid_status fluid_attention_workspace(const fluid_attention_opts* opts, const fluid_tokens* qd,
                                       const fluid_tokens* kd, uint64_t* bytes);
fluid_status fluid_attention(const fluid_attention_opts* opts, const fluid_tokens* qd, const void* q,
                             const fluid_tokens* kd, const void* k, const fluid_tokens* vd, const void* v,
                             const int32_t* q_len, const int32_t* kv_len, const fluid_tokens* od, void* out,
                             void* workspace, uint64_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FLUID_ATTENTION_H */
