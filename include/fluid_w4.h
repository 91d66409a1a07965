/*
 * fluid_w4.h -- products with matrices held in 4 bits, for the few rows of a
 * decode step: beside the planned graphs of fluid.h, whose matrices are fp32 or
 * bf16.
 *
 * Conventions are those of fluid_attention.h: every call returns a fluid_status
 * (fluid_last_error() has the cause), arguments are validated before any HIP
 * call, all device memory is the caller's, nothing is allocated or kept, and a
 * call only enqueues kernels on `hip_stream`, so it can be captured in a HIP
 * graph.  The calling thread's current device has to be the stream's and the
 * memory's.  The host-only library validates alike and then returns
 * FLUID_E_UNSUPPORTED.
 */
#ifndef FLUID_W4_H
#define FLUID_W4_H

#include "fluid.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A matrix [rows, cols] held in 4 bits, `rows` being a product's outputs and
 * `cols` what it sums over.
 *
 * Every run of `group` channels of a row (the last one may be shorter) has 4-bit
 * levels n and a pair of float16 (s, b); n stands for b + s (16 + n).  With c = w
 * clamped to [-16384, 16384], lo and hi the group's least and largest c:
 *     s = f16((hi - lo) / 15)   b = f16(lo - 16 s)
 *     n = s > 0 ? clamp(rint((c - b) / s) - 16, 0, 15) : 0
 * in fp32, ties to even, as the cache of fluid_attention.h holds its values.  A
 * group that holds an infinity or a NaN is (0, NaN).  Groups whose values are all
 * below 2^-14 lose precision with the float16 pair.
 *
 * Memory, 16-byte aligned: for every 16 rows and, within them, every 128
 * channels (the last ones padded) 64 x 4 32-bit words; word j of place 16 g + r
 * holds channels 32 j + 8 g .. + 7 of row r, element e at nibble (e >> 1) +
 * 4 (e & 1).  Behind all of them, for the same tiles, 16 rows x 128 / group words,
 * s in the low half and b in the high.  What pads is zero. */
typedef struct {
  int32_t rows, cols;
  int32_t group; /* 32, 64 or 128 */
} fluid_w4;

/* Rows of values with contiguous channels, `stride` elements apart (not
 * negative; 0 repeats an input's row; an output's is at least cols). */
typedef struct {
  int32_t dtype; /* FLUID_F32 or FLUID_BF16 */
  int32_t rows, cols;
  int64_t stride;
} fluid_matrix;

/* Bytes of the matrix.  Errors: FLUID_E_INVALID. */
fluid_status fluid_w4_bytes(const fluid_w4* w, uint64_t* bytes);

/* The matrix m (w's rows and cols) into 4 bits, and back.  Errors:
 * FLUID_E_INVALID. */
fluid_status fluid_w4_pack(const fluid_w4* w, const fluid_matrix* md, const void* m, void* packed, void* hip_stream);
fluid_status fluid_w4_read(const fluid_w4* w, const void* packed, const fluid_matrix* md, void* m, void* hip_stream);

/* out = x W^T, or SiLU(x G^T) * (x W^T) with a gate G of W's geometry, plus add
 * if there is one: x [M, cols], add and out [M, rows] of one dtype.  gate, add
 * (with ad): NULL for none.  out may be add itself with the same stride, and must
 * not overlap x, nor add in any other way.  Made for few rows: every 64 of them read
 * the matrix again.  workspace: 256-byte aligned device memory of at least the bytes
 * that fluid_w4_matmul_workspace returns for x (0: NULL will do), for this call alone
 * while it runs.
 * Arithmetic: x times 16 + n on the bf16 matrix cores (fp32: n - 8, and x in three
 * bf16 parts, exact to 2^-23), fp32 sums over a group, which s and b then enter in
 * fp32; one rounding at the end.  A row of x that is not finite, or whose sums
 * times 31 pass fp32, gives NaN or infinities in that row alone.  Errors:
 * FLUID_E_INVALID; FLUID_E_ARENA_TOO_SMALL (workspace). */
fluid_status fluid_w4_matmul_workspace(const fluid_w4* w, const fluid_matrix* xd, int32_t gated, uint64_t* bytes);
fluid_status fluid_w4_matmul(const fluid_w4* w, const void* packed, const void* gate, const fluid_matrix* xd,
                             const void* x, const fluid_matrix* ad, const void* add, const fluid_matrix* od, void* out,
                             void* workspace, uint64_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FLUID_W4_H */
