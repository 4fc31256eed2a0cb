/*
 * rmsnorm.h — the root-mean-square norm between a model's layers on MI355X (gfx950):
 * with the residual's addition, its backward pass, and its output in 8 bits.
 *
 *     h = x + residual              rounded once to the residual's type, and kept
 *     rstd = 1 / sqrt(mean(h^2) + eps)
 *     y = h rstd (weight + weight_offset)
 *
 * Conventions are those of norms.h: device pointers to contiguous row-major [N, M]
 * matrices, work on `stream`, argument errors before anything is enqueued, attn_status
 * return codes, the same bits for the same call.  X, weight and Y have one type (norm_dtype);
 * the residual, H and the gradients dH have that type or fp32 (stream_dtype).  N >= 1, 1 <= M
 * <= RMSNORM_MAX_M, N * M < 2^40; rows need no alignment.  weight NULL: y = h rstd.  residual
 * NULL: h = x, H is not written (and may be NULL), stream_dtype is that of X.  In place: Y may be X itself, H the residual, dX
 * dY or a dH of its type, and dresidual dH; otherwise what is written shares memory with nothing else.  rstd is fp32 and y
 * and the gradients are formed with it: under 2^-126 it has fewer bits (rows of a root mean square over 2^126), and rows under 2^-128 with
 * an eps of 0 have an infinite one (the 8-bit form takes its own, in 64 bits).
 */
#ifndef RMSNORM_H
#define RMSNORM_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>
#include "attn.h"
#include "norms.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RMSNORM_MAX_M 32768

typedef enum {
  QUANT8_E4M3 = 0, /* 4 exponent bits, 3 of mantissa, up to 448, no infinities */
  QUANT8_INT8 = 1  /* -127 .. 127 */
} quant8_code;

/*
 * Y [N, M], H [N, M] and rstd [N] (fp32; may be NULL).  Squares are summed in 64 bits.
 * Errors: ATTN_ERR_NULL, ATTN_ERR_SHAPE (sizes, eps negative or not finite, offset not finite, overlaps),
 * ATTN_ERR_UNSUPPORTED (types).
 */
int rmsnorm_add(const void* X, const void* residual, const void* weight, void* Y, void* H, float* rstd, int N, int M,
                double eps, float weight_offset, norm_dtype dtype, norm_dtype stream_dtype, hipStream_t stream);

/*
 * The same with y in 8 bits: codes [N, M] (one byte each) and scales [N, groups] (fp32), y ~ code * scale.
 *
 *   group   elements that share a scale: 0 for the whole row (groups = 1), or 32, 64, 128 or
 *           256 (groups = ceil(M / group), the last one may be short)
 *
 * With a the largest |y| of a group, its scale is a / 448 (E4M3) or a / 127 (INT8), rounded to fp32, and a
 * code is y / scale rounded to the nearest, ties to even.  y and the quotient are formed in 64 bits, so a code is that of the
 * definition.  A group of zeros has scale 0; one with an infinity or NaN has scale NaN and
 * codes 0.  rstd [N] may be NULL.
 * Errors: as rmsnorm_add; ATTN_ERR_SHAPE (group), ATTN_ERR_UNSUPPORTED (code).
 */
int rmsnorm_add_quant(const void* X, const void* residual, const void* weight, void* codes, float* scales, void* H,
                      float* rstd, int N, int M, int group, quant8_code code, double eps, float weight_offset,
                      norm_dtype dtype, norm_dtype stream_dtype, hipStream_t stream);

/*
 * Y [N, M] = code * scale, formed in fp32 and rounded to dtype: what rows in 8 bits stand for.  group as
 * above.  Errors as rmsnorm_add_quant.
 */
int quant8_load(const void* codes, const float* scales, void* Y, int N, int M, int group, quant8_code code,
                norm_dtype dtype, hipStream_t stream);

/*
 * Gradients of rmsnorm_add.  With g = dY (weight + weight_offset) and n = H rstd:
 *
 *     d = dH + rstd (g - n mean(g n))         the gradient of h: of x and of the residual alike
 *     dweight = sum over the rows of dY n
 *
 *   dY         [N, M] of dtype
 *   H, rstd    as rmsnorm_add left them (without a residual, H is X)
 *   dH         [N, M] of stream_dtype: the gradient that reaches h past the norm, or NULL for none
 *   dX         [N, M] of dtype: d
 *   dresidual  [N, M] of stream_dtype: d; NULL where stream_dtype is dtype (dX serves both), or if not wanted
 *   dweight    [M] fp32, or NULL if not wanted
 *   workspace  at least rmsnorm_add_bwd_workspace_bytes(N, M) bytes, 16-byte aligned, used until the call's kernels
 *              end; may be NULL without dweight
 *
 * Errors: as rmsnorm_add; ATTN_ERR_WORKSPACE.
 */
size_t rmsnorm_add_bwd_workspace_bytes(int N, int M);
int rmsnorm_add_bwd(const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX,
                    void* dresidual, float* dweight, int N, int M, float weight_offset, void* workspace,
                    size_t workspace_bytes, norm_dtype dtype, norm_dtype stream_dtype, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RMSNORM_H */
