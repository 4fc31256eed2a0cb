/*
 * rope.h — rotary positions for queries and keys on MI355X (gfx950).
 *
 * Dims 0 .. rotary_dim - 1 of every head row are rotated in pairs by the row's
 * position p; the dims behind them are copied.  With freqs[i] in radians per
 * position, t = p * freqs[i], c = magnitude * cos(t), s = magnitude * sin(t):
 *
 *     y_a = c x_a - s x_b        y_b = s x_a + c x_b
 *
 * for the pair (a, b) = (i, i + rotary_dim / 2), or (2 i, 2 i + 1) with
 * interleaved != 0, i < rotary_dim / 2.  The gradient of the inputs is the
 * transposed rotation (rope_bwd):
 *
 *     dx_a = c dy_a + s dy_b     dx_b = -s dy_a + c dy_b
 *
 * t is formed and reduced to a fraction of a turn in 64 bits, off by 3.3e-16 of
 * it: 8e-7 radians at position 2^31 and a frequency of 1, 4e-4 at 2^40.  The rest is
 * 32-bit arithmetic, rounded to the element type once.
 *
 * Conventions are those of attn.h: device pointers, work on `stream`, argument
 * errors before anything is enqueued, attn_status return codes, deterministic.
 */
#ifndef ROPE_H
#define ROPE_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ROPE_F16 = 0,
  ROPE_BF16 = 1,
  ROPE_F32 = 2
} rope_dtype;

/* Frequencies for contexts longer than the trained one; f = base^(-2 i / rotary_dim). */
typedef enum {
  ROPE_PLAIN = 0,    /* f */
  ROPE_LINEAR = 1,   /* f / factor: positions interpolated */
  ROPE_BASE = 2,     /* base * factor^(rotary_dim / (rotary_dim - 2)) in place of base: the slowest pair is
                        interpolated by factor, the fastest not at all */
  ROPE_PARTS = 3     /* f w + (f / factor)(1 - w), w = clamp((n - slow) / (fast - slow), 0, 1) of the n =
                        original_length f / (2 pi) turns that the pair makes over the trained context */
} rope_scaling;

/*
 * The rotary_dim / 2 frequencies in radians per position, to HOST memory (a
 * program uploads them once).  rotary_dim even, >= 2 (ROPE_BASE: >= 4); base
 * > 0; factor > 0 except ROPE_PLAIN; ROPE_PARTS: original_length > 0 and 0 <=
 * slow < fast.  Errors: ATTN_ERR_NULL, ATTN_ERR_SHAPE for the sizes and
 * non-finite values (a base or frequency that 64 bits do not hold among them),
 * ATTN_ERR_UNSUPPORTED for another scaling.
 */
int rope_frequencies(int rotary_dim, double base, int scaling, double factor, double original_length, double slow,
                     double fast, double* freqs);

/*
 * Rotate the queries and keys of B sequences of L tokens in one kernel.
 *
 *   Q, K   [B, Hq, L, D] and [B, Hkv, L, D] with q_strides and k_strides (three
 *          HOST values each: elements between batches, heads and tokens; the
 *          dims of a row are contiguous), so that a view of a projection's
 *          [B, L, H, D] needs no copy.  K NULL (with Hkv 0): queries alone.
 *   Qo, Ko contiguous [B, H, L, D].  Qo may be Q itself, and Ko K, if those are
 *          contiguous; no other overlap.
 *   positions  device int (positions_bits 32) or long long (64) values, of any
 *          sign: token l of sequence b is at positions[b * positions_stride + l]
 *          (positions_stride 0: the same positions for every sequence).
 *   freqs  device double[rotary_dim / 2]; rotary_dim even, 2 .. D, any D.
 *
 * Rows whose size, strides and addresses are multiples of 16 (or 8) bytes, with
 * pairs that fill such vectors, are read and written in vectors, others by
 * elements.
 * B * L * D < 2^31 and Hq + Hkv < 2^16.
 * Errors: ATTN_ERR_NULL; ATTN_ERR_SHAPE for bad sizes, a non-finite magnitude
 * or positions_bits; ATTN_ERR_UNSUPPORTED for the dtype; ATTN_ERR_HIP.
 */
int rope_fwd(const void* Q, const long long* q_strides, void* Qo, int Hq,
             const void* K, const long long* k_strides, void* Ko, int Hkv,
             int B, int L, int D, const void* positions, int positions_bits, long long positions_stride,
             const double* freqs, int rotary_dim, int interleaved, float magnitude, rope_dtype dtype,
             hipStream_t stream);

/* The gradient of rope_fwd's inputs from that of its outputs: dQ and dK in place of Q and K, the same arguments. */
int rope_bwd(const void* dQ, const long long* q_strides, void* dQo, int Hq,
             const void* dK, const long long* k_strides, void* dKo, int Hkv,
             int B, int L, int D, const void* positions, int positions_bits, long long positions_stride,
             const double* freqs, int rotary_dim, int interleaved, float magnitude, rope_dtype dtype,
             hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ROPE_H */
