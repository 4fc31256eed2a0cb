/*
 * attn_bwd.h — attention in training on MI355X (gfx950): the forward pass that keeps
 * each row's log-sum-exp, and the backward pass that recomputes the
 * probabilities from it.
 *
 * With s = mod(scale Q K^T) + bias, masked entries -inf (attn.h; mod is SoftCap or
 * nothing), and lse_i = log sum_j exp(s_ij):
 *
 *     P  = exp(s - lse)              O = P V
 *     dV = P^T dO
 *     dS = P (dO V^T - delta) mod'(scale Q K^T) scale,    delta_i = dO_i . O_i
 *     dQ = dS K                      dK = dS^T Q
 *
 * dK and dV of a KV head are summed over its query heads.  ALiBi's slopes count as
 * constants: they get no gradient.
 *
 * Conventions are those of attn.h (layouts, head groups, masks, return codes): device
 * pointers, work on `stream`, argument errors before anything is enqueued, no atomics and
 * so the same bits for the same call.  Sums are held in fp32.  The probabilities
 * and dS go to the matrix unit in the type of Q, for dQ dS as two values of it.  A row that sees no
 * key (causal, Lq > Lk) has O = 0, lse = -inf and dQ = 0, and its dO is not read.  softcap is at most
 * ATTN_TRAIN_MAX_SOFTCAP: a capped score is off by 2^-22 of the cap, which the backward pass
 * takes into an exponential.
 */
#ifndef ATTN_BWD_H
#define ATTN_BWD_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>
#include "attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ATTN_TRAIN_MAX_SOFTCAP 1024.0f

/*
 * attn_fwd_mod that also writes lse [B, Hq, Lq] (fp32, natural units).  The sums of
 * exponentials are those before their rounding to the type of Q (attn_fwd's are of
 * the rounded ones), so O may differ from attn_fwd's in the last bit.  One kernel, at any Lq (the keys of
 * few rows are not divided over workgroups).  Q, K, V and O are 16-byte aligned.
 * Errors: as attn_fwd_mod; ATTN_ERR_NULL (lse), ATTN_ERR_SHAPE for outputs that share memory with another
 * operand and for tensors that are not aligned, ATTN_ERR_UNSUPPORTED for a softcap over ATTN_TRAIN_MAX_SOFTCAP.
 */
int attn_fwd_lse(const void* Q, const void* K, const void* V, void* O, float* lse,
                 int B, int Hq, int Hkv, int Lq, int Lk, int D,
                 int causal, float scale, const float* alibi_slopes, float softcap, int window,
                 attn_dtype dtype, hipStream_t stream);

/* Bytes of attn_bwd's workspace; 0 for invalid sizes.  Depends on the current device's compute units. */
size_t attn_bwd_workspace_bytes(int B, int Hq, int Hkv, int Lq, int Lk, int D, int causal, int window);

/*
 * The gradients of Q, K and V from that of O.
 *
 *   dO         [B, Hq, Lq, D] with do_strides (three HOST values: elements between
 *              batches, heads and rows, >= 0; the dims of a row are contiguous): a view of
 *              [B, Lq, Hq, D] is taken as it is
 *   O, lse     attn_fwd_lse's of the same Q, K, V and arguments
 *   dQ, dK, dV written whole, as Q, K, V are laid out; they and the workspace share memory with
 *              nothing else that the call is given
 *   workspace  at least attn_bwd_workspace_bytes(...) bytes, 16-byte aligned, used until the
 *              call's kernels end
 *
 * Every tensor of 16-bit values is 16-byte aligned and dO's strides are multiples of
 * 8.  (Lq + 32) * D * 2, (Lk + 32) * D * 2, Lq + 32 times dO's row stride in bytes and (Lq + 32) * 8 * Hq / Hkv
 * stay below 2^31.  A product with 0 of an infinity or NaN is NaN: one in a row of Q, K, V or dO reaches the
 * rows and keys that share a tile of 32 with it, masked from it or not (attn_fwd's O alike).
 * Errors: as attn_fwd_lse; ATTN_ERR_WORKSPACE.
 */
int attn_bwd(const void* dO, const long long* do_strides, const void* Q, const void* K, const void* V, const void* O,
             const float* lse, void* dQ, void* dK, void* dV,
             int B, int Hq, int Hkv, int Lq, int Lk, int D,
             int causal, float scale, const float* alibi_slopes, float softcap, int window,
             void* workspace, size_t workspace_bytes, attn_dtype dtype, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_BWD_H */
