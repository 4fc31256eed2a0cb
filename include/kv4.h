/*
 * kv4.h — a paged cache of keys and values held in 4 bits, and decode attention
 * over it, on MI355X (gfx950).
 *
 * Format.  A value is an E2M1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives) times a power of two that it shares with the 31 others of its
 * block: dims 32 j .. 32 j + 31 of one token and head.  The block's scale byte is
 * the exponent plus 127; 255 stands for NaN.  4.25 bits a value.  For a block
 * with largest magnitude a, the exponent is the smallest e with a <= 7 * 2^e (7
 * itself is held as 6), limited to -13 .. 13 for fp16 and -125 .. 125 for bf16, so
 * that every value held is a normal number of the type, or zero; each element is held
 * as the nearest code (ties to the even code, magnitudes over 6 as 6).  A block
 * with an infinity or NaN is held as 32 NaN.  (Read in fp16, a block that was
 * written from larger or smaller bf16 values gives infinities or zeros.)
 *
 * Layout.  cache is [pages, Hkv, kv4_page_bytes(page, D)] bytes, contiguous,
 * 16-byte aligned.  `page` is the tokens of a page, a power of two from 16 to
 * 32768.  The bytes of a page and head: the codes of K [page, D / 2], two to a byte with
 * the lower dim in the lower bits, the codes of V alike, the scale bytes of K
 * [D / 32, page], those of V.  Token t of sequence b is row t % page of page
 * table[b * max_pages + t / page]; its slot is that page * page + that row.
 * (A contiguous cache is one with a table of consecutive pages.)  A table row holds
 * at most 2^30 tokens: max_pages * page <= 2^30.
 *
 * Conventions are those of attn.h: device pointers, work on `stream`, argument
 * errors before anything is enqueued, attn_status return codes.  What the
 * kernels read on the device (lens, counts, table, slots) cannot be refused on
 * the host: lengths are clamped to what the table can hold, a page outside the
 * cache is never read or written, and its tokens count as masked.  What a call
 * on the cache writes (kv4_append: the cache; kv4_load: K and V; attn_decode_kv4:
 * O and the workspace) shares memory with nothing else that it is given, but that O
 * may be Q itself: ATTN_ERR_SHAPE.
 */
#ifndef KV4_H
#define KV4_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>
#include "attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of one page of one head, page * D * 17 / 16; 0 for a page size or D that is not supported. */
size_t kv4_page_bytes(int page, int D);

/*
 * The pages and slots of new tokens: B sequences with lens[b] tokens get
 * counts[b] more (at most L are taken).  Sequence by sequence, in order, the
 * pages that the new tokens need beyond ceil(lens[b] / page) are taken off the
 * front of free_pages and written into the table [B, max_pages]; entries that
 * get no new page stay as they are.  Where the free pages or the table's row
 * run out, the tokens that fit are kept.
 *
 *   slots      [B, L] long long: the slot of token l < stored[b], -1 behind (and
 *              for a token whose page in the table or the list is negative)
 *   positions  [B, L] int: lens[b] + l, for every l
 *   new_lens   [B] int: lens[b] + stored[b]; not lens itself, which other
 *              workgroups still read (refused)
 *   taken      [1] int: pages taken off free_pages
 *
 * lens[b] is clamped to 0 .. max_pages * page.  nfree >= 0; B * max_pages
 * and B * L < 2^31, max_pages * page + L <= 2^31.  One kernel.
 * Errors: ATTN_ERR_NULL (free_pages may be NULL where nfree is 0), ATTN_ERR_SHAPE (sizes, new_lens == lens).
 */
int kv_slots(const int* lens, const int* counts, int* table, const int* free_pages, int nfree, int B, int max_pages,
             int page, int L, long long* slots, int* positions, int* new_lens, int* taken, hipStream_t stream);

/*
 * Round K and V to the cache's format and write them to their slots.
 *
 *   K, V    [B, Hkv, L, D] with k_strides and v_strides (three HOST values each:
 *           elements between batches, heads and tokens; the dims of a row
 *           are contiguous).  Pointers 16-byte aligned, strides multiples of 8.
 *   slots   device long long [B, L], distinct; a slot outside 0 .. pages * page - 1
 *           is skipped (padding).  Slots given twice keep a mixture.
 *   D 64 or 128, dtype fp16 or bf16.  L < 2^28 - 15 (D = 128) or 2^29 - 31, B * L < 2^31,
 *   Hkv < 2^16.
 * Errors: ATTN_ERR_NULL, ATTN_ERR_SHAPE (sizes, page, alignment), ATTN_ERR_UNSUPPORTED.
 */
int kv4_append(const void* K, const long long* k_strides, const void* V, const long long* v_strides, void* cache,
               const long long* slots, int B, int Hkv, int L, int D, int pages, int page, attn_dtype dtype,
               hipStream_t stream);

/*
 * K and V [B, Hkv, L, D] (contiguous) of tokens starts[b] .. starts[b] + L - 1 of
 * each sequence, exactly as held; zeros for tokens at or past lens[b], or in
 * a page that does not exist.  starts NULL: from token 0 (negative: as 0).
 * What attn_fwd takes for the next piece of a prompt: one request (or requests of
 * one length) a call, since it has one Lk and sees every key up to it, zeros too.
 * Errors as kv4_append.
 */
int kv4_load(const void* cache, const int* table, const int* starts, const int* lens, void* K, void* V, int B,
             int Hkv, int L, int D, int pages, int page, int max_pages, attn_dtype dtype, hipStream_t stream);

/*
 * Single-token decode over the cache (split-k update, Section "Split-K Update"):
 *
 *   Q [B, Hq, 1, D], O [B, Hq, 1, D]; the query of sequence b is its token
 *   lens[b] - 1 and sees tokens max(0, lens[b] - window) .. lens[b] - 1
 *   (window 0: all).  scale, alibi_slopes (i = lens[b] - 1) and softcap as
 *   attn_decode_mod; a cap of any size keeps a score to its 32-bit rounding.  A
 *   sequence that sees nothing gives 0.  For several query tokens of one sequence,
 *   pass the sequence's table row once for each, with its own length.
 *
 *   workspace  at least attn_decode_kv4_workspace_bytes(B, Hq, Hkv, D) bytes,
 *              16-byte aligned, used until the call's kernels end.  The size depends on
 *              B, the heads and the current device's compute units, not on the
 *              lengths.
 *
 * lens and table are read while the kernels run, and must not change before
 * they end.  The 32-token tiles of all sequences and KV heads are one list, of which every
 * workgroup takes an equal share, so uneven lengths balance; rows that
 * lie in several shares are joined by a second kernel.
 * B * Hq < 2^24.  The list is counted in 32 bits, with 8 more for each row, for the
 * longest contexts that the table holds whatever lens says: B * Hkv * T *
 * (max_pages * page / 32 + 8) < 2^31, where T is the workgroups of up to 32 query heads
 * that a KV head takes.
 * K . Q and P . V run on the matrix unit in the type of Q with fp32
 * accumulation; a weight of P is the sum of two values of that type.
 * Errors: ATTN_ERR_NULL, ATTN_ERR_SHAPE, ATTN_ERR_UNSUPPORTED, ATTN_ERR_WORKSPACE, ATTN_ERR_HIP.
 */
size_t attn_decode_kv4_workspace_bytes(int B, int Hq, int Hkv, int D);
int attn_decode_kv4(const void* Q, const void* cache, const int* table, const int* lens, void* O, int B, int Hq,
                    int Hkv, int D, int pages, int page, int max_pages, float scale, const float* alibi_slopes,
                    float softcap, int window, void* workspace, size_t workspace_bytes, attn_dtype dtype,
                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* KV4_H */
