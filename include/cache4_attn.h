/*
 * cache4_attn.h -- C ABI of the cache in 4 bits (gfx950): writing it, reading it back, attention over it.
 *
 * Beside the 8-bit cache of block_attn.h, whose conventions hold here (grouped heads, page tables, lengths,
 * workspaces, errors, streams), at 17 bits for 32 (K, V) values of 2 * 8 there: half the memory, half the bytes a
 * decoding step reads. A page holds TA_BLOCK tokens of every key head, K and V laid out alike:
 *   k_pages, v_pages    codes [n_pages, Hkv, TA_BLOCK, d / 2], 16-byte aligned: value e of a token in byte e / 2, even
 *                       ones in its low half. A code is e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 for 0..7, bit 3 the sign.
 *   k_scales, v_scales  bytes [n_pages, Hkv, d / 32, TA_BLOCK], 16-byte aligned: the exponent of every 32 values of a
 *                       token, biased by 127; a number is code * 2^(byte - 127). 255 stands for NaN.
 * Scales are a token's own, so writing a token never touches another one's.
 */
#ifndef CACHE4_ATTN_H
#define CACHE4_ATTN_H

#include <stddef.h>
#include <stdint.h>

#include "block_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TA_CACHE4_GROUP 32 /* values of a token that share a scale */

/*
 * Puts N new tokens behind the lens[b] tokens that a sequence holds; lens, n_new, table, pages that are none and
 * tokens past the table as for cache_attn_write. A group's scale is the least 2^e, -100 <= e <= 125, with which its
 * largest magnitude is at most 7 (6 is the largest code, and 7 is as far from it as rounding takes any number
 * between 4 and 6); codes are the nearest, ties to the even one. Infinities and NaN are left out of a group's
 * magnitude and stored as 0, and the token is marked: all its K scales are 255, so that its key reads back as NaN
 * and a row that attends to it comes out as NaN. (A V scale is never 255.) N is at most 2^28 - 256, here and in reading.
 * k, v: bf16 [B, Hkv, N, d]. k_held, v_held: bf16 of the same shape, or NULL: the numbers that the cache now holds
 * for these tokens (zeros for those that were not written), for a prompt's own attention.
 */
int cache4_attn_write(const void* k, const void* v, void* k_pages, void* v_pages, void* k_scales, void* v_scales,
                      const int32_t* table, const int32_t* lens, const int32_t* n_new, void* k_held, void* v_held,
                      int B, int Hkv, int N, int d, int max_pages, int n_pages, void* stream);

/*
 * Tokens first .. first + N - 1 of every sequence as bf16 [B, Hkv, N, d], exactly; zeros from lens[b] on and for
 * tokens whose page is none. k_out or v_out may be NULL, not both. first + N is at most 2^31 - 1.
 */
int cache4_attn_read(const void* k_pages, const void* v_pages, const void* k_scales, const void* v_scales,
                     const int32_t* table, const int32_t* lens, void* k_out, void* v_out, int B, int Hkv, int N, int d,
                     int max_pages, int n_pages, int first, void* stream);

/*
 * Attention of the last N tokens of each sequence over its pages, as cache_attn_fwd (per_head among it). V scales
 * above 252 in a page that is attended to may make all its rows NaN. Logits scale * <q, k> may be up to 2^126 in magnitude; a
 * logit is a number of fp32, and weights are off by up to 2^-23 of its magnitude, as the log-sum-exp is.
 */
int cache4_attn_fwd_workspace(int B, int H, int Hkv, int N, int d, int max_pages, size_t* bytes);
int cache4_attn_fwd(const void* q, const void* k_pages, const void* v_pages, const void* k_scales,
                    const void* v_scales, const int32_t* table, const int32_t* lens, int per_head, void* out,
                    float* lse, int B, int H, int Hkv, int N, int d, int max_pages, int n_pages, float scale,
                    void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CACHE4_ATTN_H */
