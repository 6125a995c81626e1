/*
 * block_attn.h -- C ABI of attention over selected blocks and over an 8-bit cache (gfx950).
 *
 * Where tile_attn.h takes a fixed frame mask from the host, here the kept tiles follow the data
 * and stay on the device. Keys and queries are cut into blocks of TA_BLOCK tokens. A cheap score
 * (the product of a query block's mean with a key block's mean) chooses which key blocks each
 * query block attends to (block_attn_means, block_attn_lists), attention and its gradients run
 * over the chosen blocks only (block_attn_fwd, block_attn_bwd), and a program that generates
 * token after token keeps its keys and values in 8 bits, TA_BLOCK tokens a page
 * (cache_attn_write, cache_attn_fwd).
 *
 * Conventions shared by all entry points (beside those of tile_attn.h on types, streams and
 * errors, which hold here too: bf16 tensors, contiguous, 16-byte aligned, fp32 accumulation,
 * argument errors found before any HIP call, a finite scale of any sign):
 *   - Heads are grouped: H query heads, Hkv key heads, H a multiple of Hkv; query head h reads
 *     key head h / G with G = H / Hkv.
 *   - The Sq query rows of a sequence are its last Sq positions: row r sits at position
 *     Skv - Sq + r, 1 <= Sq <= Skv. Query blocks are cut at row 0, key blocks at position 0;
 *     NQ = ceil(Sq / TA_BLOCK), NB = ceil(Skv / TA_BLOCK) <= TA_MAX_BLOCKS. Skv - Sq is the same
 *     for all sequences of a call, whatever their lens: single tokens of sequences of different
 *     lengths take a call for each (cache_attn_fwd takes them together).
 *   - lens: DEVICE int32 [B], 4-byte aligned, or NULL for Skv everywhere. Positions from lens[b]
 *     on are padding: their keys count for nobody, whatever they hold, and their query rows give
 *     zeros, a log-sum-exp of -inf and zero gradients. Values are taken into 0..Skv.
 *   - causal: nonzero lets a row attend only to positions up to its own.
 *   - For given lists a row's result depends on the tokens it attends to alone: infinities and NaN
 *     elsewhere, in later tokens too, do not reach it. A row that meets a NaN has NaN for its
 *     log-sum-exp. For gradients this holds between query blocks only: a key or value that is no
 *     number may reach its own gradients and those of all rows of a query block that lists it, and a
 *     row that is no number those of all keys of the blocks it lists. A row whose log-sum-exp is NaN
 *     gives NaN to dv of the keys it attends to, and to no other dv.
 *   - Logits scale * <q, k> up to 2^29 in magnitude: past that the rounding of a row's maximum in
 *     fp32 leaves the exponent's range, and rows may come out as zeros or NaN. The log-sum-exp is
 *     fp32 too, so weights in the gradients are off by up to 2^-23 of the logit's magnitude.
 *   - lists: DEVICE int32 [B, Hkv, NQ, n_list], 1 <= n_list <= TA_MAX_BLOCKS, the blocks a query
 *     block's rows (of all G heads) attend to, in any order. Entries outside 0..NB-1 are skipped
 *     (-1 fills up), and a block that is listed twice counts once.
 *   - Nothing is allocated and nothing is kept between calls. What a call needs beside its tensors
 *     the caller hands in: workspace, DEVICE memory of at least the bytes that the entry's
 *     ..._workspace function gives for the same sizes, 16-byte aligned (NULL if that is 0), used
 *     only by the work that the call enqueues. Its contents matter neither before nor after.
 *     Calls that may run at the same time, graphs replayed at the same time among them, need
 *     workspaces of their own.
 *   - The tensors belong to the current device. Every call may be captured into a graph.
 *   - Results do not depend on how work was scheduled: the same call gives the same bits.
 */
#ifndef BLOCK_ATTN_H
#define BLOCK_ATTN_H

#include <stddef.h>
#include <stdint.h>

#include "tile_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TA_BLOCK 128       /* tokens of a block, and of a page of the cache */
#define TA_MAX_BLOCKS 16384

/*
 * Means of key blocks: means[b, h, j, :] = the mean of x[b, h, t, :] over the valid tokens t of
 * block j, rounded once to bf16 (sums in 64 bits); zeros for a block without valid tokens.
 * x: bf16 [B, H, S, d]; means: bf16 [B, H, ceil(S / TA_BLOCK), d].
 * A program that decodes calls this for a block when its last token is there.
 */
int block_attn_means(const void* x, void* means, int B, int H, int S, int d, const int32_t* lens,
                     void* stream);

/*
 * The lists. A query block's mean (over its valid rows of all G heads, rounded to bf16) is
 * multiplied with the means of the key blocks, in 64 bits; scores do not depend on the scale.
 * Of the blocks that hold a position some row may attend to, a list takes first the forced ones
 * (the first `sink` blocks, and where local >= 1 the blocks that the rows themselves lie in, with
 * local - 1 more before them and, if not causal, behind them), then those of the highest scores,
 * n_list in all, equal scores by the lower index; a score that is NaN counts as the lowest. The
 * list is ascending, -1 behind its end. The rows of a query block share one list, chosen by the mean
 * of them all: with causal too, which blocks an early row attends to depends on rows up to
 * TA_BLOCK - 1 later (no row attends to a later token). So a model trained with the lists of whole
 * query blocks sees its choice made by later tokens, and decodes (Sq = 1) by the token's own.
 * q: bf16 [B, H, Sq, d]; kmeans: bf16 [B, Hkv, NB, d] (block_attn_means of the keys).
 * Errors: TA_ERR_BAD_SHAPE also where n_list may not hold the forced blocks.
 */
int block_attn_lists(const void* q, const void* kmeans, int32_t* lists, int B, int H, int Hkv,
                     int Sq, int Skv, int d, int n_list, int sink, int local, int causal,
                     const int32_t* lens, void* stream);

/*
 * Attention over the lists: out[r] = sum_t softmax_t(scale * <q[r], k[t]>) v[t] over the tokens t
 * of the listed blocks that the row may attend to; a row with none gives zeros.
 * q, out: bf16 [B, H, Sq, d]; k, v: bf16 [B, Hkv, Skv, d]; lse: fp32 [B, H, Sq], natural
 * logarithm, -inf for a row with no token, or NULL. d is 64, 96 or 128.
 */
int block_attn_fwd_workspace(int B, int H, int Hkv, int Sq, int Skv, int d, int n_list, size_t* bytes);
int block_attn_fwd(const void* q, const void* k, const void* v, const int32_t* lists, void* out,
                   float* lse, int B, int H, int Hkv, int Sq, int Skv, int d, int n_list, int causal,
                   const int32_t* lens, float scale, void* workspace, size_t workspace_bytes,
                   void* stream);

/*
 * Gradients of block_attn_fwd for the same lists, order, lengths and scale; out and lse are what
 * it returned, dout the gradient of out. dk and dv sum over the G heads that share a key head.
 * dq: bf16 [B, H, Sq, d]; dk, dv: bf16 [B, Hkv, Skv, d], fully written: zeros for blocks nobody
 * lists and for padding. The lists get no gradient.
 */
int block_attn_bwd_workspace(int B, int H, int Hkv, int Sq, int Skv, int d, int n_list, size_t* bytes);
int block_attn_bwd(const void* q, const void* k, const void* v, const int32_t* lists, const void* out,
                   const void* dout, const float* lse, void* dq, void* dk, void* dv, int B, int H,
                   int Hkv, int Sq, int Skv, int d, int n_list, int causal, const int32_t* lens,
                   float scale, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The 8-bit cache. k_pages: e4m3 codes [n_pages, Hkv, TA_BLOCK, d], v_pages: [n_pages, Hkv, d,
 * TA_BLOCK] (values transposed inside a page: the matrix cores then read them as they lie), both
 * 16-byte aligned; k_scales, v_scales: fp32 [n_pages, Hkv]; a number is code * scale.
 * table: int32 [B, max_pages], page i of a sequence holding its tokens 128 i .. 128 i + 127;
 * lens: int32 [B]; B * Hkv is at most 65535. An entry outside 0..n_pages-1 names no page: its
 * tokens are neither written nor read. Sequences may share pages that no call writes.
 *
 * cache_attn_write puts N new tokens behind the lens[b] tokens a sequence holds (lens itself is
 * left as it is; tokens past max_pages pages are dropped). With n_new (int32 [B], or NULL) a
 * sequence takes the first n_new[b] of its N. Scales are powers of two: of the tokens that go
 * into a page, the least 2^e (-100 <= e <= 120) with which the largest finite magnitude is at
 * most 448; a page that holds tokens already keeps the larger of its scale and that, and its old
 * codes are rounded again where the scale grew. Rounding is to nearest, ties to even; infinities
 * become the largest code, NaN stays NaN. Tokens behind the last one are left as they were.
 * k, v: bf16 [B, Hkv, N, d]. A page that is written belongs to one sequence and stands once in its
 * row of the table.
 */
int cache_attn_write(const void* k, const void* v, void* k_pages, void* v_pages, float* k_scales,
                     float* v_scales, const int32_t* table, const int32_t* lens, const int32_t* n_new,
                     int B, int Hkv, int N, int d, int max_pages, int n_pages, void* stream);

/*
 * Attention of the last N tokens of each sequence over its pages; lens counts them too. Row t
 * attends to the first lens[b] - (N - 1) + t tokens; a row with none gives zeros and -inf.
 * q, out: bf16 [B, H, N, d], H / Hkv * N at most 524280; lse: fp32 [B, H, N] or NULL. Lengths may
 * be anything from 0 to max_pages pages (longer ones are taken as that). Scales may be any finite
 * numbers here.
 * With per_head nonzero table is [B, Hkv, max_pages] and lens [B, Hkv]: every key head has pages
 * of its own choice, as the lists of a single token give them. A list that keeps the page of the
 * last token as its last entry, all others full, then needs no more than its own length.
 */
int cache_attn_fwd_workspace(int B, int H, int Hkv, int N, int d, int max_pages, size_t* bytes);
int cache_attn_fwd(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                   const float* v_scales, const int32_t* table, const int32_t* lens, int per_head,
                   void* out, float* lse, int B, int H, int Hkv, int N, int d, int max_pages,
                   int n_pages, float scale, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BLOCK_ATTN_H */
