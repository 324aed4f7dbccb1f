/*
 * moa_paged.h -- a paged key/value cache in bf16: appending new tokens with the norm
 * of their heads and the rotation by position on the way, and the attention over
 * it, with or without a sliding window.  The conventions (device pointers,
 * streams, status codes, no allocation, no synchronisation, checks before any HIP
 * call) are those of moa_attn.h.
 *
 * THE CACHE is two pools of pages of bf16, K and V, logical shape [num_pages][Hk]
 * [page][d], with element strides (page, head, row) or NULL: contiguous.  The
 * strides are non-negative multiples of 16 bytes, of rows at most 2^25 elements;
 * the pools may be views of one buffer.  `page` is a power of two, 16 to 2^20.
 * Nothing in a page needs to be set before tokens are written to it.
 *
 * ADDRESSING, the same for both entry points.  Sequence b has seq_lens[b] tokens,
 * the new ones of the call included and last.  page_table [B][max_pages] holds the
 * page of tokens 0..page-1, page..2 page-1, and so on of every sequence; NULL:
 * sequence b has page b alone (then max_pages is 1 and num_pages >= B).  A call
 * brings up to N new tokens per sequence: new_lens[b] (clamped to 0..N) of them,
 * or N where new_lens is NULL.  Row i < new_lens[b] of a [B][H][N][d] tensor is token
 * seq_lens[b] - new_lens[b] + i; rows behind are not read and left as they are.
 * seq_lens, new_lens and page_table are int32 device arrays whose values the host
 * does not see: tokens before 0, behind the capacity max_pages * page, or on a page
 * outside 0..num_pages-1 are skipped (not written, not visible).  So a window's
 * caller may give pages that it has left behind to other sequences and put -1 into
 * the table.  Pages may be shared by sequences that only read them.
 */
#ifndef MOA_PAGED_H
#define MOA_PAGED_H

#include "moa_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * moa_paged_append -- new tokens into the cache.  Every head row of Q and K is normed
 * (where there is a weight) and turned by its token's position, exactly as
 * moa_qk_norm_rope does, and rounded to bf16 once: Q's into Qo, K's into k_pool; V's
 * rows go into v_pool as they are, rounded to bf16.
 *
 * Q, K, V   device inputs of storage type dtype (MOA_F32 or MOA_BF16), logical shapes
 *           [B][Hq][N][d], [B][Hk][N][d] and [B][Hk][N][d].  Input rows may overlap.
 * Qo        device output, bf16, [B][Hq][N][d].  May be Q (bf16, same pointer and
 *           strides: in place).
 * k_pool, v_pool
 *           the cache, written: 16-byte aligned, no element of the two twice.
 * wq, wk    norm weights [d] of storage type w_dtype, or NULL: no norm.
 * positions device int64 [axes][B][N], any values, or NULL: every token's place in its
 *           sequence, seq_lens[b] - new_lens[b] + i, on every axis.
 * inv_freq, rot, axes, sections, interleaved, eps
 *           as for moa_qk_norm_rope (rot = 0: no rotation).
 * B, Hq, Hk, N, d, page, num_pages, max_pages
 *           all may be 0 but d and page; supported: d in {64, 128}, max_pages * page
 *           <= 2^30, num_pages < 2^30, B * N < 2^27, Hq + Hk < 2^30, B * N * (Hq + 2 Hk) <
 *           2^31.
 * *_strides element strides (batch, head, row), of the pools (page, head, row), or
 *           NULL: contiguous.  Non-negative multiples of 16 bytes.
 *
 * Two rows of one call must not be the same token of the same page (which one stays
 * is then undefined).  Qo and the inputs may be views that interleave in one buffer
 * of bf16 (heads of a packed projection output), and so may the two pools, where
 * their rows or their batches (pages) take turns in it; nothing else may overlap.
 * Queries of skipped tokens are turned all the same.  One kernel; deterministic.
 */
int moa_paged_append(const void* Q, const void* K, const void* V, void* Qo, void* k_pool,
                     void* v_pool, const void* wq, const void* wk, const int64_t* positions,
                     const float* inv_freq, const int32_t* seq_lens, const int32_t* new_lens,
                     const int32_t* page_table, int64_t B, int64_t Hq, int64_t Hk, int64_t N,
                     int64_t d, int64_t rot, int64_t page, int64_t num_pages, int64_t max_pages,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* v_strides,
                     const int64_t* qo_strides, const int64_t* k_pool_strides,
                     const int64_t* v_pool_strides, int axes, const int64_t* sections,
                     int interleaved, float eps, int dtype, int w_dtype, void* stream);

/*
 * moa_paged_attn_num_splits, moa_paged_attn_workspace_bytes -- the key splits that a
 * moa_paged_attn_fwd call with these arguments uses, and the device workspace it
 * then needs in bytes (0 when it does not split).  num_splits: 0 = the library's
 * choice, else 1..256.  max_len: the most tokens a sequence has (0: the capacity);
 * it only guides the choice.
 */
int moa_paged_attn_num_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page,
                              int64_t max_pages, int64_t max_len, int64_t left, int64_t right,
                              int64_t sinks, int num_splits);
size_t moa_paged_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d,
                                      int64_t page, int64_t max_pages, int64_t max_len,
                                      int64_t left, int64_t right, int64_t sinks, int num_splits);

/*
 * moa_paged_attn_fwd -- attention of new queries over the cache.  Query i of sequence
 * b stands at its token's position, p = seq_lens[b] - new_lens[b] + i, and sees the
 * tokens j of the cache, 0 <= j < seq_lens[b], with j <= p + right and (j >= p - left or
 * j < sinks), as moa_window.h says: right = 0 is the causal mask, left = w - 1 a
 * window of w tokens, negative values no limit.  The rows' own keys and values have
 * to be in the cache before (moa_paged_append on the same stream).
 *
 * Q         device input, bf16, logical shape [B][Hq][N][d], element strides (batch,
 *           head, row) or NULL; non-negative multiples of 16 bytes.
 * k_pool, v_pool
 *           the cache, only read: 16-byte aligned.
 * O, LSE    as for moa_win_attn_fwd, [B][Hq][N][d] and [B][Hq][N].
 * B, Hq, Hk, N, d, page, num_pages, max_pages
 *           B, N, Hq >= 0, Hq a multiple of Hk; supported: d in {64, 128}, max_pages *
 *           page <= 2^30, B * Hq * N < 2^26 (with num_splits of 2 and more 2^26 - 4 at
 *           most), and fewer than 2^24 workgroups (of 16, 32 or 128 rows of one
 *           key/value head and one split).
 * max_len   as above.  Any value is right; a good one is fast.
 * scale, out_dtype, workspace, workspace_bytes, num_splits
 *           as for moa_win_attn_fwd, whose computation this is.
 * A row without a visible token gets O = 0 and LSE = -inf.  Unset tokens, and what
 * the pages of other sequences hold, do not touch rows that do not see them.
 */
int moa_paged_attn_fwd(const void* Q, const void* k_pool, const void* v_pool, void* O, float* LSE,
                       const int32_t* seq_lens, const int32_t* new_lens, const int32_t* page_table,
                       int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page,
                       int64_t num_pages, int64_t max_pages, int64_t max_len,
                       const int64_t* q_strides, const int64_t* k_strides,
                       const int64_t* v_strides, const int64_t* o_strides, int64_t left,
                       int64_t right, int64_t sinks, float scale, int out_dtype, void* workspace,
                       size_t workspace_bytes, int num_splits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOA_PAGED_H */
