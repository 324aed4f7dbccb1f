/*
 * moa_kv4.h -- a key/value cache held in four bits: quantising keys and values
 * as they are written, reading them back, and the attention over the cache.
 * The conventions (device pointers, streams, status codes, no allocation, no
 * synchronisation, checks before any HIP call) are those of moa_attn.h.
 *
 * THE FORMAT.  32 successive elements of a row share one power of two
 * 2^(byte - 127); an element is a four-bit float times it: bit 3 the sign, bits
 * 0..2 the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6.  17 bytes for 32 elements.
 * Written blocks have bytes 2..252, or 255: a block that held an infinity or a
 * NaN, all of whose elements read as NaN.  Of a block with largest magnitude a
 * the byte is the smallest of 2..252 for which a <= 7 * 2^(byte - 127) (no
 * element then is off by more than half the widest step; beyond 7 * 2^125 it is
 * 252, and such elements become 6 * 2^125), and every element takes the nearest
 * value, ties to the even code.
 *
 * THE CACHE is a pool of pages, [num_pages][Hk][page_bytes] bytes in one
 * buffer.  A page holds `page` tokens (a multiple of 64) of one key/value head:
 *   key codes     [page][d/2]              byte i: elements 2i (low half), 2i + 1
 *   key scales    [page/64][d/32][16][4]   token 64a + 16t + r at [a][block][r][t]
 *   value codes   [page/4][d/4][4][2]      token 4q + j, elements 4c..4c+3 at [q][c][j]
 *   value scales  [page/64][d/32][4][4][4] token 64a + 16t + 4g + j at [a][block][g][t][j]
 * (the order in which the matrix instructions of the attention take them).
 * Nothing in a page needs to be set before tokens are written to it.
 *
 * ADDRESSING, the same for all entry points.  Sequence b has seq_lens[b] tokens,
 * the new ones of the call included and last.  page_table [B][max_pages] holds
 * the page of tokens 0..page-1, page..2 page-1, and so on of every sequence;
 * NULL: sequence b has page b alone (then max_pages is 1 and num_pages >= B: a
 * cache without pages, of capacity `page`).  A call brings up to N new tokens
 * per sequence: new_lens[b] (clamped to 0..N) of them, or N where new_lens is
 * NULL.  Row i < new_lens[b] of a [B][H][N][d] tensor is token
 * seq_lens[b] - new_lens[b] + i; rows behind are not read and left as they are.
 * seq_lens, new_lens and page_table are int32 device arrays whose values the
 * host does not see: tokens before 0, behind the capacity max_pages * page, or
 * on a page outside 0..num_pages-1 are skipped (not written, not read, not
 * visible).  Pages may be shared by sequences that only read them.
 */
#ifndef MOA_KV4_H
#define MOA_KV4_H

#include "moa_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* moa_kv4_page_bytes -- bytes of one head's page: page * (d + d/16); 0 unless
 * d is 64 or 128 and page a multiple of 64 in 64..2^20. */
size_t moa_kv4_page_bytes(int64_t page, int64_t d);

/*
 * moa_kv4_write -- quantise new keys and values into the cache.
 *
 * K, V      device inputs of storage type in_dtype (MOA_F32 or MOA_BF16),
 *           logical shape [B][Hk][N][d], element strides (batch, head, row) or
 *           NULL: contiguous; non-negative multiples of 16 bytes (ignored for
 *           a dimension of size 1).  Rows may overlap.
 * cache     device pool, written: 16-byte aligned, num_pages * Hk *
 *           moa_kv4_page_bytes(page, d) bytes, overlapping nothing else.
 * seq_lens, new_lens, page_table
 *           as above; new_lens and page_table may be NULL.
 * B, Hk, N, d, page, num_pages, max_pages
 *           B, Hk, N >= 0; supported: d in {64, 128}, page a multiple of 64 up to
 *           2^20, max_pages * page < 2^31, num_pages < 2^31, and
 *           B * Hk * (N + 6) < 2^30; at d = 128 writing and reading take
 *           B * Hk * (N + 6) up to 2^30 - 64.
 * Two rows of one call must not be the same token of the same page (which one
 * stays is then undefined).  One kernel.  Returns MOA_OK once the work is
 * enqueued, or when there are no rows.
 */
int moa_kv4_write(const void* K, const void* V, void* cache, const int32_t* seq_lens,
                  const int32_t* new_lens, const int32_t* page_table, int64_t B, int64_t Hk,
                  int64_t N, int64_t d, int64_t page, int64_t num_pages, int64_t max_pages,
                  const int64_t* k_strides, const int64_t* v_strides, int in_dtype, void* stream);

/*
 * moa_kv4_read -- the reverse: the values that the cache holds for the rows'
 * tokens (exact in bf16 and fp32), into K and V of storage type out_dtype.
 * Rows behind new_lens[b] and rows of skipped tokens are left as they are.  K
 * and V must not write an element twice, and the bytes from the first to the
 * last element of each must not meet the other's or an input's (views that
 * interleave in one buffer do).
 * (new_lens = seq_lens, with N at least the longest, reads whole sequences:
 * token i to row i.)
 */
int moa_kv4_read(const void* cache, void* K, void* V, const int32_t* seq_lens,
                 const int32_t* new_lens, const int32_t* page_table, int64_t B, int64_t Hk,
                 int64_t N, int64_t d, int64_t page, int64_t num_pages, int64_t max_pages,
                 const int64_t* k_strides, const int64_t* v_strides, int out_dtype, void* stream);

/*
 * moa_kv4_attn_num_splits, moa_kv4_attn_workspace_bytes -- the key splits that
 * a moa_kv4_attn_fwd call with these arguments uses, and the device workspace
 * it then needs in bytes (0 when it does not split).  num_splits: 0 = the
 * library's choice, else 1..256.  max_len: the most tokens a sequence has (0:
 * the capacity, max_pages * page); it only guides the choice.
 */
int moa_kv4_attn_num_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page,
                            int64_t max_pages, int64_t max_len, int num_splits);
size_t moa_kv4_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d,
                                    int64_t page, int64_t max_pages, int64_t max_len,
                                    int num_splits);

/*
 * moa_kv4_attn_fwd -- attention of new queries over the cache:
 *
 *   O[b,h,i,:] = sum_j P_ij V_j,   P_i = softmax over visible j of scale * <Q[b,h,i,:], K_j>
 *
 * with the stored keys and values of key/value head h / (Hq/Hk).  Visible are
 * the tokens j < seq_lens[b], and under the causal mask (causal = 1) only those
 * up to row i's own, j <= seq_lens[b] - new_lens[b] + i.  The rows' own keys and
 * values have to be in the cache before (moa_kv4_write on the same stream).
 *
 * Q         device input, bf16, logical shape [B][Hq][N][d], element strides
 *           (batch, head, row) or NULL; non-negative multiples of 16 bytes.
 * cache     device pool, only read.
 * O         device output of storage type out_dtype (MOA_F32 or MOA_BF16), same
 *           logical shape and stride rules; no element written twice, and its
 *           bytes from the first to the last overlapping nothing else.
 * LSE       optional device output, fp32 [B][Hq][N] contiguous: the natural log
 *           of the softmax denominator.  NULL: not written.
 * A row without a visible token gets O = 0 and LSE = -inf.  Rows behind
 * new_lens[b] are left as they are.
 * B, Hq, Hk, N, ...
 *           as for moa_kv4_write, Hq a multiple of Hk; supported:
 *           B * Hq * N < 2^26, and fewer than 2^24 workgroups (of 16 rows of one
 *           key/value head and one key split, or 32 where a head has more).
 * scale     finite, at most 2^127 in size; 0 and negative values are valid.
 * max_len   as above (0: the capacity).  Any value is right; a good one is fast.
 * workspace, workspace_bytes
 *           at least moa_kv4_attn_workspace_bytes(...) bytes, 16-byte aligned,
 *           overlapping nothing (else MOA_ERR_WORKSPACE); NULL/0 when that is 0.
 *
 * Computation: bf16 matrix products with fp32 accumulation of the exact stored
 * values (bf16 holds them); softmax statistics in fp32, from the fp32 weights; a
 * weight multiplies V as the sum of two bf16 numbers, 17 bits.  The sums of up to
 * n visible keys are taken with weights of at most 1 where values are large, so
 * that values below 2^128 / n cannot overflow.  A score whose product with
 * scale * log2(e) leaves fp32 upwards makes its row NaN, one that leaves it
 * downwards weighs nothing, and a row that sees only such is NaN (LSE: infinite,
 * of that sign).  Stored NaN blocks and unset tokens do not touch rows that do
 * not see them.  One kernel, or two when the keys are split; no atomics,
 * deterministic.
 */
int moa_kv4_attn_fwd(const void* Q, const void* cache, void* O, float* LSE, const int32_t* seq_lens,
                     const int32_t* new_lens, const int32_t* page_table, int64_t B, int64_t Hq,
                     int64_t Hk, int64_t N, int64_t d, int64_t page, int64_t num_pages,
                     int64_t max_pages, int64_t max_len, const int64_t* q_strides,
                     const int64_t* o_strides, float scale, int causal, int out_dtype,
                     void* workspace, size_t workspace_bytes, int num_splits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOA_KV4_H */
