/*
 * moa_window.h -- attention in a sliding window with a few first tokens that stay
 * visible, query heads sharing key/value heads, and the gradients.  The
 * conventions (device pointers, streams, status codes, no allocation, no
 * synchronisation, checks before any HIP call) are those of moa_attn.h.
 *
 * WHAT A QUERY SEES.  Query i of Nq stands at position p = i + Nk - Nq and sees the
 * keys j, 0 <= j < Nk, with
 *
 *   j <= p + right   and   ( j >= p - left   or   j < sinks )
 *
 * A negative left or right is no limit on that side: left = -1, right = 0 is the
 * causal mask, left = right = -1 none, left = w - 1, right = 0 a causal window of
 * w keys, left = right = w a window to both sides.  sinks >= 0 first keys stay
 * visible behind the window (not beyond `right`).  Nq may be larger than Nk; a row
 * that sees nothing gets O = 0, LSE = -inf and gradients of 0, and gives none.
 *
 * HEADS.  Key/value head g serves the query heads g * Hq/Hk .. (g + 1) * Hq/Hk - 1.
 */
#ifndef MOA_WINDOW_H
#define MOA_WINDOW_H

#include "moa_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * moa_win_attn_num_splits, moa_win_attn_workspace_bytes -- the key splits that a
 * moa_win_attn_fwd call with these arguments uses, and the device workspace it then
 * needs in bytes (0 when it does not split).  num_splits: 0 = the library's choice,
 * else 1..256.
 */
int moa_win_attn_num_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk, int64_t d,
                            int64_t left, int64_t right, int64_t sinks, int num_splits);
size_t moa_win_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk,
                                    int64_t d, int64_t left, int64_t right, int64_t sinks,
                                    int num_splits);

/*
 * moa_win_attn_fwd -- O[b,h,i,:] = sum_j P_ij V_j, P_i = softmax over the keys j that
 * query i sees of scale * <Q[b,h,i,:], K_j>.
 *
 * Q         device input, bf16, logical shape [B][Hq][Nq][d].
 * K, V      device inputs, bf16, [B][Hk][Nk][d].
 * O         device output of storage type out_dtype (MOA_F32 or MOA_BF16),
 *           [B][Hq][Nq][d]; no element written twice, its bytes from the first to
 *           the last overlapping nothing else.
 * LSE       optional device output, fp32 [B][Hq][Nq] contiguous: the natural log of
 *           the softmax denominator.  NULL: not written.
 * *_strides element strides (batch, head, row) or NULL: contiguous.  Non-negative
 *           multiples of 16 bytes, of K's and V's rows at most 2^25 elements; the
 *           stride of a dimension of size 1 is ignored.
 * B, Hq, Hk, Nq, Nk, d
 *           All may be 0 but Hk and d; Hq a multiple of Hk; supported: d in {64,
 *           128}, Nq and Nk up to 2^30, B * Hq * Nq < 2^26, and fewer than 2^24
 *           workgroups (of 16, 32 or 128 rows of one key/value head and one split).
 * scale     finite, at most 2^127 in size; 0 and negative values are valid.
 * workspace, workspace_bytes
 *           at least moa_win_attn_workspace_bytes(...) bytes, 16-byte aligned,
 *           overlapping nothing (else MOA_ERR_WORKSPACE); NULL/0 when that is 0.
 *           Calls that may run at the same time need workspaces of their own.
 *
 * Computation: bf16 matrix products with fp32 accumulation; softmax statistics and
 * the sums of the unrounded weights in fp32.  A weight multiplies V as one bf16
 * number where O is bf16 and a key/value head has more than 32 rows (queries times
 * the query heads that share it), as the sum of two (17 bits) with fewer, and of
 * three (25 bits) where O is fp32.  Keys and values that a row does not see
 * have no part in it, whatever they hold: rows whose sums do not come out finite
 * are done again by the definition, with scores in fp64.  One kernel, or two when
 * the keys are split; no atomics, deterministic.
 */
int moa_win_attn_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int64_t B,
                     int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk, int64_t d,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* v_strides,
                     const int64_t* o_strides, int64_t left, int64_t right, int64_t sinks,
                     float scale, int out_dtype, void* workspace, size_t workspace_bytes,
                     int num_splits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOA_WINDOW_H */
