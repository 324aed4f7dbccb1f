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
 *           128}, Nq and Nk up to 2^30, B * Hq * Nq < 2^26 (with num_splits of 2 and more
 *           2^26 - 4 at most), and fewer than 2^24 workgroups (of 16, 32 or 128 rows of
 *           one key/value head and one split).
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
 * three (all bits of an fp32 number) where O is fp32.  Keys and values that a row does
 * not see have no part in it, whatever they hold: rows whose sums do not come out
 * finite (values or scores that are infinite or NaN, values or scores that leave fp32,
 * scores that rise by 127 log2 units above those of the row's first keys) are done
 * again by the definition, each by one wave: a call full of such rows takes up to 300
 * times as long.  LSE is an fp32 number: infinite for scores beyond its range.  One
 * kernel, or two when the keys are split; no atomics, deterministic.
 */
int moa_win_attn_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int64_t B,
                     int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk, int64_t d,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* v_strides,
                     const int64_t* o_strides, int64_t left, int64_t right, int64_t sinks,
                     float scale, int out_dtype, void* workspace, size_t workspace_bytes,
                     int num_splits, void* stream);

/*
 * moa_win_attn_bwd_workspace_bytes -- device workspace of a moa_win_attn_bwd call, in
 * bytes (0 for dimensions that are invalid or not supported): a sum for every query
 * row, and partial sums of dK and dV where first keys stay visible behind a window, or
 * where the key tiles alone would leave compute units idle.
 */
size_t moa_win_attn_bwd_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk,
                                        int64_t d, int64_t left, int64_t right, int64_t sinks);

/*
 * moa_win_attn_bwd -- gradients of moa_win_attn_fwd.  With P the forward's weights,
 * D_i = <dO_i, O_i> and dS_ij = P_ij (<dO_i, V_j> - D_i) over the pairs of which query i
 * sees key j,
 *
 *   dQ_i = scale * sum_j dS_ij K_j
 *   dK_j = scale * sum_i dS_ij Q_i,   dV_j = sum_i P_ij dO_i
 *
 * the last two over the queries of all heads that share the key/value head.
 *
 * Q, K, V   the forward's inputs.
 * O, LSE    its outputs: O of storage type o_dtype (MOA_F32 or MOA_BF16), LSE required.
 * dO        device input, bf16, [B][Hq][Nq][d].
 * dQ, dK, dV
 *           device outputs, bf16, written as a whole: no element written twice, the
 *           bytes from the first to the last of each overlapping nothing else.
 * *_strides as for the forward; here rows of all tensors are at most 2^23 elements
 *           apart.
 * B, Hq, Hk, Nq, Nk, d, left, right, sinks, scale
 *           the forward's; supported besides: B * Hk * Nk < 2^26, at most 2^23
 *           workgroups of 512 threads (of 128 keys of one key/value head), and at most
 *           2^24 of 256 where partial sums are joined (d/4 for 128 keys).
 * workspace, workspace_bytes
 *           at least moa_win_attn_bwd_workspace_bytes(...) bytes, 16-byte aligned,
 *           overlapping nothing.
 *
 * Computation: bf16 matrix products with fp32 accumulation; P and dS enter them as one
 * bf16 number each, one rounding at the end.  D comes from O and dO, or, where O is
 * bf16 and rows of a tile of 128 see fewer than 64 keys, from the keys: sum_j P_ij
 * <dO_i, V_j>, which has no part of O's rounding.  Rows and keys that do not see each
 * other have no part in each other's gradients, whatever they hold: sums that do not
 * come out finite are done again by the definition, each by one wave (up to 150 times as
 * long where all are).  Two kernels, or three with
 * partial sums; no atomics, deterministic.
 */
int moa_win_attn_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                     const float* LSE, void* dQ, void* dK, void* dV, int64_t B, int64_t Hq,
                     int64_t Hk, int64_t Nq, int64_t Nk, int64_t d, const int64_t* q_strides,
                     const int64_t* k_strides, const int64_t* v_strides, const int64_t* o_strides,
                     const int64_t* do_strides, const int64_t* dq_strides,
                     const int64_t* dk_strides, const int64_t* dv_strides, int64_t left,
                     int64_t right, int64_t sinks, float scale, int o_dtype, void* workspace,
                     size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOA_WINDOW_H */
