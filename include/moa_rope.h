/*
 * moa_rope.h -- norms of queries and keys for each head with the rotation by
 * position in the same pass, and the gradients: what stands between the input
 * projections and the attention of moa_attn.h.  The conventions (device
 * pointers, streams, status codes, no allocation, no synchronisation, checks
 * before any HIP call) are those of moa_attn.h.
 */
#ifndef MOA_ROPE_H
#define MOA_ROPE_H

#include "moa_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * moa_qk_norm_rope -- for every head row x of Q and of K (d elements):
 *
 *   n_e = x_e / sqrt(sum_i x_i^2 / d + eps)          (without weights: n = x)
 *   t_e = w_e * n_e                                  (without weights: t = x)
 *   y_a = t_a cos(p) - t_b sin(p),   y_b = t_b cos(p) + t_a sin(p)
 *
 * over the rot/2 pairs (a, b) of the first rot elements, y_e = t_e behind
 * them.  Pair i is (i, i + rot/2), or (2i, 2i + 1) when `interleaved`; its
 * angle is p = position * inv_freq[i].
 *
 * Q, K      device inputs of storage type dtype (MOA_F32 or MOA_BF16), logical
 *           shapes [B][Hq][N][d] and [B][Hk][N][d].
 * Qo, Ko    device outputs of the same type and shapes.  Qo may be Q and Ko may
 *           be K (same pointer and strides: in place).
 * wq, wk    norm weights [d] of storage type w_dtype, or NULL: that tensor is
 *           rotated without a norm.
 * positions device int64 [axes][B][N], any values (beyond 2^53 rounded to fp64),
 *           or NULL: token n is at position n on every axis.
 * inv_freq  device fp32 [rot/2] (NULL when rot == 0): radians per position of
 *           each pair.
 * B, Hq, Hk, N, d, rot
 *           batch, query heads, key heads, tokens, head size, rotated
 *           elements.  All may be 0 but d; supported: d in {64, 128}, rot a
 *           multiple of 16 up to d, B * N < 2^27, Hq + Hk < 2^30,
 *           B * (Hq + Hk) * N < 2^31.
 * *_strides element strides (batch, head, row) as for moa_attn_fwd_strided, or
 *           NULL: contiguous.  Non-negative, multiples of 16 bytes; an output
 *           must not write an element twice.  Input rows may overlap.  The
 *           stride of a dimension of size 1 is ignored.
 * axes, sections
 *           1 to 4 position axes.  sections (HOST array of axes values >= 0 with
 *           sum rot/2; may be NULL when axes == 1): the first sections[0] pairs turn by
 *           the position on axis 0, the next sections[1] by axis 1, and so on.
 * eps       finite, >= 0.
 * stream    hipStream_t as void*.
 *
 * Buffers: Qo and Ko must not share an element with each other or with any
 * input, but for the two in-place forms.  Q, K, Qo and Ko may be views that
 * interleave in one buffer (heads of a packed projection output) as long as
 * either their rows or their batches take turns in it.  Pointers are 16-byte
 * aligned, positions 8-byte, inv_freq 4-byte; a pointer may be NULL only when
 * its tensor has no elements.
 *
 * Computation: fp32 from exact inputs, one rounding at the end; angles in
 * fp64 with the products' errors carried along, reduced to one turn before sine
 * and cosine are taken in fp32, so that far positions lose nothing.  Rows whose squares leave fp32 (elements of 2^60
 * and more, or below 2^-45 with an eps too small to hide them) are divided by a
 * power of two first and lose nothing either, with weights below 2^60; a row of
 * zeros without an eps is 0 / 0, NaN.  One kernel; deterministic.
 */
int moa_qk_norm_rope(const void* Q, const void* K, void* Qo, void* Ko, const void* wq,
                     const void* wk, const int64_t* positions, const float* inv_freq, int64_t B,
                     int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t rot,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* qo_strides,
                     const int64_t* ko_strides, int axes, const int64_t* sections, int interleaved,
                     float eps, int dtype, int w_dtype, void* stream);

/*
 * moa_qk_norm_rope_bwd_workspace_bytes -- device workspace a
 * moa_qk_norm_rope_bwd call with weights needs, in bytes: partial sums of the
 * weights' gradients.  0 for invalid dimensions.
 */
size_t moa_qk_norm_rope_bwd_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d);

/*
 * moa_qk_norm_rope_bwd -- gradients of moa_qk_norm_rope.  With g the output's
 * gradient turned back by the same angles, r = 1 / sqrt(mean x^2 + eps) and
 * n = r x:
 *
 *   dw_e = sum over the rows of g_e n_e
 *   dx_e = r (g_e w_e - n_e * mean_i(g_i w_i n_i))     (without weights: dx = g)
 *
 * Q, K      the forward's inputs (not its outputs); Q is not read and may be
 *           NULL when wq is NULL, likewise K.
 * dQo, dKo  device inputs of storage type dtype: gradients of the outputs.
 * dQ, dK    device outputs of storage type dtype; dQ may be dQo and dK may be
 *           dKo (same pointer and strides).
 * dwq, dwk  device outputs, fp32 [d]: required when wq (wk) is given, else
 *           ignored.  Written as a whole, also when there are no rows (zeros).
 * workspace, workspace_bytes
 *           device scratch of at least moa_qk_norm_rope_bwd_workspace_bytes(...)
 *           bytes, 16-byte aligned (required when wq or wk is given).
 * The other arguments, the buffer rules and the status codes are those of the
 * forward.  At most two kernels; no atomics, deterministic.
 */
int moa_qk_norm_rope_bwd(const void* Q, const void* K, const void* dQo, const void* dKo,
                         const void* wq, const void* wk, const int64_t* positions,
                         const float* inv_freq, void* dQ, void* dK, float* dwq, float* dwk,
                         int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t rot,
                         const int64_t* q_strides, const int64_t* k_strides,
                         const int64_t* dqo_strides, const int64_t* dko_strides,
                         const int64_t* dq_strides, const int64_t* dk_strides, int axes,
                         const int64_t* sections, int interleaved, float eps, int dtype, int w_dtype,
                         void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOA_ROPE_H */
