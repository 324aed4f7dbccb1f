// Operands of matrix products from LDS stages, for the gradient kernels.
#pragma once

#include "prefill_bf16_common.h"

namespace moa {
namespace pf {

// Per-lane LDS addresses of a stage (the layout of the forward's tiles: 64 rows of D
// bf16, 16-byte chunks XOR-swizzled per row).
template <int D>
struct TileAddr {
    uint32_t row[D / 16];      // A operand of a row-major stage: row col (+32 u), chunk 2s + half
    uint32_t tr[D / 32][2];    // transposing reads: D-block b, lo / hi row quads
    __device__ __forceinline__ TileAddr(int lane) {
        constexpr uint32_t RB = Cfg<D>::ROW_BYTES;
        const int col = lane & 31, half = lane >> 5;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
            row[s] = (uint32_t)col * RB + (uint32_t)(((2 * s + half) ^ swz<D>(col)) * 16);
        const int g = lane >> 4, j = (lane >> 2) & 3, q = lane & 3;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int h8 = 0; h8 < 2; ++h8) {
                const int r = 4 * (g >> 1) + j + 8 * h8;
                const int dv = dv_of<D>(b, 16 * (g & 1) + 4 * q);
                tr[b][h8] = (uint32_t)r * RB + (uint32_t)((((dv >> 3) ^ swz<D>(r)) * 16) + (dv & 7) * 2);
            }
    }
};

// MFMA A operand from a stage: rows 32u + (lane % 32), contraction chunk s.
template <int D>
__device__ __forceinline__ bf16x8 stage_rows(const unsigned char* st, const TileAddr<D>& a, int u, int s) {
    return *reinterpret_cast<const bf16x8*>(st + a.row[s] + u * 32 * Cfg<D>::ROW_BYTES);
}
// MFMA A operand of the transposed stage: D-block b, 16-row chunk cc.
template <int D>
__device__ __forceinline__ bf16x8 stage_tr(const unsigned char* st, const TileAddr<D>& a, int b, int cc) {
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(st + a.tr[b][0] + cc * 16 * Cfg<D>::ROW_BYTES));
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(st + a.tr[b][1] + cc * 16 * Cfg<D>::ROW_BYTES));
    const v4s both[2] = {lo, hi};
    return __builtin_bit_cast(bf16x8, both);
}

// Packs an fp32 accumulator (16 values) into two bf16x8 MFMA B operands in the
// key (or query) order of the transposing reads: chunk c2 takes elements
// 8 c2 .. 8 c2 + 7.
__device__ __forceinline__ void pack16(const float (&x)[16], bf16x8 (&pb)[2]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x2 pp = {(__bf16)x[8 * g + 2 * j], (__bf16)x[8 * g + 2 * j + 1]};
            w[j] = __builtin_bit_cast(uint32_t, pp);
        }
        pb[g] = __builtin_bit_cast(bf16x8, w);
    }
}

}  // namespace pf
}  // namespace moa
