// Attention with a window for many rows (moa_window.h, moa_paged.h).
//
// One workgroup = 4 waves x 32 rows of one key/value head, a row being a query and
// one of the G = Hq/Hk heads that share it, query by query: keys and values are
// read once for all of them, and 128 rows are only 128/G positions wide, so that
// a window's ragged ends cost little.  K and V stream through a two-stage LDS ring
// in tiles of 64 or 32 keys, one barrier per tile, in the layout and with the products of
// the prefill kernels (prefill_bf16_common.h).  Each wave loads 16 or 8 of a
// tile's rows, which lie in one page whatever its size.  Only tiles that a row of the
// workgroup sees are walked: those of the first visible keys, then the windows'.
//
// Softmax: one reference per row, the largest score of the first 32 keys of which it
// sees any; all others are weighed against it as they come.  fp32 and bf16 hold
// weights up to 2^127 as well as small ones, so the reference need not follow the
// maximum: only a row whose scores rise by more than 127 log2 units (88 of the
// exponent) above it comes out infinite, and is done by the definition.  A state's sums
// may then be 2^127 against its reference, so where states meet, of two key streams or
// of splits, the one with the lower reference is never left out for that.  (Raised in
// the loop where sums grew, the rarely taken branch cost a copy of all sums in every
// step: 4096 tokens in a window of 512, 114 us.)  The sums are of the fp32 weights.
//
// A weight meets V as one bf16 number for a bf16 output, off by 2^-8 of it at most, as in
// the prefill.  That leaves the output's error at 1.4 times its own rounding's (2.25e-3 to
// 2.35e-3 against 64 bits for 1.65e-3); two numbers would leave the rounding's alone and
// cost a quarter of the time in the matrix cores and the packing (4096 tokens in a
// window of 512 95 -> 119 us, 200 queries on 20011 keys 94 -> 122, 4 x 1000 causal, d = 64,
// 17 -> 21).  Who needs more takes an fp32 output, whose weights are three numbers, all of
// their bits (two left it at 2.3e-6, nine times what fp32 sums alone make).
//
// What bounds it: matrix and vector instructions, which overlap in part (matrix cores
// 0.43 to 0.48 of a unit's cycles, 6 to 8 vector instructions for each matrix
// instruction).  d = 128, 32 heads on 8: 2 x 4096 tokens in a window of 512 94 us, 8192 in
// one of 1024 163 us (0.79 PFLOP/s of visible pairs), 8192 causal of 32 heads 544 us.
#include <limits>

#include "prefill_bf16_common.h"
#include "split_join.h"
#include "win_common.h"

namespace moa {
namespace {

using namespace win;
using pf::Cfg;
using pf::dv_of;
using pf::lds_v4s;
using pf::swz;
using pf::v4s;

constexpr int MW = 4;            // waves
constexpr int MROWS = MW * 32;   // rows per workgroup

// How O leaves: bf16, fp32, or the fp32 state of a split.
enum { TO_BF16, TO_F32, TO_STATE };

template <int D, int OUT, int TERMS, int BN, int KS>
__global__ __launch_bounds__(KS * MW * 64, KS == 1 && (D == 64 || BN == 32) ? 3 : 2) void win_many_kernel(WinAttn p, float c, uint32_t qflip, int row_tiles) {
    using C = Cfg<D>;
    constexpr uint32_t RB = C::ROW_BYTES;
    constexpr int SN = 32;                                // keys per step
    constexpr int TILE = BN * C::ROW_BYTES;
    constexpr int LPW = TILE / (MW * 1024);               // 16-byte loads per lane per tile
    constexpr int RPW = BN / MW, GROUPS = BN / 16;        // rows that a wave loads, page groups of a tile
    constexpr int ALL = (1 << GROUPS) - 1;
    // One array per ring stage: the compiler tracks direct-to-LDS loads per object.
    __shared__ __attribute__((aligned(1024))) unsigned char k_st0[KS][TILE];
    __shared__ __attribute__((aligned(1024))) unsigned char k_st1[KS][TILE];
    __shared__ __attribute__((aligned(1024))) unsigned char v_st0[KS][TILE];
    __shared__ __attribute__((aligned(1024))) unsigned char v_st1[KS][TILE];
    __shared__ float state[KS == 2 ? MW : 1][2][64];
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;

    const int lane = threadIdx.x & 63;
    // Waves MW .. of two key streams hold the rows of waves 0 .. and take every second tile.
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % MW;
    const int stream = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / MW;
    const int col = lane & 31, half = lane >> 5;
    const KeySource& src = p.s;
    const int G = (int)p.group.n;
    // Row tiles last, those of the highest positions first; the heads next to each
    // other, so that the row tiles of a head mostly go to one XCD.
    const int up = over(p.per_tile, blockIdx.x), rt = row_tiles - 1 - up, in_tile = blockIdx.x - up * (int)p.per_tile.n;
    const int bh = over(p.per_head, in_tile), sp = in_tile - bh * p.splits, b = over(p.heads, bh), h = bh - b * p.hk;

    const int count = new_tokens(src.new_lens, b, p.n), rows = count * G, row0 = rt * MROWS;
    if (row0 >= rows) return;
    const int len = length(src, b), end = max(0, min(len, capacity(src)));
    const long long first = (long long)len - count;   // position of query 0
    const auto seen_of = [&](int row) { return seen_from(p.w, first + over(p.group, row), end); };
    const auto uniform = [](Seen s) {
        return Seen{__builtin_amdgcn_readfirstlane(s.lo), __builtin_amdgcn_readfirstlane(s.hi)};
    };
    const Seen low = uniform(seen_of(row0)), high = uniform(seen_of(min(row0 + MROWS, rows) - 1));
    const Tiles<BN> tiles(low, high, p.w.sinks);
    const int per = (tiles.count + p.splits - 1) / p.splits, begin = sp * per, stop = min(tiles.count, begin + per);

    // This wave's rows.
    const int w0 = row0 + wave * 32, row = w0 + col;
    const bool live = w0 < rows, in = row < rows;
    const int sinks = p.w.sinks;
    const Seen wl = uniform(seen_of(min(w0, rows - 1))), wh = uniform(seen_of(min(w0 + 32, rows) - 1));
    const Seen seen = seen_of(min(row, rows - 1));

    bf16x8 qf[D / 16];
    {
        const int qi = in ? over(p.group, row) : 0, hh = h * G + (in ? row - qi * G : 0);
        const u16* at = static_cast<const u16*>(p.q) + b * p.qs[0] + hh * p.qs[1] + qi * p.qs[2] + half * 8;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            u32x4 w = {0, 0, 0, 0};
            if (in) w = *reinterpret_cast<const u32x4*>(at + 16 * s);
            qf[s] = __builtin_bit_cast(bf16x8, w ^ qflip);
        }
    }

    const uint32_t krb = (uint32_t)src.ks[2] * 2u, vrb = (uint32_t)src.vs[2] * 2u;
    uint32_t ld_koff[LPW], ld_voff[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
        const int slot = (wave * LPW + i) * 64 + lane;
        const int r = slot / C::CHUNKS, ch = slot % C::CHUNKS;
        const uint32_t chunk = (uint32_t)((ch ^ swz<D>(r)) * 16);
        ld_koff[i] = (uint32_t)(r % RPW) * krb + chunk;   // this wave's rows of the tile
        ld_voff[i] = (uint32_t)(r % RPW) * vrb + chunk;
    }
    // Lane GROUPS i + t holds the page of 16-key group t of this stream's i-th tile from
    // `known` on.
    int pages = 0, known = begin + stream;
    const auto look = [&]() {
        const int v = known + lane / GROUPS * KS, key = tiles.at(v) * BN + 16 * (lane % GROUPS);
        pages = v < stop && key < end ? page_of(src, b, key) : -1;
    };
    // Starts the loads of the v-th tile; bit t of the result: group t has a page.
    // Tokens behind the last, and those without a page, become zeros.
    auto issue = [&](int v, auto stage) __attribute__((always_inline)) -> int {
        unsigned char* ks = decltype(stage)::value == 0 ? k_st0[stream] : k_st1[stream];
        unsigned char* vs = decltype(stage)::value == 0 ? v_st0[stream] : v_st1[stream];
        if (v - known == 64 / GROUPS * KS) {
            known = v;
            look();
        }
        const int i = (v - known) / KS, key = tiles.at(v) * BN + RPW * wave;
        const int page = __builtin_amdgcn_readlane(pages, GROUPS * i + wave * RPW / 16);
        const int n = page >= 0 ? max(0, min(RPW, end - key)) : 0;
        const u16* kb = static_cast<const u16*>(src.k) + (n ? key_offset(src.ks, src.shift, page, h, key) : 0);
        const u16* vb = static_cast<const u16*>(src.v) + (n ? key_offset(src.vs, src.shift, page, h, key) : 0);
        const auto rk = make_rsrc(kb, rows_extent(n, krb, RB)), rv = make_rsrc(vb, rows_extent(n, vrb, RB));
#pragma unroll
        for (int j = 0; j < LPW; ++j) buffer_load16_to_lds(rk, ks + (wave * LPW + j) * 1024, ld_koff[j]);
#pragma unroll
        for (int j = 0; j < LPW; ++j) buffer_load16_to_lds(rv, vs + (wave * LPW + j) * 1024, ld_voff[j]);
        return (int)(__ballot(pages >= 0) >> (GROUPS * i)) & ALL;
    };
    uint32_t kaddr[D / 16], vaddr[D / 32][2];
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
        kaddr[s] = (uint32_t)col * RB + (uint32_t)(((2 * s + half) ^ swz<D>(col)) * 16);
    {
        const int g = lane >> 4, j = (lane >> 2) & 3, q = lane & 3;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int h8 = 0; h8 < 2; ++h8) {
                const int r = 4 * (g >> 1) + j + 8 * h8, dv = dv_of<D>(d, 16 * (g & 1) + 4 * q);
                vaddr[d][h8] = (uint32_t)r * RB + (uint32_t)((((dv >> 3) ^ swz<D>(r)) * 16) + (dv & 7) * 2);
            }
    }

    f32x16 oacc[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) oacc[d] = f32x16{};
    float ref = kNegInf;     // log2 units
    float neg = 0.0f;        // -ref, or 0 while it is -inf
    float l = 0.0f;          // sum over this half-wave's keys

    auto tile = [&](int v, int have, auto stage) __attribute__((always_inline)) {
        const unsigned char* ks = decltype(stage)::value == 0 ? k_st0[stream] : k_st1[stream];
        unsigned char* vs = decltype(stage)::value == 0 ? v_st0[stream] : v_st1[stream];
        const int k0 = tiles.at(v) * BN;
        if (!live) return;
#pragma unroll
        for (int sb = 0; sb < BN / SN; ++sb) {
            if (!any_sees(wl, wh, sinks, k0 + sb * SN)) continue;
            f32x16 s = f32x16{};
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    *reinterpret_cast<const bf16x8*>(ks + kaddr[k] + sb * SN * RB), qf[k], s, 0, 0, 0);
            const int paged = (have >> (2 * sb)) & 3;
            if (paged != 3 || !all_see(wl, wh, sinks, k0 + sb * SN)) {
                uint32_t bits = seen_bits(seen, sinks, k0 + sb * SN);
                if (paged != 3) bits &= (paged & 1 ? 0x0000ffffu : 0u) | (paged & 2 ? 0xffff0000u : 0u);
                keep(s, bits, half);
            }
            // Rows that see their first keys here take their reference from them.
            if (wave_any(ref == kNegInf)) {
                float m = kNegInf;
#pragma unroll
                for (int i = 0; i < 16; ++i) m = fmaxf(m, s[i]);
                m = half_max(m) * c;
                ref = ref == kNegInf ? m : ref;
                neg = ref == kNegInf ? 0.0f : -ref;
            }
            u32x4 pt[SN / 16][TERMS];
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int g = 0; g < SN / 16; ++g) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = g * 8 + 2 * j;
                    const float a = exp2_hw(__builtin_fmaf(s[i], c, neg)), d = exp2_hw(__builtin_fmaf(s[i + 1], c, neg));
                    sum[0] += a;
                    sum[1] += d;
                    uint32_t x[TERMS];
                    bf16_terms<TERMS>(a, d, x);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) pt[g][k][j] = x[k];
                }
            }
            l += sum[0] + sum[1];
#pragma unroll
            for (int cc = 0; cc < SN / 16; ++cc)
#pragma unroll
                for (int d = 0; d < D / 32; ++d) {
                    const int r = (sb * (SN / 16) + cc) * 16;
                    const v4s both[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(vs + vaddr[d][0] + r * RB)),
                                         __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(vs + vaddr[d][1] + r * RB))};
                    const bf16x8 a = __builtin_bit_cast(bf16x8, both);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k)
                        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, pt[cc][k]), oacc[d], 0, 0, 0);
                }
        }
    };

    // A stream's tiles alternate between the two stages.  After the barrier at a tile's
    // start every wave has its part of it in LDS and is done with the tile before, into
    // whose stage the next one is loaded while this one is worked on.
    auto turn = [&](int v, int have, auto stage, int& later, auto other) __attribute__((always_inline)) {
        pf::wait_vmcnt<0>();
        __syncthreads();
        if (v + KS < stop) later = issue(v + KS, other);
        if (KS == 1 || v < stop) tile(v, have, stage);
    };
    if (begin < stop) {
        look();
        int have0 = 0, have1 = 0;
        if (begin + stream < stop) have0 = issue(begin + stream, S0{});
        for (int v = begin; v < stop; v += 2 * KS) {
            turn(v + stream, have0, S0{}, have1, S1{});
            if (v + KS >= stop) break;
            turn(v + KS + stream, have1, S1{}, have0, S0{});
        }
    }
    __syncthreads();   // every wave is done with the stages
    if constexpr (KS == 2) {
        // The second stream's sums, through LDS, against a common reference.
        float* x = reinterpret_cast<float*>(wave < 2 ? &k_st0[0][0] : &k_st1[0][0]) + (wave & 1) * (D / 2) * 64;
        if (stream == 1) {
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[(d * 16 + i) * 64 + lane] = oacc[d][i];
            state[wave][0][lane] = ref;
            state[wave][1][lane] = l;
        }
        __syncthreads();
        if (stream == 1) return;
        const float r = state[wave][0][lane], top = fmaxf(ref, r);
        // (sums without a reference are 0, or NaN of a score that is)
        const TwoFactors mine(ref == kNegInf ? 0.0f : ref - top), its(r == kNegInf ? 0.0f : r - top);
        {
#pragma clang fp contract(off)   // a row's sum is the same from either stream
            l = mine.of(l) + its.of(state[wave][1][lane]);
        }
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[d][i] = __builtin_fmaf(oacc[d][i] * mine.rest, mine.a, its.of(x[(d * 16 + i) * 64 + lane]));
        ref = top;
    }
    if (!live) return;
    const WinAttn late = arguments_again<WinAttn>();

    // O = acc / l (or the sums as they are) through a 32-row slice of the stages,
    // whole rows per store.
    // (with two streams beside the sums that other waves still read)
    unsigned char* stg;
    if constexpr (KS == 2) {
        static_assert(BN == 64, "two slices in each stage");
        stg = (wave < 2 ? v_st0[0] : v_st1[0]) + (wave & 1) * 32 * RB;
    } else {
        constexpr int SLICES = BN / 32;   // of one stage
        stg = (wave / SLICES == 0 ? k_st0[0] : wave / SLICES == 1 ? k_st1[0] : wave / SLICES == 2 ? v_st0[0] : v_st1[0]) + wave % SLICES * 32 * RB;
    }
    const float total = half_sum(l);
    const bool none = ref == kNegInf;   // no visible key
    const float inv = OUT == TO_STATE ? 1.0f : none ? 0.0f : 1.0f / total;
    // Sums that are not finite, or none at all in a row that sees keys.
    constexpr float most = OUT == TO_STATE ? (float)kMaxSplits : 1.0f;
    float zero = 0.0f * (total * most);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(oacc[d][i] * most, 0.0f, zero);
    zero = half_sum(zero);
    const bool odd = in && (!(zero == 0.0f) || (total == 0.0f && begin < stop && sees_any(seen, sinks)));
    int ln = lane;
    asm volatile("" : "+v"(ln));   // staging addresses are formed here, not above the loop
    const int cl = ln & 31, hf = ln >> 5;
    // Row r of this wave's 32: its query head and query.
    const auto place = [&](int r, int& hh, int& qi) {
        qi = over(late.group, w0 + r);
        hh = h * (int)late.group.n + (w0 + r) - qi * (int)late.group.n;
    };
    if constexpr (OUT == TO_BF16) {
        constexpr int CHK = C::CHUNKS, RPI = 64 / CHK;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int dv = dv_of<D>(d, g * 8 + hf * 4);
                *reinterpret_cast<uint2*>(stg + (uint32_t)cl * RB + (uint32_t)((((dv >> 3) ^ (cl & (CHK - 1))) * 16) + (dv & 7) * 2)) =
                    make_uint2(pack2(oacc[d][g * 4 + 0] * inv, oacc[d][g * 4 + 1] * inv),
                               pack2(oacc[d][g * 4 + 2] * inv, oacc[d][g * 4 + 3] * inv));
            }
        pf::wait_lgkmcnt0();   // only this wave reads its rows
        const int rr = ln / CHK, ch = ln % CHK;
#pragma unroll
        for (int i = 0; i < 32 / RPI; ++i) {
            const int r = i * RPI + rr;
            const uint4 x = *reinterpret_cast<const uint4*>(stg + (uint32_t)r * RB + (uint32_t)((ch ^ (r & (CHK - 1))) * 16));
            if (w0 + r >= rows) continue;
            int hh, qi;
            place(r, hh, qi);
            *reinterpret_cast<uint4*>(static_cast<u16*>(late.o) + b * late.os[0] + hh * late.os[1] + qi * late.os[2] + ch * 8) = x;
        }
    } else {
        // fp32 rows in two passes of D / 2 columns
        constexpr int HB = D * 2, HCH = HB / 16, RPI = 64 / HCH;
        const int rr = ln / HCH, ch = ln % HCH;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (dv_of<D>(d, g * 8) / (D / 2) != u) continue;
                    const int cc = (dv_of<D>(d, g * 8 + hf * 4) - u * (D / 2)) / 4;
                    *reinterpret_cast<float4*>(stg + (uint32_t)cl * HB + (uint32_t)((cc ^ (cl & (HCH - 1))) * 16)) =
                        make_float4(oacc[d][g * 4 + 0] * inv, oacc[d][g * 4 + 1] * inv, oacc[d][g * 4 + 2] * inv, oacc[d][g * 4 + 3] * inv);
                }
            pf::wait_lgkmcnt0();
#pragma unroll
            for (int i = 0; i < 32 / RPI; ++i) {
                const int r = i * RPI + rr;
                const float4 x = *reinterpret_cast<const float4*>(stg + (uint32_t)r * HB + (uint32_t)((ch ^ (r & (HCH - 1))) * 16));
                if (w0 + r >= rows) continue;
                int hh, qi;
                place(r, hh, qi);
                float* to;
                if constexpr (OUT == TO_STATE) to = late.ws + ((((size_t)b * late.hq + hh) * late.n + qi) * late.splits + sp) * D;
                else to = static_cast<float*>(late.o) + b * late.os[0] + hh * late.os[1] + qi * late.os[2];
                *reinterpret_cast<float4*>(to + u * (D / 2) + ch * 4) = x;
            }
            pf::wait_lgkmcnt0();
        }
    }
    if (half == 0 && in) {
        int hh, qi;
        place(col, hh, qi);
        const size_t at = ((size_t)b * late.hq + hh) * late.n + qi;
        if constexpr (OUT == TO_STATE) {
            float* ml = late.ws + (size_t)late.B * late.hq * late.n * late.splits * D + (at * late.splits + sp) * 2;
            ml[0] = ref;
            ml[1] = total;
        } else {
            if (late.lse) late.lse[at] = none ? kNegInf : (ref + __log2f(total)) * kLn2;
        }
    }
    // Rows that have to be done by their definition.
    for (uint32_t left = (uint32_t)__ballot(odd); left; left &= left - 1) {
        int hh, qi;
        const int r = __builtin_ctz(left);
        place(r, hh, qi);
        float f[D / 64], M, L;
        row_by_definition<D, BN>(late, b, h, static_cast<const u16*>(late.q) + b * late.qs[0] + hh * late.qs[1] + qi * late.qs[2],
                                 seen_of(w0 + r), tiles, begin, stop, OUT == TO_STATE, f, M, L);
        store_row<D>(late, b, hh, qi, sp, f, M, L);
    }
}

template <int D>
hipError_t go(WinAttn p, hipStream_t stream) {
    set_divisions(p);
    const long long rows = (long long)p.n * (p.hq / p.hk);
    const int tiles = (int)((rows + MROWS - 1) / MROWS);
    // As in the kernel of few rows.
    float c = p.scale * kLog2e;
    const uint32_t flip = c < 0.0f ? 0x80008000u : 0u;
    c = c < 0.0f ? -c : c;
    if (c == 0.0f) c = std::numeric_limits<float>::denorm_min();
    const long long blocks = (long long)p.B * p.hk * tiles * p.splits;
    const auto run = [&](auto kernel, int streams = 1) {
        return launch_kernel(kernel, dim3((unsigned)blocks), dim3(streams * MW * 64), stream, p, c, flip, tiles);
    };
    // At d = 128 two workgroups with 64-key tiles fit a compute unit, and three with
    // tiles of 32, which wait for each other less but have twice the barriers: for more
    // workgroups than two for every unit (4096 tokens in a window of 512, 2048 of them
    // 100 -> 94 us, 8192 in 1024 176 -> 166; 504 of 200 queries on 20011 keys 85 -> 90).
    if constexpr (D == 128)
        if (p.splits == 1 && blocks > 512) return p.out_bf16 ? run(win_many_kernel<D, TO_BF16, 1, 32, 1>) : run(win_many_kernel<D, TO_F32, 3, 32, 1>);
    // Where a unit has one workgroup, its keys go to two streams of four waves.
    const bool two = blocks <= 256;
    const auto go_as = [&](auto out, auto terms) {
        constexpr int O = decltype(out)::value, N = decltype(terms)::value;
        return two ? run(win_many_kernel<D, O, N, 64, 2>, 2) : run(win_many_kernel<D, O, N, 64, 1>);
    };
    constexpr std::integral_constant<int, 1> one_term;
    constexpr std::integral_constant<int, 3> three_terms;
    if (p.splits == 1)
        return p.out_bf16 ? go_as(std::integral_constant<int, TO_BF16>{}, one_term) : go_as(std::integral_constant<int, TO_F32>{}, three_terms);
    constexpr std::integral_constant<int, TO_STATE> state;
    const hipError_t e = p.out_bf16 ? go_as(state, one_term) : go_as(state, three_terms);
    if (e != hipSuccess) return e;
    const SplitJoin j{p.ws, p.o, p.lse, p.s.new_lens, {p.os[0], p.os[1], p.os[2]}, p.B, p.hq, p.n, p.splits, p.out_bf16};
    return launch_split_join<D>(j, stream, RowsAgain{p});
}

}  // namespace

hipError_t launch_win_many(const WinAttn& p, hipStream_t stream) {
    return p.d == 64 ? go<64>(p, stream) : go<128>(p, stream);
}

}  // namespace moa
