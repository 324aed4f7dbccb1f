// Gradients of the attention with a window (moa_window.h) on gfx950 matrix cores,
// the weights recomputed from the forward's LSE.
//
// With s = <q_i, k_j>, c = scale * log2(e) and lse2_i = LSE_i * log2(e), over the pairs
// of which query i sees key j:
//   P_ij  = 2^(s_ij c - lse2_i),   dP_ij = <dO_i, v_j>,   D_i = <dO_i, O_i>
//   dS_ij = P_ij (dP_ij - D_i)
//   dQ_i  = scale * sum_j dS_ij k_j
//   dK_j  = scale * sum_i dS_ij q_i,   dV_j = sum_i P_ij dO_i     (i over the queries of
//           all heads that share the key/value head)
//
// * win_dq: one workgroup = 4 waves x 32 rows of one key/value head, a row being a
//   query and one of the G = Hq/Hk heads that share it; K and V tiles of 64 keys
//   stream through LDS as in the forward, only those that a row sees.  D_i of its
//   rows comes first, for the other kernel too: from O, or where a row sees few keys
//   and O is bf16, from the keys.
// * win_dkdv: one workgroup = 128 keys; Q and dO of the queries that see one of them
//   stream through LDS, 64 queries of one head at a time, head after head, so that
//   shared heads meet in the same sums.  A pair of waves on one SIMD owns 32 keys:
//   one forms S and P and sums dV, the other forms dP and dS with the partner's P and
//   sums dK, one stage behind.  P crosses with the upper 24 bits of its fp32 number,
//   four in three registers.  (In bf16 its rounding made dK's error 2.9e-3, with these
//   2.4e-3.)
// * The first keys stay visible to all later queries, so their sums would be as long
//   as the sequence where all others are as long as the window.  The queries behind
//   their windows are cut into chunks with workgroups of their own, and where there
//   are few key tiles the tiles' queries into parts, about as long as each other; they
//   leave fp32 sums that win_join adds in a fixed order.
// No atomics; deterministic.  P and dS are rounded to one bf16 number each for the matrix
// products, which makes the gradients' errors 2.1e-3 to 2.5e-3 where their own rounding to
// bf16 makes 1.65e-3; as two numbers, 1.7e-3, 8192 tokens in a window of 1024 took 264 us
// for 220 in dQ and 418 for 322 in dK/dV.
// Rows whose sums do not come out finite are done again by the definition.
//
// What bounds them: matrix instructions with an operand from LDS in each (matrix cores
// 0.50 of a unit's cycles in dQ, 0.44 in dK/dV, two waves to a SIMD, which is what d = 128
// has registers for).  8192 tokens, 32 heads on 8, d = 128, a window of 1024: dQ 226 us,
// dK/dV 332 us, the join of the first keys' sums 6 us.
#include <algorithm>
#include <type_traits>

#include "prefill_bf16_common.h"
#include "stage_common.h"
#include "win_common.h"

namespace moa {
namespace {

using namespace win;
using pf::BN;
using pf::Cfg;
using pf::dv_of;
using pf::pack16;
using pf::stage_rows;
using pf::stage_tr;
using pf::swz;
using pf::TileAddr;

// Element offset of row i of head hh of sequence b.
__device__ __forceinline__ long long at_row(const long long (&s)[3], int b, int hh, int i) {
    return b * s[0] + hh * s[1] + i * s[2];
}

__device__ __forceinline__ Seen seen_by(const WinGrad& p, int i) {
    return seen_from(p.w, (long long)i + p.nk - p.nq, p.nk);
}

// What one pair gives to a gradient: P and dS.  s0, s1: the rows of the score, t0, t1:
// those of dP; s0 and t0 are the same in all lanes.
template <int D>
__device__ __forceinline__ void pair_by_definition(const u16* s0, const u16* s1, const u16* t0, const u16* t1, double c, float lse2,
                                                   float dsum, float& w, float& ds) {
    w = exp2_hw((float)(dot<D>(s0, s1) * c - (double)lse2));
    ds = w * (float)(dot<D>(t0, t1) - (double)dsum);
}

template <int D>
__device__ __forceinline__ void store_lane(u16* to, const float (&o)[D / 64], float mul) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < E; ++e) reinterpret_cast<__bf16*>(to)[E * lane + e] = (__bf16)(o[e] * mul);
}

// A lane's row of D elements from an accumulator in the transposed layout.
template <int D>
__device__ __forceinline__ void store_row16(u16* to, int half, const f32x16 (&acc)[D / 32], float mul) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<uint2*>(to + dv_of<D>(d, g * 8 + half * 4)) =
                make_uint2(pack2(acc[d][g * 4 + 0] * mul, acc[d][g * 4 + 1] * mul), pack2(acc[d][g * 4 + 2] * mul, acc[d][g * 4 + 3] * mul));
}
template <int D>
__device__ __forceinline__ void store_row16(float* to, int half, const f32x16 (&acc)[D / 32], float mul) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4*>(to + dv_of<D>(d, g * 8 + half * 4)) =
                make_float4(acc[d][g * 4 + 0] * mul, acc[d][g * 4 + 1] * mul, acc[d][g * 4 + 2] * mul, acc[d][g * 4 + 3] * mul);
}

// Whether a lane's row has an element that is not finite (the two halves of a row
// are lanes l and l ^ 32).
template <int D>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[D / 32]) {
    float zero = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(acc[d][i], 0.0f, zero);
    return !(half_sum(zero) == 0.0f);
}

// ---- dQ ----------------------------------------------------------------------

constexpr int QW = 4;            // waves
constexpr int QROWS = QW * 32;   // rows per workgroup
// Row tiles with a row that sees fewer keys take D_i from the keys.
constexpr int kFewKeys = 64;

// How many keys a row sees; fewest at a tile's first or last row, since both limits
// rise with the position and the keys' ends cut them.
__device__ __forceinline__ int keys_seen(Seen s, int sinks) { return s.hi - s.lo + min(sinks, s.lo); }

template <int D, int KS>
__global__ __launch_bounds__(KS * QW * 64, 2) void win_dq_kernel(WinGrad p, float c, int row_tiles) {
    using C = Cfg<D>;
    constexpr uint32_t RB = C::ROW_BYTES;
    constexpr int LPW = C::TILE_BYTES / (QW * 1024);
    __shared__ __attribute__((aligned(1024))) unsigned char k_st0[KS][C::TILE_BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char k_st1[KS][C::TILE_BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char v_st0[KS][C::TILE_BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char v_st1[KS][C::TILE_BYTES];
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;

    const int lane = threadIdx.x & 63;
    // Waves QW .. of two key streams hold the rows of waves 0 .. and take every second tile.
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % QW;
    const int stream = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / QW;
    const int col = lane & 31, half = lane >> 5;
    const int G = (int)p.group.n, up = over(p.per_item, blockIdx.x), rt = row_tiles - 1 - up;
    const int bh = blockIdx.x - up * (int)p.per_item.n, b = over(p.heads, bh), h = bh - b * p.hk;
    const int rows = p.nq * G, row0 = rt * QROWS;
    const auto uniform = [](Seen s) {
        return Seen{__builtin_amdgcn_readfirstlane(s.lo), __builtin_amdgcn_readfirstlane(s.hi)};
    };
    const Seen tl = uniform(seen_by(p, over(p.group, row0))), th = uniform(seen_by(p, over(p.group, min(row0 + QROWS, rows) - 1)));
    const Tiles<BN> tiles(tl, th, p.w.sinks);

    // This wave's rows; this lane's row, its Q and dO fragments, LSE and D.
    const int w0 = row0 + wave * 32, row = w0 + col;
    const bool live = w0 < rows, in = row < rows;
    const int sinks = p.w.sinks;
    const Seen wl = uniform(seen_by(p, over(p.group, min(w0, rows - 1)))), wh = uniform(seen_by(p, over(p.group, min(w0 + 32, rows) - 1)));
    const int qi = over(p.group, min(row, rows - 1)), hh = h * G + min(row, rows - 1) - qi * G;
    const Seen seen = seen_by(p, qi);
    const u16* qr = static_cast<const u16*>(p.q) + at_row(p.qs, b, hh, qi);
    const u16* gr = static_cast<const u16*>(p.dout) + at_row(p.gs, b, hh, qi);
    bf16x8 qf[D / 16], gf[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
        if (in) {
            x = *reinterpret_cast<const u32x4*>(qr + 16 * s + 8 * half);
            y = *reinterpret_cast<const u32x4*>(gr + 16 * s + 8 * half);
        }
        qf[s] = __builtin_bit_cast(bf16x8, x);
        gf[s] = __builtin_bit_cast(bf16x8, y);
    }
    const size_t stat = ((size_t)b * p.hq + hh) * p.nq + qi;
    float lse2 = in ? p.lse[stat] * kLog2e : 0.0f;
    if (lse2 == kNegInf) lse2 = 0.0f;   // a row that sees nothing: all its weights are masked
    float dsum = 0.0f;
    if (in) {
        const long long o0 = at_row(p.os, b, hh, qi) + 8 * half;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            float o[8];
            if (p.o_bf16) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const u16*>(p.o) + o0 + 16 * s);
#pragma unroll
                for (int j = 0; j < 4; ++j) { o[2 * j] = bf16lo_to_f32(x[j]); o[2 * j + 1] = bf16hi_to_f32(x[j]); }
            } else {
                const f32x4* x = reinterpret_cast<const f32x4*>(static_cast<const float*>(p.o) + o0 + 16 * s);
#pragma unroll
                for (int j = 0; j < 4; ++j) { o[j] = x[0][j]; o[4 + j] = x[1][j]; }
            }
            const u32x4 y = __builtin_bit_cast(u32x4, gf[s]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dsum = __builtin_fmaf(bf16lo_to_f32(y[j]), o[2 * j], dsum);
                dsum = __builtin_fmaf(bf16hi_to_f32(y[j]), o[2 * j + 1], dsum);
            }
        }
    }
    dsum = half_sum(dsum);

    const u16* Kh = static_cast<const u16*>(p.k) + at_row(p.ks, b, h, 0);
    const u16* Vh = static_cast<const u16*>(p.v) + at_row(p.vs, b, h, 0);
    const uint32_t krb = (uint32_t)p.ks[2] * 2u, vrb = (uint32_t)p.vs[2] * 2u;
    uint32_t koff[LPW], voff[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
        const int slot = (wave * LPW + i) * 64 + lane, r = slot / C::CHUNKS, ch = slot % C::CHUNKS;
        const uint32_t chunk = (uint32_t)((ch ^ swz<D>(r)) * 16);
        koff[i] = (uint32_t)(r & 15) * krb + chunk;   // this wave's 16 rows of the tile
        voff[i] = (uint32_t)(r & 15) * vrb + chunk;
    }
    auto issue = [&](int v, auto stage) __attribute__((always_inline)) {
        unsigned char* ks = decltype(stage)::value == 0 ? k_st0[stream] : k_st1[stream];
        unsigned char* vs = decltype(stage)::value == 0 ? v_st0[stream] : v_st1[stream];
        const int key = tiles.at(v) * BN + 16 * wave, n = max(0, min(16, p.nk - key));
        const auto rk = make_rsrc(Kh + (n ? key * p.ks[2] : 0), rows_extent(n, krb, RB));
        const auto rv = make_rsrc(Vh + (n ? key * p.vs[2] : 0), rows_extent(n, vrb, RB));
#pragma unroll
        for (int j = 0; j < LPW; ++j) buffer_load16_to_lds(rk, ks + (wave * LPW + j) * 1024, koff[j]);
#pragma unroll
        for (int j = 0; j < LPW; ++j) buffer_load16_to_lds(rv, vs + (wave * LPW + j) * 1024, voff[j]);
    };
    const TileAddr<D> ta(lane);
    // S and dP of 32 keys, S as the exponent of the weights.
    auto scores = [&](const unsigned char* ks, const unsigned char* vs, int u, int key, f32x16& s, f32x16& dp) __attribute__((always_inline)) {
        s = f32x16{};
        dp = f32x16{};
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_rows<D>(ks, ta, u, k), qf[k], s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_rows<D>(vs, ta, u, k), gf[k], dp, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], c, -lse2);
        if (!all_see(wl, wh, sinks, key)) keep(s, seen_bits(seen, sinks, key), half);
    };
    // The tiles, with `tile` for each: pairs of turns on the ring's two stages.
    auto walk = [&](auto tile) __attribute__((always_inline)) {
        auto turn = [&](int v, auto stage, auto other) __attribute__((always_inline)) {
            pf::wait_vmcnt<0>();
            __syncthreads();
            if (v + KS < tiles.count) issue(v + KS, other);
            if (KS == 1 || v < tiles.count) tile(v, stage);
        };
        if (stream < tiles.count) issue(stream, S0{});
        for (int v = 0; v < tiles.count; v += 2 * KS) {
            turn(v + stream, S0{}, S1{});
            if (v + KS >= tiles.count) break;
            turn(v + KS + stream, S1{}, S0{});
        }
    };
    // D_i from O has the error of its bf16 numbers, |dO| |O| 2^-8 at most, and O is large and
    // dS small where a row sees few keys.  There D_i is taken from them: sum_j P_ij dP_ij,
    // exact to fp32, one more walk over one or two tiles.  (4 x 1000 causal tokens, d = 64:
    // error of dQ and dK 2.4e-3 for 2.6e-3, at the same time.  One key to a row: exact for
    // an error as large as the gradients of others.)
    if (p.o_bf16 && min(keys_seen(tl, sinks), keys_seen(th, sinks)) < kFewKeys) {
        float sum = 0.0f;
        walk([&](int v, auto stage) __attribute__((always_inline)) {
            if (!live) return;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int key = tiles.at(v) * BN + 32 * u;
                if (!any_sees(wl, wh, sinks, key)) continue;
                f32x16 s, dp;
                scores(decltype(stage)::value == 0 ? k_st0[stream] : k_st1[stream], decltype(stage)::value == 0 ? v_st0[stream] : v_st1[stream], u, key, s, dp);
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(exp2_hw(s[i]), dp[i], sum);
            }
        });
        sum = half_sum(sum);
        __syncthreads();   // every wave is through with the stages
        if constexpr (KS == 2) {
            float* x = reinterpret_cast<float*>(&k_st0[0][0]) + wave * 64 + lane;
            x[stream * QW * 64] = sum;
            __syncthreads();
            sum += x[(1 - stream) * QW * 64];
            __syncthreads();
        }
        // (Not finite: a key that the row does not see may be the cause, so O stays.)
        if (__builtin_fabsf(sum) < -kNegInf) dsum = sum;
    }
    if (in && half == 0 && stream == 0) p.dsum[stat] = dsum;

    f32x16 acc[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) acc[d] = f32x16{};
    walk([&](int v, auto stage) __attribute__((always_inline)) {
        const unsigned char* ks = decltype(stage)::value == 0 ? k_st0[stream] : k_st1[stream];
        const unsigned char* vs = decltype(stage)::value == 0 ? v_st0[stream] : v_st1[stream];
        const int k0 = tiles.at(v) * BN;
        if (!live) return;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (!any_sees(wl, wh, sinks, k0 + 32 * u)) continue;
            f32x16 s, dp;
            scores(ks, vs, u, k0 + 32 * u, s, dp);
            float ds[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] = exp2_hw(s[i]) * (dp[i] - dsum);
            bf16x8 dsb[2];
            pack16(ds, dsb);
#pragma unroll
            for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_tr<D>(ks, ta, d, 2 * u + c2), dsb[c2], acc[d], 0, 0, 0);
        }
    });
    if constexpr (KS == 2) {   // the second stream's sums, through LDS
        __syncthreads();
        float* x = reinterpret_cast<float*>(wave < 2 ? &k_st0[0][0] : &k_st1[0][0]) + (wave & 1) * (D / 2) * 64;
        if (stream == 1) {
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[(d * 16 + i) * 64 + lane] = acc[d][i];
        }
        __syncthreads();
        if (stream == 1) return;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] += x[(d * 16 + i) * 64 + lane];
    }
    if (!live) return;
    const WinGrad late = arguments_again<WinGrad>();
    const bool odd = not_finite<D>(acc) && in;
    if (in) store_row16<D>(static_cast<u16*>(late.dq) + at_row(late.dqs, b, hh, qi), half, acc, late.scale);
    const u16* Kl = static_cast<const u16*>(late.k) + at_row(late.ks, b, h, 0);
    const u16* Vl = static_cast<const u16*>(late.v) + at_row(late.vs, b, h, 0);
    for (uint32_t left = (uint32_t)__ballot(odd); left; left &= left - 1) {
        const int r = __builtin_ctz(left), i = over(late.group, w0 + r), head = h * (int)late.group.n + (w0 + r) - i * (int)late.group.n;
        const Seen see = seen_by(late, i);
        const u16* q = static_cast<const u16*>(late.q) + at_row(late.qs, b, head, i);
        const u16* g = static_cast<const u16*>(late.dout) + at_row(late.gs, b, head, i);
        const float l = __shfl(lse2, r), dd = __shfl(dsum, r);
        float o[D / 64] = {};
        for (int v = 0; v < tiles.count; ++v) {
            const int key = tiles.at(v) * BN + lane;
            const bool mine = sees(see, late.w.sinks, key);
            float w = 0.0f, ds = 0.0f;
            if (mine) pair_by_definition<D>(q, Kl + key * late.ks[2], g, Vl + key * late.vs[2], (double)late.scale * 1.4426950408889634, l, dd, w, ds);
            add_rows<D>(o, __ballot(mine), ds, [&](int j) { return Kl + (long long)(tiles.at(v) * BN + j) * late.ks[2]; });
        }
        store_lane<D>(static_cast<u16*>(late.dq) + at_row(late.dqs, b, head, i), o, late.scale);
    }
}

// ---- dK, dV ------------------------------------------------------------------

constexpr int KW = 8;             // waves

// Four numbers with their upper 24 bits in three registers: the fourth in the others'
// low bytes, which are left there when the three are used (2^-16 of them).
__device__ __forceinline__ void pack24(const float (&w)[4], uint32_t (&x)[3]) {
    const uint32_t last = __float_as_uint(w[3]);
    x[0] = __builtin_amdgcn_perm(last, __float_as_uint(w[0]), 0x03020107u);
    x[1] = __builtin_amdgcn_perm(last, __float_as_uint(w[1]), 0x03020106u);
    x[2] = __builtin_amdgcn_perm(last, __float_as_uint(w[2]), 0x03020105u);
}
__device__ __forceinline__ void unpack24(const uint32_t (&x)[3], float (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i] = __uint_as_float(x[i]);
    w[3] = __uint_as_float(__builtin_amdgcn_perm(__builtin_amdgcn_perm(x[0], x[1], 0x04000c0cu), x[2], 0x0706000cu));
}
constexpr int KT = kWinKeyTile;   // keys per workgroup
constexpr int SR = kWinStage;     // queries per stage

// The queries that see a key: lo .. hi.
struct Span {
    int lo, hi;
};
__device__ __forceinline__ Span seen_of_key(const WinGrad& p, int key) {
    const long long off = (long long)p.nk - p.nq;
    Span s;
    s.lo = p.w.right == kNoLimit ? 0 : (int)max(0ll, min((long long)p.nq, key - off - p.w.right));
    s.hi = p.w.left == kNoLimit || key < p.w.sinks ? p.nq - 1 : (int)max(-1ll, min((long long)p.nq - 1, key - off + p.w.left));
    return s;
}

// The stages of one workgroup: `count` of the list that has, head after head, the
// stages first .. first + each - 1.
struct Stages {
    int first, each, begin, count;
};

__device__ __forceinline__ Near near_of(const WinGrad& p, int kt) { return near_stages(p.w, p.nq, p.nk, p.chunks > 0, kt); }
__device__ __forceinline__ int parts_of(const WinGrad& p, const Near& x) { return moa::parts_of(p.parts, x.each * (int)p.group.n, p.part_stages); }

// Partial sums: of every tile room for all parts, of the first keys' tiles those of
// their chunks behind them; none of a tile with one part and no chunks.  The first
// ones of tile kt of key/value head bh.
__device__ __forceinline__ size_t first_part(const WinGrad& p, int sink_tiles, int bh, int kt) {
    const int key_tiles = (p.nk + KT - 1) / KT, far = p.parts + p.chunks, near = p.parts > 1 ? p.parts : 0;
    const size_t all = (size_t)sink_tiles * far + (size_t)(key_tiles - sink_tiles) * near;
    return bh * all + (kt < sink_tiles ? (size_t)kt * far : (size_t)sink_tiles * far + (size_t)(kt - sink_tiles) * near);
}

template <int D>
__global__ __launch_bounds__(KW * 64, 1) void win_dkdv_kernel(WinGrad p, float c, int sink_tiles) {
    using C = Cfg<D>;
    constexpr uint32_t RB = C::ROW_BYTES;
    constexpr int U = SR / 32;                             // steps per stage
    constexpr int LPS = SR * C::ROW_BYTES / (KW * 1024);   // 16-byte loads per lane per stage of Q or dO
    // One array per ring slot: the compiler tracks direct-to-LDS loads per object.
    __shared__ __attribute__((aligned(1024))) unsigned char q_0[SR * C::ROW_BYTES], q_1[SR * C::ROW_BYTES], q_2[SR * C::ROW_BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char g_0[SR * C::ROW_BYTES], g_1[SR * C::ROW_BYTES], g_2[SR * C::ROW_BYTES];
    // Exchanged weights: [stage parity][pair][step][register quad][lane].
    __shared__ __attribute__((aligned(1024))) u32x4 p_x[2][4][U][3][64];
    __shared__ __attribute__((aligned(16))) float l_r[3][2][SR];   // [slot][lse2, D][query]

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int role = wave >> 2, pair = wave & 3;   // role 0: P and dV; role 1: dS and dK
    const int col = lane & 31, half = lane >> 5;
    const int G = (int)p.group.n, item = over(p.per_item, blockIdx.x);
    const int bh = blockIdx.x - item * (int)p.per_item.n, b = over(p.heads, bh), h = bh - b * p.hk;
    // Items of a head: the parts of every tile's queries whose windows reach it, then
    // the chunks of the far queries of the first keys' tiles, short ones that fill up
    // the last round.
    const bool far = item >= p.near_items;
    int kt = item, cut = 0;
    if (far) {
        kt = (item - p.near_items) / p.chunks;
        cut = (item - p.near_items) % p.chunks;
    } else if (p.parts > 1) {
        // The tile among whose parts the item is: a tile a lane.  (A part's number beyond
        // its tile's, with room for all parts in the grid, left whole shader engines idle:
        // 31 -> 36 us for the parts that take 25 without gaps.)
        const int key_tiles = (p.nk + KT - 1) / KT;
        for (int t0 = 0, before = 0;; t0 += 64) {
            if (t0 >= key_tiles) return;
            const int t = t0 + lane, n = t < key_tiles ? parts_of(p, near_of(p, t)) : 0;
            int sum = n;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) {
                const int below = __shfl_up(sum, s);
                if (lane >= s) sum += below;
            }
            const uint64_t past = __ballot(before + sum > item);
            if (past) {
                const int l = __builtin_ctzll(past);
                kt = t0 + l;
                cut = item - before - __builtin_amdgcn_readlane(sum - n, l);
                break;
            }
            before += __builtin_amdgcn_readlane(sum, 63);
        }
    }
    const int k0 = kt * KT;
    const bool split = kt < sink_tiles && p.chunks > 0;

    Stages st;
    {
        const Near x = near_of(p, kt);
        st.first = x.first;
        st.each = x.each;
        if (far) {
            st.first = max(x.first, (x.near_hi + SR) / SR);   // the stage behind near_hi's
            st.each = max(0, (p.nq + SR - 1) / SR - st.first);
        }
        const int cuts = far ? p.chunks : parts_of(p, x);
        const int all = st.each * G, per = (all + cuts - 1) / cuts;
        st.begin = min(all, cut * per);
        st.count = min(per, all - st.begin);
    }
    const int n_stages = st.count;

    const int w0 = k0 + pair * 32, key = w0 + col;   // this pair's keys, this lane's
    const Span mine = seen_of_key(p, min(key, p.nk - 1));
    // Queries that a key of the pair's is seen by, and those that see all of them.
    // (the first key behind the sinks has the earliest end)
    const Span wa = seen_of_key(p, min(w0, p.nk - 1)), wb = seen_of_key(p, min(w0 + 31, p.nk - 1));
    const Span wc = seen_of_key(p, min(min(max(w0, p.w.sinks), w0 + 31), p.nk - 1));
    const int some_lo = __builtin_amdgcn_readfirstlane(wa.lo), all_lo = __builtin_amdgcn_readfirstlane(wb.lo);
    const int some_hi = __builtin_amdgcn_readfirstlane(max(wa.hi, wb.hi));
    const int all_hi = __builtin_amdgcn_readfirstlane(min(wa.hi, wc.hi));
    const bool live = w0 < p.nk && !(far && w0 >= p.w.sinks);

    const uint32_t qrb = (uint32_t)p.qs[2] * 2u, grb = (uint32_t)p.gs[2] * 2u;
    uint32_t qoff[LPS], goff[LPS];
#pragma unroll
    for (int i = 0; i < LPS; ++i) {
        const int slot = (wave * LPS + i) * 64 + lane, r = slot / C::CHUNKS, ch = slot % C::CHUNKS;
        const uint32_t at = (uint32_t)((ch ^ swz<D>(r)) * 16);
        qoff[i] = (uint32_t)r * qrb + at;
        goff[i] = (uint32_t)r * grb + at;
    }
    const TileAddr<D> ta(lane);

    // K (role 0) or V (role 1) of this lane's key: B operands.
    bf16x8 kvf[D / 16];
    {
        const u16* src = role == 0 ? static_cast<const u16*>(p.k) + at_row(p.ks, b, h, 0) + key * p.ks[2]
                                   : static_cast<const u16*>(p.v) + at_row(p.vs, b, h, 0) + key * p.vs[2];
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (key < p.nk) x = *reinterpret_cast<const u32x4*>(src + 16 * s + 8 * half);
            kvf[s] = __builtin_bit_cast(bf16x8, x);
        }
    }
    f32x16 acc[D / 32];     // dV^T (role 0) or dK^T (role 1)
#pragma unroll
    for (int d = 0; d < D / 32; ++d) acc[d] = f32x16{};

    // Whether the pair has anything to do in the stage from query q0 on.  (Tested for
    // each half of it, the steps did not overlap.)
    const auto wanted = [&](int q0) { return live && q0 <= some_hi && q0 + SR > some_lo; };

    auto step_a = [&](const unsigned char* qs, const unsigned char* gs, const float* ls, u32x4* px, int u, int q0)
                      __attribute__((always_inline)) {
        f32x16 s = f32x16{};
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_rows<D>(qs, ta, u, k), kvf[k], s, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 l4 = *reinterpret_cast<const float4*>(ls + 32 * u + 8 * g + 4 * half);
            const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * g + r] = __builtin_fmaf(s[4 * g + r], c, -lv[r]);
        }
        if (q0 < all_lo || q0 + 31 > all_hi) keep(s, ones(mine.hi + 1 - q0) & ~ones(mine.lo - q0), half);
        float w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = exp2_hw(s[i]);
        u32x4 x[3];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float four[4] = {w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]};
            uint32_t y[3];
            pack24(four, y);
#pragma unroll
            for (int i = 0; i < 3; ++i) x[(3 * g + i) / 4][(3 * g + i) % 4] = y[i];
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) px[i * 64 + lane] = x[i];
        bf16x8 pb[2];
        pack16(w, pb);
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_tr<D>(gs, ta, d, 2 * u + c2), pb[c2], acc[d], 0, 0, 0);
    };
    auto step_b = [&](const unsigned char* qs, const unsigned char* gs, const float* dv, const u32x4* px, int u)
                      __attribute__((always_inline)) {
        f32x16 dp = f32x16{};
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_rows<D>(gs, ta, u, k), kvf[k], dp, 0, 0, 0);
        u32x4 x[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) x[i] = px[i * 64 + lane];
        float ds[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint32_t y[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) y[i] = x[(3 * g + i) / 4][(3 * g + i) % 4];
            float w[4];
            unpack24(y, w);
            const float4 d4 = *reinterpret_cast<const float4*>(dv + 32 * u + 8 * g + 4 * half);
            const float dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) ds[4 * g + r] = w[r] * (dp[4 * g + r] - dd[r]);
        }
        bf16x8 dsb[2];
        pack16(ds, dsb);
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(stage_tr<D>(qs, ta, d, 2 * u + c2), dsb[c2], acc[d], 0, 0, 0);
    };

    // The list's stages one after the other: head `hh`, stage `at`.
    struct Cursor {
        int hh, at;
    };
    const auto start = [&]() {
        const int g = st.each ? st.begin / st.each : 0;
        return Cursor{h * G + g, st.first + st.begin - g * st.each};
    };
    const auto next = [&](Cursor& x) {
        if (++x.at == st.first + st.each) {
            x.at = st.first;
            ++x.hh;
        }
    };
    Cursor load = start(), work = load;
    const float* stats = role == 0 ? p.lse : p.dsum;
    float sx = 0.0f;
    auto issue = [&](unsigned char* qd, unsigned char* gd) __attribute__((always_inline)) {
        const int q0 = load.at * SR, n = min(SR, p.nq - q0);
        const auto rq = make_rsrc(static_cast<const u16*>(p.q) + at_row(p.qs, b, load.hh, q0), rows_extent(n, qrb, RB));
        const auto rg = make_rsrc(static_cast<const u16*>(p.dout) + at_row(p.gs, b, load.hh, q0), rows_extent(n, grb, RB));
#pragma unroll
        for (int i = 0; i < LPS; ++i) buffer_load16_to_lds(rq, qd + (wave * LPS + i) * 1024, qoff[i]);
#pragma unroll
        for (int i = 0; i < LPS; ++i) buffer_load16_to_lds(rg, gd + (wave * LPS + i) * 1024, goff[i]);
        // LSE or D of the stage's queries, a query a lane (behind the last: masked).
        sx = stats[((size_t)b * p.hq + load.hh) * p.nq + min(q0 + lane, p.nq - 1)];
        next(load);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    const auto q_slot = [&](auto s) -> unsigned char* { return decltype(s)::value == 0 ? q_0 : decltype(s)::value == 1 ? q_1 : q_2; };
    const auto g_slot = [&](auto s) -> unsigned char* { return decltype(s)::value == 0 ? g_0 : decltype(s)::value == 1 ? g_1 : g_2; };
    // Iteration j: stage j is in slot j % 3 after the barrier.  Role 0 works on it,
    // role 1 on the one before, whose weights role 0 wrote in iteration j - 1; the
    // loads of stage j + 1 start into the slot whose last reader is done.
    auto advance = [&](int j, auto slot, auto after) __attribute__((always_inline)) {
        if (j < n_stages && pair == 0) l_r[decltype(slot)::value][role][lane] = role == 0 ? sx * kLog2e : sx;
        pf::wait_vmcnt<0>();
        pf::wait_lgkmcnt0();
        pf::barrier_no_fence();
        if (j + 1 < n_stages) issue(q_slot(after), g_slot(after));
    };
    auto iteration_a = [&](int j, auto slot, auto after) __attribute__((always_inline)) {
        advance(j, slot, after);
        if (j >= n_stages) return;
        if (wanted(work.at * SR))
#pragma unroll
            for (int u = 0; u < U; ++u)
                step_a(q_slot(slot), g_slot(slot), l_r[decltype(slot)::value][0], &p_x[j & 1][pair][u][0][0], u, work.at * SR + 32 * u);
        next(work);
    };
    auto iteration_b = [&](int j, auto slot, auto after, auto before) __attribute__((always_inline)) {
        advance(j, slot, after);
        if (j == 0) return;
        if (wanted(work.at * SR))
#pragma unroll
            for (int u = 0; u < U; ++u)
                step_b(q_slot(before), g_slot(before), l_r[decltype(before)::value][1], &p_x[(j - 1) & 1][pair][u][0][0], u);
        next(work);
    };
    if (n_stages > 0) {
        issue(q_0, g_0);
        if (role == 0) {
            for (int j = 0; j <= n_stages; j += 3) {
                iteration_a(j, I0{}, I1{});
                if (j + 1 > n_stages) break;
                iteration_a(j + 1, I1{}, I2{});
                if (j + 2 > n_stages) break;
                iteration_a(j + 2, I2{}, I0{});
            }
        } else {
            for (int j = 0; j <= n_stages; j += 3) {
                iteration_b(j, I0{}, I1{}, I2{});
                if (j + 1 > n_stages) break;
                iteration_b(j + 1, I1{}, I2{}, I0{});
                if (j + 2 > n_stages) break;
                iteration_b(j + 2, I2{}, I0{}, I1{});
            }
        }
    }
    if (!live) return;

    const WinGrad late = arguments_again<WinGrad>();
    // Where this wave's rows go: the gradient, or the sums [2][KT][D] (dV first) of a
    // part or chunk.
    const bool partial = late.parts > 1 || split;
    float* part = nullptr;
    if (partial) part = late.part + ((first_part(late, sink_tiles, bh, kt) + (far ? late.parts : 0) + cut) * 2 + role) * KT * D;
    u16* out = role == 0 ? static_cast<u16*>(late.dv) + at_row(late.dvs, b, h, 0) : static_cast<u16*>(late.dk) + at_row(late.dks, b, h, 0);
    const long long out_row = role == 0 ? late.dvs[2] : late.dks[2];
    const float mul = role == 0 ? 1.0f : late.scale;
    const bool odd = not_finite<D>(acc) && key < late.nk;
    if (key < late.nk) {
        if (partial) store_row16<D>(part + (size_t)(key - k0) * D, half, acc, mul);
        else store_row16<D>(out + key * out_row, half, acc, mul);
    }
    for (uint32_t left = (uint32_t)__ballot(odd); left; left &= left - 1) {
        const int at = w0 + __builtin_ctz(left);
        const Span span = seen_of_key(late, at);
        const u16* k = static_cast<const u16*>(late.k) + at_row(late.ks, b, h, at);
        const u16* v = static_cast<const u16*>(late.v) + at_row(late.vs, b, h, at);
        float o[D / 64] = {};
        Cursor x = start();
        for (int j = 0; j < n_stages; ++j, next(x)) {
            const int qi = x.at * SR + lane;
            const bool seen = qi < late.nq && qi >= span.lo && qi <= span.hi;
            const u16* q0 = static_cast<const u16*>(late.q) + at_row(late.qs, b, x.hh, x.at * SR);
            const u16* g0 = static_cast<const u16*>(late.dout) + at_row(late.gs, b, x.hh, x.at * SR);
            float w = 0.0f, ds = 0.0f;
            if (seen) {
                const size_t stat = ((size_t)b * late.hq + x.hh) * late.nq + qi;
                pair_by_definition<D>(k, q0 + lane * late.qs[2], v, g0 + lane * late.gs[2], (double)late.scale * 1.4426950408889634,
                                      late.lse[stat] * kLog2e, late.dsum[stat], w, ds);
            }
            add_rows<D>(o, __ballot(seen), role == 0 ? w : ds, [&](int i) { return role == 0 ? g0 + i * late.gs[2] : q0 + i * late.qs[2]; });
        }
        if (partial) {
            for (int e = 0; e < D / 64; ++e) part[(size_t)(at - k0) * D + (D / 64) * lane + e] = o[e] * mul;
        } else {
            store_lane<D>(out + at * out_row, o, mul);
        }
    }
}

// Adds the sums of a tile's parts and chunks, in their order: four elements a thread.
template <int D>
__global__ __launch_bounds__(256) void win_join_kernel(WinGrad p, int tiles, int sink_tiles) {
    constexpr int PER = KT * D / 4 / 256;   // workgroups per tile and tensor
    int x = blockIdx.x;
    const int e4 = (x % PER) * 256 + threadIdx.x; x /= PER;
    const int role = x & 1; x >>= 1;
    const int kt = x % tiles, bh = x / tiles, b = bh / p.hk, h = bh - b * p.hk;
    const int key = kt * KT + e4 / (D / 4), e = e4 % (D / 4) * 4;
    if (key >= p.nk) return;
    // chunks hold sums of the first keys alone
    const int near = parts_of(p, near_of(p, kt));
    const int n = near + (kt < sink_tiles && key < p.w.sinks ? p.chunks : 0), over = p.parts - near;
    const float* at = p.part + (first_part(p, sink_tiles, bh, kt) * 2 + role) * KT * D + (size_t)e4 * 4;
    f32x4 sum = {0, 0, 0, 0};
    for (int i = 0; i < n; i += 4) {
        f32x4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int x = min(i + u, n - 1);
            y[u] = *reinterpret_cast<const f32x4*>(at + (size_t)(x < near ? x : x + over) * 2 * KT * D);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u < n) sum += y[u];
    }
    u16* out = role == 0 ? static_cast<u16*>(p.dv) + at_row(p.dvs, b, h, key) : static_cast<u16*>(p.dk) + at_row(p.dks, b, h, key);
    *reinterpret_cast<uint2*>(out + e) = make_uint2(pack2(sum[0], sum[1]), pack2(sum[2], sum[3]));
}

template <int D>
hipError_t go(WinGrad p, hipStream_t stream) {
    const int groups = p.B * p.hk;
    p.per_item = div_by(groups);
    p.heads = div_by(p.hk);
    if (p.hq > 0) p.group = div_by(p.hq / p.hk);   // else 0: no queries
    const float c = p.scale * kLog2e;
    if (p.nq > 0 && p.hq > 0) {
        const long long rows = (long long)p.nq * (p.hq / p.hk);
        const int tiles = (int)((rows + QROWS - 1) / QROWS);
        const unsigned blocks = (unsigned)groups * tiles;
        const hipError_t e = blocks <= 256
            ? launch_kernel(win_dq_kernel<D, 2>, dim3(blocks), dim3(2 * QW * 64), stream, p, c, tiles)
            : launch_kernel(win_dq_kernel<D, 1>, dim3(blocks), dim3(QW * 64), stream, p, c, tiles);
        if (e != hipSuccess) return e;
    }
    if (p.nk == 0) return hipSuccess;
    const int key_tiles = (p.nk + KT - 1) / KT, sink_tiles = p.chunks ? win_sink_tiles(p.w, p.nk) : 0;
    p.near_items = key_tiles;
    if (p.parts > 1) {
        p.near_items = 0;
        for (int t = 0; t < key_tiles; ++t)
            p.near_items += moa::parts_of(p.parts, near_stages(p.w, p.nq, p.nk, p.chunks > 0, t).each * (p.hq / p.hk), p.part_stages);
    }
    const int items = p.near_items + sink_tiles * p.chunks;
    hipError_t e = launch_kernel(win_dkdv_kernel<D>, dim3((unsigned)groups * items), dim3(KW * 64), stream, p, c, sink_tiles);
    const int joined = p.parts > 1 ? key_tiles : sink_tiles;
    if (e != hipSuccess || !joined) return e;
    return launch_kernel(win_join_kernel<D>, dim3((unsigned)groups * joined * 2 * (KT * D / 4 / 256)), dim3(256), stream, p, joined, sink_tiles);
}

}  // namespace

hipError_t launch_win_bwd(const WinGrad& p, hipStream_t stream) {
    return p.d == 64 ? go<64>(p, stream) : go<128>(p, stream);
}

}  // namespace moa
