// Device-side pieces of the norms of heads with the rotation by position, which
// rope.hip and the appending to a paged cache (paged.hip) share.
#pragma once

#include <cfloat>

#include "device_common.h"
#include "rope.h"

namespace moa {
namespace rope {

constexpr int THREADS = 256;
// The rows written are not read again here; stores that pass the caches by
// leave them to the rows read (16 heads each of 8192 tokens, bf16, d = 128: 33.2
// -> 29.0 us, the gradients 53.3 -> 44.8; loads past the caches gained nothing).
__device__ __forceinline__ void store16(void* p, u32x4 v) { __builtin_nontemporal_store(v, static_cast<u32x4*>(p)); }

// Eight elements of a row as they are stored.
template <typename T>
struct Chunk;
template <>
struct Chunk<u16> {
    uint4 a;
    __device__ __forceinline__ void load(const u16* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = bf16lo_to_f32(a.x); f[1] = bf16hi_to_f32(a.x);
        f[2] = bf16lo_to_f32(a.y); f[3] = bf16hi_to_f32(a.y);
        f[4] = bf16lo_to_f32(a.z); f[5] = bf16hi_to_f32(a.z);
        f[6] = bf16lo_to_f32(a.w); f[7] = bf16hi_to_f32(a.w);
    }
    __device__ __forceinline__ void set(const float (&f)[8]) { a = pack(f); }
    __device__ __forceinline__ Chunk from_lane(int lane) const {
        Chunk r;
        r.a = make_uint4(__shfl(a.x, lane), __shfl(a.y, lane), __shfl(a.z, lane), __shfl(a.w, lane));
        return r;
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2 t = {(__bf16)f[2 * i], (__bf16)f[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void store(u16* p, const float (&f)[8]) {
        store16(p, __builtin_bit_cast(u32x4, pack(f)));
    }
};
template <>
struct Chunk<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ Chunk from_lane(int lane) const {
        Chunk r;
        r.a = make_float4(__shfl(a.x, lane), __shfl(a.y, lane), __shfl(a.z, lane), __shfl(a.w, lane));
        r.b = make_float4(__shfl(b.x, lane), __shfl(b.y, lane), __shfl(b.z, lane), __shfl(b.w, lane));
        return r;
    }
    static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
        store16(p, __builtin_bit_cast(u32x4, make_float4(f[0], f[1], f[2], f[3])));
        store16(p + 4, __builtin_bit_cast(u32x4, make_float4(f[4], f[5], f[6], f[7])));
    }
};

// at * freq / (2 pi) less the nearest whole number.  Both products' rounding errors
// and the constant's second half are carried along: of an angle of 2^40 rad
// fp64's own rounding would be off by 2^-12.
__device__ __forceinline__ double part_of_turn(double at, double freq) {
    constexpr double HI = 0x1.45f306dc9c883p-3, LO = -0x1.6b01ec5417056p-57;   // 1 / (2 pi)
    const double angle = at * freq, rest = fma(at, freq, -angle);
    double part = fma(angle, HI, -rint(angle * HI));
    part = fma(angle, LO, part);
    part = fma(rest, HI, part);
    return part - rint(part);
}

// cos and sin of the rot/2 pairs of the workgroup's tokens t0 .. t0 + tb - 1; place:
// a token's position where none are given.
template <typename F>
__device__ __forceinline__ void take_angles(const RopeProblem& p, float2* cs, int t0, int tb, int tokens, F place) {
    const int pairs = p.rot >> 1;
    for (int i = threadIdx.x; i < tb * pairs; i += THREADS) {
        const int t = i / pairs, pr = i - t * pairs, tok = t0 + t;
        if (tok >= tokens) break;
        int axis = 0;
        for (int a = 1; a < p.axes; ++a) axis = pr >= p.first[a] ? a : axis;
        const long long at = p.pos ? p.pos[(long long)axis * tokens + tok] : place(tok);
        float s, c;
        sincospif((float)(2.0 * part_of_turn((double)at, (double)p.freq[pr])), &s, &c);
        cs[i] = make_float2(c, s);
    }
}

// This lane's share of a token's rotation: for its elements 8 j .. 8 j + 7 the
// cosine and the signed sine (of element e: y_e = t_e c_e + t_e' s_e), 1 and 0
// behind the rotated ones; the lane that holds the partners; `turned`: whether
// this lane's elements are rotated at all.
template <bool IL>
struct Turn {
    float c[8], s[8];
    int partner;
    bool turned;
    __device__ __forceinline__ void set(const RopeProblem& p, const float2* cs, int j, int lane) {
        const int half = p.rot >> 4;   // lanes per half of the rotated elements
        turned = 8 * j < p.rot;
        const bool upper = !IL && turned && j >= half;
        partner = IL || !turned ? lane : upper ? lane - half : lane + half;
        const int first = IL ? 4 * j : 8 * (upper ? j - half : j);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 v = turned ? cs[first + (IL ? e >> 1 : e)] : make_float2(1.0f, 0.0f);
            c[e] = v.x;
            s[e] = (IL ? (e & 1) != 0 : upper) ? v.y : -v.y;
        }
    }
    // The partners' values of this lane's eight.
    template <typename T>
    __device__ __forceinline__ void partners(const Chunk<T>& x, const float (&own)[8], float (&o)[8]) const {
        if constexpr (IL) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = own[e ^ 1];
        } else {
            x.from_lane(partner).get(o);
        }
        // behind the rotated elements the factor is 0: an infinity there has no part in it
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = turned ? o[e] : 0.0f;
    }
};

// Mean of a row's squares; f: this lane's elements.
template <int LPR>
__device__ __forceinline__ float mean_square(const float (&f)[8]) {
    float sq = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(f[e], f[e], sq);
    return group_sum<LPR>(sq) * (1.0f / (8 * LPR));
}

// Whether fp32 held the terms of m, a mean of squares and eps, with all their
// digits.  It does not in rows below 2^-45 without an eps that hides them and in
// rows of 2^60 and more; such rows are done again, divided by a power of two.
__device__ __forceinline__ bool in_range(float m) { return m > 0x1p-90f && m < 0x1p120f; }

// Divides a row x by 2^down, which brings the larger of its largest element and
// sqrt(eps) near 1 (elements that become subnormal by it are 2^-126 of that).
// With r = 1 / sqrt(mean square + eps / 4^down) of the divided row, r x is the
// norm, and 1 / sqrt of the undivided row is r 2^-down.
template <int LPR, typename T>
__device__ __forceinline__ void divide(Chunk<T>& x, float eps, float& r, int& down) {
    constexpr int NONE = -200;
    float f[8], top = 0.0f;
    x.get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
#pragma unroll
    for (int k = 1; k < LPR; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    const int of_eps = eps > 0.0f ? (__builtin_amdgcn_frexp_expf(eps) + 1) >> 1 : NONE;
    const int of_top = top > FLT_MAX ? 128 : top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : NONE;
    down = max(of_eps, of_top);
    down = down == NONE ? 0 : down;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = ldexpf(f[e], -down);
    x.set(f);
    r = __builtin_amdgcn_rsqf(mean_square<LPR>(f) + ldexpf(eps, -2 * down));
}

// This lane's eight weights of tensor ts (1 without a norm).
__device__ __forceinline__ void load_weights(const RopeProblem& p, int ts, int j, float (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    if (!p.w[ts]) return;
    if (p.w_bf16) {
        Chunk<u16> c;
        c.load(static_cast<const u16*>(p.w[ts]) + 8 * j);
        c.get(w);
    } else {
        Chunk<float> c;
        c.load(static_cast<const float*>(p.w[ts]) + 8 * j);
        c.get(w);
    }
}

}  // namespace rope
}  // namespace moa
