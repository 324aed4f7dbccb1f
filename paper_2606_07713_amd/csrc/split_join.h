// Exact join of the key splits of attention rows.
#pragma once

#include "device_common.h"

namespace moa {

// Rows [B][hq][n] with partial states: [row][splits][d] fp32, then
// [row][splits][2] (reference in log2 units, sum).
struct SplitJoin {
    const float* ws;
    void* o;
    float* lse;             // nullable
    const int* new_lens;    // rows of each sequence that are real, or null: n
    long long os[3];
    int B, hq, n, splits;
    bool out_bf16;
};

// States that ask for their row to be done another way have a reference of NaN; no state
// of these kernels does.
struct NoRows {
    static constexpr bool any = false;
};

// Splits without a visible key have a reference of -inf and sums of 0.  Sums of others
// need not be near their references: one of 2^120 against the lowest reference counts
// beside one of 2^-40 against the highest, so references are met in two factors.
//
// With few rows the pass is a chain of load latencies, so W = 4 waves share a row of
// more than 4 splits, each takes U of its splits at a time, and all of these loads are
// in flight together: up to 32 splits cost one latency.  From 2048 rows on there
// are enough waves with one for each (us by one wave a row and by four, d = 128:
// 512 rows of 16 splits 4.8 and 3.9, 1024 of 16 5.4 and 4.8, 1024 of 5 4.0 and 4.3;
// 2048 of 16 5.9 and 6.7, 8192 of 8 7.4 and 17.3; 512 of 4 3.3 and 3.9).
template <int D, int W, typename Again>
__global__ __launch_bounds__(256) void split_join_kernel(SplitJoin p, Again again) {
    constexpr int PER = D / 64, U = W == 1 ? 4 : 8;
    typedef float vec __attribute__((ext_vector_type(PER)));
    __shared__ vec part[4][64];
    __shared__ float part_m[4], part_l[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const long long row = (long long)blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
    if (row >= (long long)p.B * p.hq * p.n) return;
    const int i = (int)(row % p.n);
    const long long bh = row / p.n;
    const int b = (int)(bh / p.hq), hh = (int)(bh - (long long)b * p.hq);
    const vec* acc = reinterpret_cast<const vec*>(p.ws + (size_t)row * p.splits * D) + lane;
    const float* ml = p.ws + (size_t)p.B * p.hq * p.n * p.splits * D + (size_t)row * p.splits * 2;
    float M = kNegInf, L = 0.0f;
    vec o = 0.0f;
    bool asks = false;
    for (int s0 = W == 1 ? 0 : wave; s0 < p.splits; s0 += U * W) {
        float ms[U], ls[U], top = M;
        vec a[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u * W, p.splits - 1);
            ms[u] = ml[2 * s];
            ls[u] = ml[2 * s + 1];
            a[u] = acc[(size_t)s * 64];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (Again::any) asks |= ms[u] != ms[u];
            if (s0 + u * W >= p.splits) ms[u] = kNegInf;
            top = fmaxf(top, ms[u]);
        }
        if (M != kNegInf) {   // (else nothing yet)
            const TwoFactors alpha(M - top);
            L = alpha.of(L);
            o = alpha.of(o);
        }
        M = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (ms[u] == kNegInf) continue;
            const TwoFactors w(ms[u] - M);
            L += w.of(ls[u]);
            o += w.of(a[u]);
        }
    }
    // nothing was written for rows behind the new tokens, and nothing is
    if (p.new_lens && i >= min(max(p.new_lens[b], 0), p.n)) return;
    if constexpr (W > 1) {
        part[wave][lane] = o;
        if (lane == 0) { part_m[wave] = asks ? __builtin_nanf("") : M; part_l[wave] = L; }
        __syncthreads();
        if (wave != 0) return;
        if constexpr (Again::any)
#pragma unroll
            for (int w = 0; w < 4; ++w) asks |= part_m[w] != part_m[w];
        const float top = fmaxf(fmaxf(part_m[0], part_m[1]), fmaxf(part_m[2], part_m[3]));
        L = 0.0f;
        o = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (part_m[w] == kNegInf) continue;
            const TwoFactors f(part_m[w] - top);
            L += f.of(part_l[w]);
            o += f.of(part[w][lane]);
        }
        M = top;
    }
    if constexpr (Again::any)
        if (wave_any(asks)) {
            again.template row<D>(b, hh, i);
            return;
        }
    const bool none = M == kNegInf;   // no visible key
    o *= none ? 0.0f : 1.0f / L;
    const long long to = b * p.os[0] + hh * p.os[1] + i * p.os[2] + PER * lane;
    if (p.out_bf16) {
        typedef __bf16 out __attribute__((ext_vector_type(PER)));
        *reinterpret_cast<out*>(static_cast<__bf16*>(p.o) + to) = __builtin_convertvector(o, out);
    } else {
        *reinterpret_cast<vec*>(static_cast<float*>(p.o) + to) = o;
    }
    if (!p.lse || lane != 0) return;
    float whole = M, of = L;
    if constexpr (Again::any)
        if (L < 0x1p-20f && L > 0.0f) {   // a high reference and a small sum: what they cancel is taken first
            const int e = __builtin_amdgcn_frexp_expf(L);
            whole += (float)e;
            of = ldexpf(L, -e);
        }
    p.lse[row] = none ? kNegInf : (whole + __log2f(of)) * kLn2;
}

template <int D, typename Again = NoRows>
hipError_t launch_split_join(const SplitJoin& p, hipStream_t stream, const Again& again = {}) {
    const long long all = (long long)p.B * p.hq * p.n;
    if (p.splits <= 4 || all >= 2048)
        return launch_kernel(split_join_kernel<D, 1, Again>, dim3((unsigned)((all + 3) / 4)), dim3(256), stream, p, again);
    return launch_kernel(split_join_kernel<D, 4, Again>, dim3((unsigned)all), dim3(256), stream, p, again);
}

}  // namespace moa
