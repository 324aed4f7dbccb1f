// Norms of queries and keys for each head with the rotation by position, and
// the gradients (moa_rope.h has the formulas).
//
// Each row of d elements is read once and written once and takes about ten
// operations an element, so device memory bounds it.  A group of d/8 lanes
// holds a row, eight elements a lane; the sum of squares is a reduction inside
// the group.  The rotation is folded with the weight: of a rotated element e
// with partner e' (the other element of its pair)
//   y_e = r (x_e A_e + x_e' B_e),  A_e = w_e cos,  B_e = -/+ w_e' sin,
// and A and B depend on the token only, so a group keeps its token while it
// walks over heads and holds A and B in registers.  The sines and cosines of a
// workgroup's tokens are taken once, by all its threads, into LDS: fp64 angles,
// reduced to one turn (fp32 angles of position 10^6 would be off by 0.06).
// Partners are eight-element chunks of another lane of the group (rot/2 is a
// multiple of 8), or neighbours in the same lane when pairs are interleaved.
#include "device_common.h"
#include "rope.h"

namespace moa {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_TB = 16;   // tokens per workgroup at a time

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
    __device__ __forceinline__ Chunk from_lane(int lane) const {
        Chunk r;
        r.a = make_uint4(__shfl(a.x, lane), __shfl(a.y, lane), __shfl(a.z, lane), __shfl(a.w, lane));
        return r;
    }
    static __device__ __forceinline__ void store(u16* p, const float (&f)[8]) {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2 t = {(__bf16)f[2 * i], (__bf16)f[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
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
    __device__ __forceinline__ Chunk from_lane(int lane) const {
        Chunk r;
        r.a = make_float4(__shfl(a.x, lane), __shfl(a.y, lane), __shfl(a.z, lane), __shfl(a.w, lane));
        r.b = make_float4(__shfl(b.x, lane), __shfl(b.y, lane), __shfl(b.z, lane), __shfl(b.w, lane));
        return r;
    }
    static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
};

// cos and sin of the rot/2 pairs of the workgroup's tokens t0 .. t0 + tb - 1.
__device__ __forceinline__ void take_angles(const RopeProblem& p, float2* cs, int t0, int tb, int tokens) {
    const int pairs = p.rot >> 1;
    for (int i = threadIdx.x; i < tb * pairs; i += THREADS) {
        const int t = i / pairs, pr = i - t * pairs, tok = t0 + t;
        if (tok >= tokens) break;
        int axis = 0;
        for (int a = 1; a < p.axes; ++a) axis = pr >= p.first[a] ? a : axis;
        const long long at = p.pos ? p.pos[(long long)axis * tokens + tok] : tok % p.N;
        const double turns = (double)at * (double)p.freq[pr] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
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

__device__ __forceinline__ void load_weights(const RopeProblem& p, int ts, int e0, float (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        w[e] = !p.w[ts] ? 1.0f
               : p.w_bf16 ? __uint_as_float((uint32_t)static_cast<const u16*>(p.w[ts])[e0 + e] << 16)
                          : static_cast<const float*>(p.w[ts])[e0 + e];
}

template <typename T, int D, bool IL>
__global__ __launch_bounds__(THREADS) void rope_fwd_kernel(RopeProblem p, int log_tb, int heads_per_block) {
    constexpr int LPR = D / 8, GROUPS = THREADS / LPR, U = 2;
    __shared__ float2 cs[MAX_TB * D / 2];
    const int tokens = p.B * p.N, tb = 1 << log_tb, t0 = blockIdx.x << log_tb;
    take_angles(p, cs, t0, tb, tokens);
    __syncthreads();
    const int j = threadIdx.x % LPR, grp = threadIdx.x / LPR, lane = threadIdx.x & 63;
    const int t = grp & (tb - 1), hs = grp >> log_tb, step = GROUPS >> log_tb;
    const int tok = t0 + t;
    if (tok >= tokens) return;
    const int b = tok / p.N, n = tok - b * p.N;
    Turn<IL> turn;
    turn.set(p, cs + t * (p.rot >> 1), j, lane);
    const int y0 = blockIdx.y * heads_per_block, y1 = min(y0 + heads_per_block, p.H[0] + p.H[1]);
    for (int ts = 0; ts < 2; ++ts) {
        const int off = ts ? p.H[0] : 0;
        const int lo = max(y0 - off, 0), hi = min(y1 - off, p.H[ts]);
        if (lo >= hi) continue;
        const bool norm = p.w[ts] != nullptr;
        float A[8], Bp[8];
        load_weights(p, ts, 8 * j, A);
        load_weights(p, ts, 8 * (j + (turn.partner - lane)), Bp);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            if constexpr (IL) { const float x = Bp[e]; Bp[e] = Bp[e + 1]; Bp[e + 1] = x; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) { A[e] *= turn.c[e]; Bp[e] = turn.turned ? Bp[e] * turn.s[e] : 0.0f; }
        const T* x = static_cast<const T*>(p.x[ts]) + b * p.xs[ts][0] + n * p.xs[ts][2] + 8 * j;
        T* y = static_cast<T*>(p.y[ts]) + b * p.ys[ts][0] + n * p.ys[ts][2] + 8 * j;
        for (int h = lo + hs; h < hi; h += step * U) {
            Chunk<T> c[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u * step < hi) c[u].load(x + (h + u * step) * p.xs[ts][1]);
                else c[u].zero();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8], o[8];
                c[u].get(f);
                turn.partners(c[u], f, o);
                float r = 1.0f;
                if (norm) {
                    float sq = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(f[e], f[e], sq);
                    r = __builtin_amdgcn_rsqf(group_sum<LPR>(sq) * (1.0f / D) + p.eps);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = r * __builtin_fmaf(f[e], A[e], o[e] * Bp[e]);
                if (h + u * step < hi) Chunk<T>::store(y + (h + u * step) * p.ys[ts][1], f);
            }
        }
    }
}

// Gradients: the same walk; the sine's sign turns the gradient back.  A lane
// keeps the sum of g n of its eight elements over all its rows; the workgroup
// adds its groups' sums in a fixed order and writes one partial sum per tensor.
template <typename T, int D, bool IL>
__global__ __launch_bounds__(THREADS) void rope_bwd_kernel(RopeProblem p, int log_tb) {
    constexpr int LPR = D / 8, GROUPS = THREADS / LPR;
    __shared__ float2 cs[MAX_TB * D / 2];
    __shared__ float red[GROUPS][D];
    const int tokens = p.B * p.N, tb = 1 << log_tb;
    const int j = threadIdx.x % LPR, grp = threadIdx.x / LPR, lane = threadIdx.x & 63;
    const int t = grp & (tb - 1), hs = grp >> log_tb, step = GROUPS >> log_tb;
    float dw[2][8];
#pragma unroll
    for (int ts = 0; ts < 2; ++ts)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[ts][e] = 0.0f;
    for (int t0 = blockIdx.x << log_tb; t0 < tokens; t0 += gridDim.x << log_tb) {
        __syncthreads();
        take_angles(p, cs, t0, tb, tokens);
        __syncthreads();
        const int tok = t0 + t;
        if (tok >= tokens) continue;
        const int b = tok / p.N, n = tok - b * p.N;
        Turn<IL> turn;
        turn.set(p, cs + t * (p.rot >> 1), j, lane);
#pragma unroll
        for (int ts = 0; ts < 2; ++ts) {
            const bool norm = p.w[ts] != nullptr;
            float w[8];
            load_weights(p, ts, 8 * j, w);
            const T* x = static_cast<const T*>(p.x[ts]) + b * p.xs[ts][0] + n * p.xs[ts][2] + 8 * j;
            const T* g = static_cast<const T*>(p.g[ts]) + b * p.gs[ts][0] + n * p.gs[ts][2] + 8 * j;
            T* y = static_cast<T*>(p.y[ts]) + b * p.ys[ts][0] + n * p.ys[ts][2] + 8 * j;
            for (int h = hs; h < p.H[ts]; h += step) {
                Chunk<T> cx, cg;
                cg.load(g + h * p.gs[ts][1]);
                if (norm) cx.load(x + h * p.xs[ts][1]);
                float gv[8], o[8];
                cg.get(gv);
                turn.partners(cg, gv, o);
#pragma unroll
                for (int e = 0; e < 8; ++e) gv[e] = __builtin_fmaf(gv[e], turn.c[e], -o[e] * turn.s[e]);
                if (norm) {
                    float f[8], sq = 0.0f, dot = 0.0f;
                    cx.get(f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(f[e], f[e], sq);
                    const float r = __builtin_amdgcn_rsqf(group_sum<LPR>(sq) * (1.0f / D) + p.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f[e] *= r;
                        dw[ts][e] = __builtin_fmaf(gv[e], f[e], dw[ts][e]);
                        gv[e] *= w[e];
                        dot = __builtin_fmaf(gv[e], f[e], dot);
                    }
                    dot = group_sum<LPR>(dot) * (1.0f / D);
#pragma unroll
                    for (int e = 0; e < 8; ++e) gv[e] = r * __builtin_fmaf(-f[e], dot, gv[e]);
                }
                Chunk<T>::store(y + h * p.ys[ts][1], gv);
            }
        }
    }
    if (!p.w[0] && !p.w[1]) return;
#pragma unroll
    for (int ts = 0; ts < 2; ++ts) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) red[grp][8 * j + e] = dw[ts][e];
        __syncthreads();
        if (threadIdx.x < D) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) sum += red[i][threadIdx.x];
            p.ws[((size_t)blockIdx.x * 2 + ts) * D + threadIdx.x] = sum;
        }
    }
}

// Sums the workgroups' partial sums in a fixed order: a workgroup per tensor
// and 16 elements, 64 threads per element.
template <int D>
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float* __restrict__ ws, float* dwq,
                                                       float* dwk, int blocks) {
    __shared__ float red[64][17];
    const int e = threadIdx.x & 15, k = threadIdx.x >> 4;
    const int ts = blockIdx.x / (D / 16), col = (blockIdx.x % (D / 16)) * 16 + e;
    float* out = ts ? dwk : dwq;
    if (!out) return;
    float sum = 0.0f;
#pragma unroll 4
    for (int i = k; i < blocks; i += 64) sum += ws[((size_t)i * 2 + ts) * D + col];
    red[k][e] = sum;
    __syncthreads();
    if (k == 0) {
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) all += red[i][e];
        out[col] = all;
    }
}

// Tokens a workgroup takes at a time: as many as still leave a few workgroups
// for every compute unit, so that the angles are shared.
int pick_log_tb(int tokens) {
    int l = 4;
    while (l > 0 && (tokens >> l) < 1024) --l;
    return l;
}

template <typename T, int D, bool IL>
hipError_t fwd(const RopeProblem& p, hipStream_t stream) {
    const int tokens = p.B * p.N, heads = p.H[0] + p.H[1];
    const int log_tb = pick_log_tb(tokens);
    const int tiles = (tokens + (1 << log_tb) - 1) >> log_tb, least = (THREADS / (D / 8)) >> log_tb;
    // Few tokens: their heads go to several workgroups.
    int per = heads;
    while (per > least && (long long)tiles * ((heads + per - 1) / per) < 512) per = per / 2 > least ? per / 2 : least;
    return launch_kernel(rope_fwd_kernel<T, D, IL>, dim3(tiles, (heads + per - 1) / per), dim3(THREADS), stream, p,
                         log_tb, per);
}

template <typename T, int D, bool IL>
hipError_t bwd(const RopeProblem& p, hipStream_t stream) {
    const int tokens = p.B * p.N;
    int blocks = 0;
    if (tokens > 0 && p.H[0] + p.H[1] > 0) {
        const int log_tb = pick_log_tb(tokens);
        blocks = (tokens + (1 << log_tb) - 1) >> log_tb;
        if (blocks > kRopeBwdMaxBlocks) blocks = kRopeBwdMaxBlocks;
        const hipError_t e =
            launch_kernel(rope_bwd_kernel<T, D, IL>, dim3(blocks), dim3(THREADS), stream, p, log_tb);
        if (e != hipSuccess) return e;
    }
    if (!p.w[0] && !p.w[1]) return hipSuccess;
    return launch_kernel(rope_dw_kernel<D>, dim3(2 * (D / 16)), dim3(1024), stream, p.ws, p.dw[0], p.dw[1], blocks);
}

template <typename F>
hipError_t by_type(const RopeProblem& p, F f) {
    if (p.bf16) {
        if (p.d == 64) return f(u16{}, std::integral_constant<int, 64>{});
        return f(u16{}, std::integral_constant<int, 128>{});
    }
    if (p.d == 64) return f(float{}, std::integral_constant<int, 64>{});
    return f(float{}, std::integral_constant<int, 128>{});
}

}  // namespace

hipError_t launch_rope_fwd(const RopeProblem& p, hipStream_t stream) {
    return by_type(p, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        return p.interleaved ? fwd<T, D, true>(p, stream) : fwd<T, D, false>(p, stream);
    });
}

hipError_t launch_rope_bwd(const RopeProblem& p, hipStream_t stream) {
    return by_type(p, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        return p.interleaved ? bwd<T, D, true>(p, stream) : bwd<T, D, false>(p, stream);
    });
}

}  // namespace moa
