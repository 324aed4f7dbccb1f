// Appending new tokens to a paged bf16 cache, with the norm of their heads and the
// rotation by position on the way (moa_paged.h; the formulas are moa_rope.h's).
//
// Every row of d elements, of queries, keys and values alike, is read once and
// written once: memory's.  The walk is that of rope.hip: a group of d/8 lanes holds
// a token and goes over its heads, weight and rotation folded into two factors
// per element that it keeps in registers, the next rows on their way while it
// works on the present ones; the angles are taken once per token, into LDS.  What
// a key or value row adds is its page, looked up once per token.
#include "rope_common.h"
#include "paged.h"
#include "win_common.h"

namespace moa {
namespace {

using namespace rope;

template <typename T, int D, bool IL>
__global__ __launch_bounds__(THREADS) void paged_append_kernel(AppendProblem a, int log_tb, int heads_per_block) {
    constexpr int LPR = D / 8, GROUPS = THREADS / LPR, U = sizeof(T) == 2 ? 4 : 2;   // rows in flight per group
    __shared__ float2 cs[THREADS / LPR * D / 2];
    const RopeProblem& p = a.r;
    const int tokens = p.B * p.N, tb = 1 << log_tb, t0 = blockIdx.x << log_tb;
    const int j = threadIdx.x % LPR, grp = threadIdx.x / LPR, lane = threadIdx.x & 63;
    const int t = grp & (tb - 1), tok = min(t0 + t, tokens - 1);
    const int b = tok / p.N, n = tok - b * p.N;
    const int hq = p.H[0], hk = p.H[1], step = GROUPS >> log_tb;
    const int y0 = blockIdx.y * heads_per_block, y1 = min(y0 + heads_per_block, hq + 2 * hk);
    // Token n of sequence b is its token `at`.
    const auto place = [&](int tok) {
        const int b = tok / p.N, n = tok - b * p.N;
        return (long long)a.to.seq_lens[b] - win::new_tokens(a.to.new_lens, b, p.N) + n;
    };
    const bool real = t0 + t < tokens && n < win::new_tokens(a.to.new_lens, b, p.N);
    const long long at = place(tok);
    const int page = at >= 0 && at < win::capacity(a.to) ? win::page_of(a.to, b, (int)at) : -1;
    // Heads are counted over Q's, K's and V's.
    const auto part = [&](int h) { return h < hq ? 0 : h < hq + hk ? 1 : 2; };
    const auto row_of = [&](int h) -> const T* {
        const int ts = part(h);
        const void* base = ts == 0 ? p.x[0] : ts == 1 ? p.x[1] : a.v;
        const int head = h - (ts == 0 ? 0 : ts == 1 ? hq : hq + hk);
        const long long s0 = ts == 0 ? p.xs[0][0] : ts == 1 ? p.xs[1][0] : a.vs[0];
        const long long s1 = ts == 0 ? p.xs[0][1] : ts == 1 ? p.xs[1][1] : a.vs[1];
        const long long s2 = ts == 0 ? p.xs[0][2] : ts == 1 ? p.xs[1][2] : a.vs[2];
        return static_cast<const T*>(base) + b * s0 + head * s1 + n * s2 + 8 * j;
    };
    int h = y0 + (grp >> log_tb);
    // Keys and values of a token without a page are not read.
    const auto wanted = [&](int h) { return real && h < y1 && (h < hq || page >= 0); };
    const auto load = [&](Chunk<T> (&c)[U], int h) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (wanted(h + u * step)) c[u].load(row_of(h + u * step));
            else c[u].zero();
    };
    // The first rows and the weights are on their way while the angles are taken.
    Chunk<T> next[U];
    load(next, h);
    float wq[8], wk[8];
    load_weights(p, 0, j, wq);
    load_weights(p, 1, j, wk);
    take_angles(p, cs, t0, tb, tokens, place);
    __syncthreads();
    if (!real) return;
    Turn<IL> turn;
    turn.set(p, cs + t * (p.rot >> 1), j, lane);
    float A[8], Bp[8];
    int have = -1;
    while (h < y1) {
        Chunk<T> c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = next[u];
        const int h0 = h;
        h += U * step;
        load(next, h);
        bool redo[U];
        const auto row = [&](int u, float r, auto again) {
            const int hu = h0 + u * step, ts = part(hu);
            // Partners move between lanes, so every lane of the group takes part.
            if (ts < 2 && ts != have) {
                have = ts;
#pragma unroll
                for (int e = 0; e < 8; ++e) A[e] = ts == 1 ? wk[e] : wq[e];
#pragma unroll
                for (int e = 0; e < 8; ++e) Bp[e] = IL ? A[e ^ 1] : __shfl(A[e], turn.partner);
#pragma unroll
                for (int e = 0; e < 8; ++e) { A[e] *= turn.c[e]; Bp[e] = turn.turned ? Bp[e] * turn.s[e] : 0.0f; }
            }
            float f[8], o[8];
            c[u].get(f);
            turn.partners(c[u], f, o);
            if (!again) redo[u] = false;
            if (ts < 2) {
                if (!again && p.w[ts ? 1 : 0] != nullptr) {
                    const float m = mean_square<LPR>(f) + p.eps;
                    r = __builtin_amdgcn_rsqf(m);
                    redo[u] = wanted(hu) && !in_range(m);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = r * __builtin_fmaf(f[e], A[e], o[e] * Bp[e]);
            }
            if (!wanted(hu) || redo[u] != again) return;
            u16* to;
            if (ts == 0) {
                to = static_cast<u16*>(p.y[0]) + b * p.ys[0][0] + hu * p.ys[0][1] + n * p.ys[0][2];
            } else {
                const int head = hu - (ts == 1 ? hq : hq + hk);
                to = static_cast<u16*>(const_cast<void*>(ts == 1 ? a.to.k : a.to.v)) +
                     (ts == 1 ? win::key_offset(a.to.ks, a.to.shift, page, head, (int)at)
                              : win::key_offset(a.to.vs, a.to.shift, page, head, (int)at));
            }
            Chunk<u16>::store(to + 8 * j, f);
        };
        bool any = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row(u, 1.0f, std::false_type{});
            any |= redo[u];
        }
        if (!wave_any(any)) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float r;
            int down;
            divide<LPR>(c[u], p.eps, r, down);
            row(u, r, std::true_type{});
        }
    }
}

// Tokens a workgroup takes at a time and the heads it walks over, as in rope.hip.
template <typename T, int D, bool IL>
hipError_t go(const AppendProblem& a, hipStream_t stream) {
    const int tokens = a.r.B * a.r.N, heads = a.r.H[0] + 2 * a.r.H[1], groups = THREADS / (D / 8);
    int log_tb = 0;
    while ((2 << log_tb) <= groups && (tokens >> (log_tb + 1)) >= 256) ++log_tb;
    const int tiles = (tokens + (1 << log_tb) - 1) >> log_tb, least = groups >> log_tb;
    int per = heads;
    while (per > least && (long long)tiles * ((heads + per - 1) / per) < 256) per = per / 2 > least ? per / 2 : least;
    return launch_kernel(paged_append_kernel<T, D, IL>, dim3(tiles, (heads + per - 1) / per), dim3(THREADS), stream, a,
                         log_tb, per);
}

template <typename T, int D>
hipError_t by_pairs(const AppendProblem& a, hipStream_t stream) {
    return a.r.interleaved ? go<T, D, true>(a, stream) : go<T, D, false>(a, stream);
}

}  // namespace

hipError_t launch_paged_append(const AppendProblem& a, hipStream_t stream) {
    if (a.r.bf16) return a.r.d == 64 ? by_pairs<u16, 64>(a, stream) : by_pairs<u16, 128>(a, stream);
    return a.r.d == 64 ? by_pairs<float, 64>(a, stream) : by_pairs<float, 128>(a, stream);
}

}  // namespace moa
