// Appending new tokens to a paged bf16 cache, with the norm of their heads and the
// rotation by position on the way (moa_paged.h; the formulas are moa_rope.h's).
//
// Every row of d elements, of queries, keys and values alike, is read once and
// written once: memory's.  The walk is that of rope.hip: a group of d/8 lanes holds
// a token and goes over its heads, weight and rotation folded into two factors
// per element that it keeps in registers, the next rows on their way while it
// works on the present ones; the angles are taken once per token, into LDS.  What
// a key or value row adds is its page, looked up once per token.
//
// What bounds it: memory.  2 x 4096 tokens, 16 + 16 + 16 heads, d = 128: 34 us alone,
// 5.9 TB/s, waiting for rows 0.68 of its time; 44 among other work (4.6 TB/s, a copy of
// that size 5.1).  (All three tensors mixed in a group's rows, each row's addresses
// formed anew: 87.)  One token: 5 us, latencies.
#include "rope_common.h"
#include "paged.h"
#include "win_common.h"

namespace moa {
namespace {

using namespace rope;

// The heads that one lane group takes of its token: heads first, first + step, ..
// below end, counted over Q's, K's and V's, one tensor at a time.
struct Walk {
    int start[4];          // the first head of each tensor, and the end
    int step, first, end;
    int ts, h;             // head h of tensor ts; ts = 3: none left
    __device__ __forceinline__ Walk(int hq, int hk, int step_, int first_, int end_)
        : start{0, hq, hq + hk, hq + 2 * hk}, step(step_), first(first_), end(end_) { enter(0); }
    __device__ __forceinline__ int limit() const { return min(end, start[1]) - start[0]; }
    // The first head of this group's in tensor t or a later one.  (The tensor's own
    // limits move to the front, so that no array is indexed.)
    __device__ __forceinline__ void enter(int t) {
        ts = t;
        while (ts < 3) {
            const int from = first >= start[0] ? first : first + (start[0] - first + step - 1) / step * step;
            h = from - start[0];
            if (h < limit()) return;
            leave();
        }
    }
    __device__ __forceinline__ void leave() {
        ++ts;
        start[0] = start[1];
        start[1] = start[2];
        start[2] = start[3];
    }
    // U heads on
    template <int U>
    __device__ __forceinline__ void next() {
        h += U * step;
        if (h < limit()) return;
        leave();
        enter(ts);
    }
};

// One of three values.  (Their places in the arguments or in a closure to choose from
// sent these to scratch memory.)
template <typename V>
__device__ __forceinline__ V pick(int i, V a, V b, V c) { return i == 0 ? a : i == 1 ? b : c; }

template <typename T, int D, bool IL>
__global__ __launch_bounds__(THREADS) void paged_append_kernel(AppendProblem a, int log_tb, int heads_per_block) {
    constexpr int LPR = D / 8, GROUPS = THREADS / LPR, U = sizeof(T) == 2 ? 4 : 2;   // rows in flight per group
    __shared__ float2 cs[THREADS / LPR * D / 2];
    const RopeProblem& p = a.r;
    const int tokens = p.B * p.N, tb = 1 << log_tb, t0 = blockIdx.x << log_tb;
    const int j = threadIdx.x % LPR, grp = threadIdx.x / LPR, lane = threadIdx.x & 63;
    const int t = grp & (tb - 1), tok = min(t0 + t, tokens - 1);
    const int b = tok / p.N, n = tok - b * p.N;
    const int hq = p.H[0], hk = p.H[1];
    const int y0 = blockIdx.y * heads_per_block, y1 = min(y0 + heads_per_block, hq + 2 * hk);
    // Token n of sequence b is its token `at`.
    const auto place = [&](int tok) {
        const int b = tok / p.N, n = tok - b * p.N;
        return (long long)a.to.seq_lens[b] - win::new_tokens(a.to.new_lens, b, p.N) + n;
    };
    const bool real = t0 + t < tokens && n < win::new_tokens(a.to.new_lens, b, p.N);
    const long long at = place(tok);
    const int page = at >= 0 && at < win::capacity(a.to) ? win::page_of(a.to, b, (int)at) : -1;
    const T* const xq = static_cast<const T*>(p.x[0]) + b * p.xs[0][0] + n * p.xs[0][2] + 8 * j;
    const T* const xk = static_cast<const T*>(p.x[1]) + b * p.xs[1][0] + n * p.xs[1][2] + 8 * j;
    const T* const xv = static_cast<const T*>(a.v) + b * a.vs[0] + n * a.vs[2] + 8 * j;
    u16* const yq = static_cast<u16*>(p.y[0]) + b * p.ys[0][0] + n * p.ys[0][2] + 8 * j;
    u16* const yk = static_cast<u16*>(const_cast<void*>(a.to.k)) + (page >= 0 ? win::key_offset(a.to.ks, a.to.shift, page, 0, (int)at) : 0) + 8 * j;
    u16* const yv = static_cast<u16*>(const_cast<void*>(a.to.v)) + (page >= 0 ? win::key_offset(a.to.vs, a.to.shift, page, 0, (int)at) : 0) + 8 * j;
    Walk w(hq, hk, GROUPS >> log_tb, y0 + (grp >> log_tb), y1);
    // Keys and values of a token without a page are not read.
    const auto wanted = [&](int ts) { return real && ts < 3 && (ts == 0 || page >= 0); };
    const auto load = [&](Chunk<T> (&c)[U]) {
        const T* base = pick(w.ts, xq, xk, xv);
        const long long stride = pick(w.ts, p.xs[0][1], p.xs[1][1], a.vs[1]);
        const int limit = wanted(w.ts) ? w.limit() : 0;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (w.h + u * w.step < limit) c[u].load(base + (w.h + u * w.step) * stride);
            else c[u].zero();
    };
    // The first rows and the weights are on their way while the angles are taken.
    Chunk<T> next[U];
    load(next);
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
    while (w.ts < 3) {
        const int ts = w.ts, h = w.h, limit = wanted(ts) ? w.limit() : 0, step = w.step;
        Chunk<T> c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = next[u];
        w.template next<U>();
        load(next);
        u16* to = pick(ts, yq, yk, yv);
        const long long stride = pick(ts, p.ys[0][1], a.to.ks[1], a.to.vs[1]);
        if (ts == 2) {   // values go over as they are
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8];
                c[u].get(f);
                if (h + u * step < limit) Chunk<u16>::store(to + (h + u * step) * stride, f);
            }
            continue;
        }
        if (ts != have) {
            have = ts;
#pragma unroll
            for (int e = 0; e < 8; ++e) A[e] = ts ? wk[e] : wq[e];
#pragma unroll
            for (int e = 0; e < 8; ++e) Bp[e] = IL ? A[e ^ 1] : __shfl(A[e], turn.partner);
#pragma unroll
            for (int e = 0; e < 8; ++e) { A[e] *= turn.c[e]; Bp[e] = turn.turned ? Bp[e] * turn.s[e] : 0.0f; }
        }
        const bool norm = pick(ts, p.w[0], p.w[1], p.w[1]) != nullptr;
        bool redo[U];
        const auto row = [&](int u, float r, auto again) {
            float f[8], o[8];
            c[u].get(f);
            turn.partners(c[u], f, o);
            const bool in = h + u * step < limit;
            if (!again) {
                redo[u] = false;
                if (norm) {
                    const float m = mean_square<LPR>(f) + p.eps;
                    r = __builtin_amdgcn_rsqf(m);
                    redo[u] = in && !in_range(m);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = r * __builtin_fmaf(f[e], A[e], o[e] * Bp[e]);
            if (in && redo[u] == again) Chunk<u16>::store(to + (h + u * step) * stride, f);
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
