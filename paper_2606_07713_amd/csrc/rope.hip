// Norms of queries and keys for each head with the rotation by position, and
// the gradients (moa_rope.h has the formulas).
//
// Each row of d elements is read once and written once and takes about ten
// operations an element: mostly memory's (32 heads of 8192 tokens, bf16, d = 128:
// 134 MB in 26 us, 5.1 TB/s, and 201 MB in 41 us, 4.9 TB/s, for the gradients;
// copies of as much read and written reach 7.0 and 5.9).  A group of d/8 lanes
// holds a row, eight elements a lane; the sum of squares is a reduction inside
// the group.  The rotation is folded with the weight: of a rotated element e
// with partner e' (the other element of its pair)
//   y_e = r (x_e A_e + x_e' B_e),  A_e = w_e cos,  B_e = -/+ w_e' sin,
// and A and B depend on the token only, so a group keeps its token while it
// walks over heads and holds A and B in registers, the next heads' rows on their
// way while it works on the present ones (the gradients with one row in flight
// on two workgroups per unit: 54 us).  The sines and cosines of a
// workgroup's tokens are taken once, by all its threads, into LDS: fp64 angles,
// reduced to one turn (fp32 angles of position 10^6 would be off by 0.06).
// Partners are eight-element chunks of another lane of the group (rot/2 is a
// multiple of 8), or neighbours in the same lane when pairs are interleaved.
#include "device_common.h"
#include "rope_common.h"

namespace moa {
namespace {

using namespace rope;

// The heads that one lane group takes of its token: heads first, first + step,
// .. below end, counted over Q's and then K's, one tensor at a time.
struct Walk {
    int hq, step, first, end;
    int ts, h;   // head h of tensor ts; ts = 2: none left
    __device__ __forceinline__ void start(int hq_, int step_, int first_, int end_) {
        hq = hq_; step = step_; first = first_; end = end_;
        ts = first < end ? first >= hq : 2;
        h = ts == 1 ? first - hq : first;
    }
    __device__ __forceinline__ int limit() const { return ts == 0 ? min(end, hq) : end - hq; }
    // U heads on
    template <int U>
    __device__ __forceinline__ void next() {
        h += U * step;
        if (h < limit()) return;
        if (ts == 0 && end > hq) {   // K's first head of this group's
            const int over = hq > first ? (hq - first + step - 1) / step * step + first - hq : first - hq;
            h = over;
            ts = over < end - hq ? 1 : 2;
        } else {
            ts = 2;
        }
    }
};

template <typename T, int D, bool IL>
__global__ __launch_bounds__(THREADS) void rope_fwd_kernel(RopeProblem p, int log_tb, int heads_per_block) {
    constexpr int LPR = D / 8, GROUPS = THREADS / LPR, U = sizeof(T) == 2 ? 4 : 2;   // rows in flight per group
    __shared__ float2 cs[THREADS / LPR * D / 2];
    const int tokens = p.B * p.N, tb = 1 << log_tb, t0 = blockIdx.x << log_tb;
    const int j = threadIdx.x % LPR, grp = threadIdx.x / LPR, lane = threadIdx.x & 63;
    const auto place = [&](int tok) { return (long long)(tok % p.N); };   // without positions
    const int t = grp & (tb - 1), tok = min(t0 + t, tokens - 1);
    const int b = tok / p.N, n = tok - b * p.N;
    const int y0 = blockIdx.y * heads_per_block, y1 = min(y0 + heads_per_block, p.H[0] + p.H[1]);
    const T* x[2];
    T* y[2];
#pragma unroll
    for (int ts = 0; ts < 2; ++ts) {
        x[ts] = static_cast<const T*>(p.x[ts]) + b * p.xs[ts][0] + n * p.xs[ts][2] + 8 * j;
        y[ts] = static_cast<T*>(p.y[ts]) + b * p.ys[ts][0] + n * p.ys[ts][2] + 8 * j;
    }
    Walk w;
    w.start(p.H[0], GROUPS >> log_tb, y0 + (grp >> log_tb), y1);
    const auto load = [&](Chunk<T> (&c)[U]) {
        const T* base = w.ts ? x[1] : x[0];
        const long long stride = w.ts ? p.xs[1][1] : p.xs[0][1];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (w.ts < 2 && w.h + u * w.step < w.limit()) c[u].load(base + (w.h + u * w.step) * stride);
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
    if (t0 + t >= tokens) return;
    Turn<IL> turn;
    turn.set(p, cs + t * (p.rot >> 1), j, lane);
    float A[8], Bp[8];
    int have = -1;
    while (w.ts < 2) {
        const int ts = w.ts, h = w.h, limit = w.limit();
        Chunk<T> c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = next[u];
        w.template next<U>();
        load(next);
        if (ts != have) {
            have = ts;
#pragma unroll
            for (int e = 0; e < 8; ++e) A[e] = ts ? wk[e] : wq[e];
#pragma unroll
            for (int e = 0; e < 8; ++e) Bp[e] = IL ? A[e ^ 1] : __shfl(A[e], turn.partner);
#pragma unroll
            for (int e = 0; e < 8; ++e) { A[e] *= turn.c[e]; Bp[e] = turn.turned ? Bp[e] * turn.s[e] : 0.0f; }
        }
        const bool norm = (ts ? p.w[1] : p.w[0]) != nullptr;
        T* to = ts ? y[1] : y[0];
        const long long stride = ts ? p.ys[1][1] : p.ys[0][1];
        bool redo[U];
        const auto row = [&](int u, float r, auto again) {
            float f[8], o[8];
            c[u].get(f);
            turn.partners(c[u], f, o);
            const bool in = h + u * w.step < limit;
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
            if (in && redo[u] == again) Chunk<T>::store(to + (h + u * w.step) * stride, f);
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

// Gradients: the same walk; the sine's sign turns the gradient back.  A lane
// keeps the sum of g n of its eight elements over all its rows; the workgroup
// adds its groups' sums in a fixed order and writes one partial sum per tensor.
template <typename T, int D, bool IL>
__global__ __launch_bounds__(THREADS) void rope_bwd_kernel(RopeProblem p, int log_tb) {
    constexpr int LPR = D / 8, GROUPS = THREADS / LPR, U = 2;
    __shared__ float2 cs[THREADS / LPR * D / 2];
    __shared__ float red[GROUPS][D];
    const int tokens = p.B * p.N, tb = 1 << log_tb;
    const int j = threadIdx.x % LPR, grp = threadIdx.x / LPR, lane = threadIdx.x & 63;
    const auto place = [&](int tok) { return (long long)(tok % p.N); };   // without positions
    const int t = grp & (tb - 1);
    float dw[2][8], wq[8], wk[8];
    load_weights(p, 0, j, wq);
    load_weights(p, 1, j, wk);
#pragma unroll
    for (int ts = 0; ts < 2; ++ts)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[ts][e] = 0.0f;
    for (int t0 = blockIdx.x << log_tb; t0 < tokens; t0 += gridDim.x << log_tb) {
        const int tok = min(t0 + t, tokens - 1);
        const int b = tok / p.N, n = tok - b * p.N;
        const T *x[2], *g[2];
        T* y[2];
#pragma unroll
        for (int ts = 0; ts < 2; ++ts) {
            x[ts] = static_cast<const T*>(p.x[ts]) + b * p.xs[ts][0] + n * p.xs[ts][2] + 8 * j;
            g[ts] = static_cast<const T*>(p.g[ts]) + b * p.gs[ts][0] + n * p.gs[ts][2] + 8 * j;
            y[ts] = static_cast<T*>(p.y[ts]) + b * p.ys[ts][0] + n * p.ys[ts][2] + 8 * j;
        }
        Walk walk;
        walk.start(p.H[0], GROUPS >> log_tb, grp >> log_tb, p.H[0] + p.H[1]);
        const auto load = [&](Chunk<T> (&cx)[U], Chunk<T> (&cg)[U]) {
            const int ts = walk.ts;
            const T *bg = ts ? g[1] : g[0], *bx = ts ? x[1] : x[0];
            const long long sg = ts ? p.gs[1][1] : p.gs[0][1], sx = ts ? p.xs[1][1] : p.xs[0][1];
            const bool norm = (ts ? p.w[1] : p.w[0]) != nullptr;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = walk.h + u * walk.step;
                const bool in = ts < 2 && h < walk.limit();
                if (in) cg[u].load(bg + h * sg);
                else cg[u].zero();
                if (in && norm) cx[u].load(bx + h * sx);
                else cx[u].zero();
            }
        };
        Chunk<T> nx[U], ng[U];
        load(nx, ng);
        __syncthreads();   // the angles of the tile before have been read
        take_angles(p, cs, t0, tb, tokens, place);
        __syncthreads();
        if (t0 + t >= tokens) continue;
        Turn<IL> turn;
        turn.set(p, cs + t * (p.rot >> 1), j, lane);
        while (walk.ts < 2) {
            const int ts = walk.ts, h0 = walk.h, limit = walk.limit();
            Chunk<T> cx[U], cg[U];
#pragma unroll
            for (int u = 0; u < U; ++u) { cx[u] = nx[u]; cg[u] = ng[u]; }
            walk.template next<U>();
            load(nx, ng);
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = ts ? wk[e] : wq[e];
            const bool norm = (ts ? p.w[1] : p.w[0]) != nullptr;
            T* to = ts ? y[1] : y[0];
            const long long stride = ts ? p.ys[1][1] : p.ys[0][1];
            bool redo[U];
            const auto row = [&](int u, float r, int down, auto again) {
                float gv[8], o[8];
                cg[u].get(gv);
                turn.partners(cg[u], gv, o);
                const bool in = h0 + u * walk.step < limit;
                if (!again) redo[u] = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) gv[e] = __builtin_fmaf(gv[e], turn.c[e], -o[e] * turn.s[e]);
                if (norm) {   // only rows that this pass stores add to dw
                    float f[8], dot = 0.0f;
                    cx[u].get(f);
                    if (!again) {
                        const float m = mean_square<LPR>(f) + p.eps;
                        r = __builtin_amdgcn_rsqf(m);
                        redo[u] = in && !in_range(m);
                    }
                    r = in && redo[u] == again ? r : 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f[e] *= r;
                        const float add = gv[e] * f[e];
                        dw[0][e] += ts ? 0.0f : add;
                        dw[1][e] += ts ? add : 0.0f;
                        gv[e] *= w[e];
                        dot = __builtin_fmaf(gv[e], f[e], dot);
                    }
                    dot = group_sum<LPR>(dot) * (1.0f / D);
#pragma unroll
                    for (int e = 0; e < 8; ++e) gv[e] = r * __builtin_fmaf(-f[e], dot, gv[e]);
                    if (again)
#pragma unroll
                        for (int e = 0; e < 8; ++e) gv[e] = ldexpf(gv[e], -down);
                }
                if (in && redo[u] == again) Chunk<T>::store(to + (h0 + u * walk.step) * stride, gv);
            };
            bool any = false;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                row(u, 1.0f, 0, std::false_type{});
                any |= redo[u];
            }
            if (!wave_any(any)) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float r;
                int down;
                divide<LPR>(cx[u], p.eps, r, down);
                row(u, r, down, std::true_type{});
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
// and 16 elements, 64 threads per element, all loads of a thread in flight at
// once.
template <int D>
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float* __restrict__ ws, float* dwq,
                                                       float* dwk, int blocks) {
    constexpr int PER = kRopeBwdMaxBlocks / 64;
    __shared__ float red[16][16];
    const int e = threadIdx.x & 15, k = threadIdx.x >> 4;
    const int ts = blockIdx.x / (D / 16), col = (blockIdx.x % (D / 16)) * 16 + e;
    float* out = ts ? dwk : dwq;
    if (!out) return;
    float v[PER], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = k + 64 * i < blocks ? ws[((size_t)(k + 64 * i) * 2 + ts) * D + col] : 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += v[i];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][e] = sum;
    __syncthreads();
    if (threadIdx.x < 16) {
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) all += red[i][e];
        out[col] = all;
    }
}

// Tokens a workgroup takes at a time (a power of two, at most one for each of
// its groups): as many as leave a workgroup for every compute unit.  What a
// group does once per token then serves as many heads as there are: 16 heads of
// 4000 tokens, fp32, d = 64, forward and gradients: 1024 workgroups at least 10.9
// and 16.6 us, 512 9.3 and 15.2, 256 9.2 and 10.6.
int pick_log_tb(int tokens, int groups) {
    int l = 0;
    while ((2 << l) <= groups && (tokens >> (l + 1)) >= 256) ++l;
    return l;
}

template <typename T, int D, bool IL>
hipError_t fwd(const RopeProblem& p, hipStream_t stream) {
    const int tokens = p.B * p.N, heads = p.H[0] + p.H[1];
    const int log_tb = pick_log_tb(tokens, THREADS / (D / 8));
    const int tiles = (tokens + (1 << log_tb) - 1) >> log_tb, least = (THREADS / (D / 8)) >> log_tb;
    // Few tokens: their heads go to several workgroups, until there is one for
    // every compute unit (24 heads of 6216 tokens, fp32, d = 64: 19.2 us with the
    // heads in two halves on 778 workgroups, 15.9 whole on 389).
    int per = heads;
    while (per > least && (long long)tiles * ((heads + per - 1) / per) < 256) per = per / 2 > least ? per / 2 : least;
    return launch_kernel(rope_fwd_kernel<T, D, IL>, dim3(tiles, (heads + per - 1) / per), dim3(THREADS), stream, p,
                         log_tb, per);
}

template <typename T, int D, bool IL>
hipError_t bwd(const RopeProblem& p, hipStream_t stream) {
    const int tokens = p.B * p.N;
    int blocks = 0;
    if (tokens > 0 && p.H[0] + p.H[1] > 0) {
        const int log_tb = pick_log_tb(tokens, THREADS / (D / 8));
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
