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
#include <cfloat>

#include "device_common.h"
#include "rope.h"

namespace moa {
namespace {

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

// cos and sin of the rot/2 pairs of the workgroup's tokens t0 .. t0 + tb - 1.
__device__ __forceinline__ void take_angles(const RopeProblem& p, float2* cs, int t0, int tb, int tokens) {
    const int pairs = p.rot >> 1;
    for (int i = threadIdx.x; i < tb * pairs; i += THREADS) {
        const int t = i / pairs, pr = i - t * pairs, tok = t0 + t;
        if (tok >= tokens) break;
        int axis = 0;
        for (int a = 1; a < p.axes; ++a) axis = pr >= p.first[a] ? a : axis;
        const long long at = p.pos ? p.pos[(long long)axis * tokens + tok] : tok % p.N;
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
    take_angles(p, cs, t0, tb, tokens);
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
        take_angles(p, cs, t0, tb, tokens);
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
