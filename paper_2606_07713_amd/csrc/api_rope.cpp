// C-ABI front end of the head norms with rotation (moa_rope.h): argument
// validation and dispatch.  Host code; allocates nothing, never synchronises.
#include <cmath>
#include <limits>

#include "../../include/moa_rope.h"
#include "api_checks.h"
#include "packed.h"
#include "rope.h"

namespace {

using namespace moa;

struct View {
    const void* p;
    Strides s;
    int64_t H;
};

// The arguments that forward and backward share.
struct Common {
    int64_t B, Hq, Hk, N, d, rot;
    const int64_t* positions;
    const float* inv_freq;
    int axes;
    const int64_t* sections;
    int interleaved;
    float eps;
    int dtype, w_dtype;
    size_t es() const { return dtype == MOA_F32 ? 4 : 2; }
    int64_t heads(int i) const { return i ? Hk : Hq; }
    bool any(int i) const { return B > 0 && N > 0 && heads(i) > 0; }
};

int check_common(const Common& c, const void* const (&w)[2]) {
    if (c.B < 0 || c.Hq < 0 || c.Hk < 0 || c.N < 0 || c.d < 1 || c.rot < 0) return MOA_ERR_INVALID_ARG;
    if (c.axes < 1 || c.axes > kRopeMaxAxes) return MOA_ERR_INVALID_ARG;
    if (c.interleaved != 0 && c.interleaved != 1) return MOA_ERR_INVALID_ARG;
    if (!std::isfinite(c.eps) || c.eps < 0) return MOA_ERR_INVALID_ARG;
    for (int t : {c.dtype, c.w_dtype})
        if (t != MOA_F32 && t != MOA_BF16) return MOA_ERR_INVALID_ARG;
    if (c.d != 64 && c.d != 128) return MOA_ERR_UNSUPPORTED;
    if (c.rot > c.d) return MOA_ERR_INVALID_ARG;
    if (c.rot % 16) return MOA_ERR_UNSUPPORTED;
    if (c.axes > 1 && !c.sections) return MOA_ERR_INVALID_ARG;
    if (c.sections) {
        int64_t sum = 0;
        for (int a = 0; a < c.axes; ++a) {
            if (c.sections[a] < 0 || c.sections[a] > c.rot) return MOA_ERR_INVALID_ARG;
            sum += c.sections[a];
        }
        if (sum != c.rot / 2) return MOA_ERR_INVALID_ARG;
    }
    if ((c.any(0) || c.any(1)) && c.rot > 0 && !c.inv_freq) return MOA_ERR_INVALID_ARG;
    if (!aligned16(w[0]) || !aligned16(w[1])) return MOA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(c.inv_freq) & 3) || (reinterpret_cast<uintptr_t>(c.positions) & 7)) return MOA_ERR_INVALID_ARG;
    const int64_t lim = std::numeric_limits<int32_t>::max();
    if (c.B > lim || c.N > lim || c.Hq > lim || c.Hk > lim) return MOA_ERR_UNSUPPORTED;
    const int64_t tokens = c.B * c.N, heads = c.Hq + c.Hk;
    // 2^27 tokens: 16 and more of them a workgroup, whose threads are counted in 32 bits
    // and the kernels step over heads a few times 32 past the last one
    if (tokens >= (int64_t(1) << 27) || heads >= (int64_t(1) << 30) || (tokens > 0 && heads > lim / tokens)) return MOA_ERR_UNSUPPORTED;
    return MOA_OK;
}

int check_view(const View& v, const Common& c, int i, bool out) {
    if (!v.p) return c.any(i) ? MOA_ERR_INVALID_ARG : MOA_OK;
    if (!aligned16(v.p)) return MOA_ERR_INVALID_ARG;
    if (!c.any(i)) return MOA_OK;
    const int64_t es = (int64_t)c.es();
    for (int64_t s : {v.s.b, v.s.h, v.s.r}) {
        if (s < 0) return MOA_ERR_INVALID_ARG;
        if (s > (int64_t(1) << 40) || (s * es) % 16) return MOA_ERR_UNSUPPORTED;
    }
    // elements from the first to the last: below 2^46, so byte offsets fit
    const __int128 n = (__int128)(c.B - 1) * v.s.b + (__int128)(v.H - 1) * v.s.h + (__int128)(c.N - 1) * v.s.r + c.d;
    if (n > ((__int128)1 << 46)) return MOA_ERR_UNSUPPORTED;
    if (out && !injective(v.s, c.B, v.H, c.N, c.d)) return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

size_t bytes(const View& v, const Common& c) { return extent_bytes(v.s, c.B, v.H, c.N, c.d, c.es()); }

// Whether two views certainly share no element: their byte ranges do not meet,
// or they take turns in one buffer: whole batches, or the heads of one token, be
// they [B][N][heads] or [N][B][heads].
bool disjoint(const View& a, const View& b, const Common& c) {
    if (!overlaps(a.p, bytes(a, c), b.p, bytes(b, c))) return true;
    const View &lo = a.p <= b.p ? a : b, &hi = a.p <= b.p ? b : a;
    const int64_t gap = (int64_t)(static_cast<const char*>(hi.p) - static_cast<const char*>(lo.p));
    if (gap % (int64_t)c.es()) return false;
    const int64_t delta = gap / (int64_t)c.es();
    const auto inner = [&](const View& v, bool rows) {   // elements of one row's heads, or of one batch
        return (v.H - 1) * v.s.h + (rows ? (c.N - 1) * v.s.r : 0) + c.d;
    };
    if (lo.s.b == hi.s.b && inner(lo, true) <= delta && delta + inner(hi, true) <= lo.s.b) return true;
    const int64_t end = delta + inner(hi, false);
    const bool rows = lo.s.r == hi.s.r, batches = lo.s.b == hi.s.b;
    if (inner(lo, false) > delta) return false;
    if (rows && end <= lo.s.r && (c.B == 1 || (batches && lo.s.b >= c.N * lo.s.r))) return true;
    return rows && batches && end <= lo.s.b && lo.s.r >= c.B * lo.s.b;
}

bool same(const View& a, const View& b) {
    return a.p == b.p && a.s.b == b.s.b && a.s.h == b.s.h && a.s.r == b.s.r;
}

// A dimension of size 1 has no stride to keep to.
Strides strides_of(const int64_t* s, int64_t H, const Common& c) {
    return s ? Strides{c.B > 1 ? s[0] : 0, H > 1 ? s[1] : 0, c.N > 1 ? s[2] : 0} : contiguous(H, c.N, c.d);
}

// Outputs against every input and each other; out[i] may be its own in[i].
int check_buffers(const View (&out)[2], const View (&in)[2], const View (&in2)[2], bool two, const Common& c,
                  const void* const (&w)[2]) {
    const size_t tokens = (size_t)(c.B * c.N), wn = (size_t)c.d * (c.w_dtype == MOA_F32 ? 4 : 2);
    for (int i = 0; i < 2; ++i) {
        if (!out[i].p || !c.any(i)) continue;
        for (int k = 0; k < 2; ++k) {
            if (in[k].p && c.any(k) && !(i == k && same(out[i], in[k])) && !disjoint(out[i], in[k], c))
                return MOA_ERR_INVALID_ARG;
            if (two && in2[k].p && c.any(k) && !disjoint(out[i], in2[k], c)) return MOA_ERR_INVALID_ARG;
            if (w[k] && overlaps(out[i].p, bytes(out[i], c), w[k], wn)) return MOA_ERR_INVALID_ARG;
        }
        if (c.positions && overlaps(out[i].p, bytes(out[i], c), c.positions, tokens * 8 * c.axes)) return MOA_ERR_INVALID_ARG;
        if (c.inv_freq && overlaps(out[i].p, bytes(out[i], c), c.inv_freq, (size_t)c.rot * 2)) return MOA_ERR_INVALID_ARG;
    }
    if (out[0].p && out[1].p && c.any(0) && c.any(1) && !disjoint(out[0], out[1], c)) return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

void fill(RopeProblem& p, const Common& c, const void* const (&w)[2]) {
    for (int i = 0; i < 2; ++i) {
        p.w[i] = w[i];
        p.H[i] = (int)c.heads(i);
    }
    p.pos = reinterpret_cast<const long long*>(c.positions);
    p.freq = c.inv_freq;
    p.B = (int)c.B; p.N = (int)c.N; p.d = (int)c.d; p.rot = (int)c.rot;
    p.axes = c.axes;
    int at = 0;
    for (int a = 0; a < c.axes; ++a) {
        p.first[a] = at;
        if (c.axes > 1) at += (int)c.sections[a];
    }
    p.eps = c.eps;
    p.interleaved = c.interleaved != 0;
    p.bf16 = c.dtype == MOA_BF16;
    p.w_bf16 = c.w_dtype == MOA_BF16;
}

void put(long long (&to)[3], const Strides& s) { to[0] = s.b; to[1] = s.h; to[2] = s.r; }

}  // namespace

extern "C" {

int moa_qk_norm_rope(const void* Q, const void* K, void* Qo, void* Ko, const void* wq,
                     const void* wk, const int64_t* positions, const float* inv_freq, int64_t B,
                     int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t rot,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* qo_strides,
                     const int64_t* ko_strides, int axes, const int64_t* sections, int interleaved,
                     float eps, int dtype, int w_dtype, void* stream) {
    const Common c{B, Hq, Hk, N, d, rot, positions, inv_freq, axes, sections, interleaved, eps, dtype, w_dtype};
    const void* const w[2] = {wq, wk};
    int st = check_common(c, w);
    if (st) return st;
    const View in[2] = {{Q, strides_of(q_strides, Hq, c), Hq}, {K, strides_of(k_strides, Hk, c), Hk}};
    const View out[2] = {{Qo, strides_of(qo_strides, Hq, c), Hq}, {Ko, strides_of(ko_strides, Hk, c), Hk}};
    for (int i = 0; i < 2; ++i)
        if ((st = check_view(in[i], c, i, false)) || (st = check_view(out[i], c, i, true))) return st;
    if ((st = check_buffers(out, in, in, false, c, w))) return st;
    if (!c.any(0) && !c.any(1)) return MOA_OK;
    RopeProblem p{};
    fill(p, c, w);
    for (int i = 0; i < 2; ++i) {
        p.x[i] = in[i].p; p.y[i] = const_cast<void*>(out[i].p);
        put(p.xs[i], in[i].s); put(p.ys[i], out[i].s);
    }
    return hip_status(launch_rope_fwd(p, static_cast<hipStream_t>(stream)));
}

size_t moa_qk_norm_rope_bwd_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d) {
    if (B < 0 || Hq < 0 || Hk < 0 || N < 0 || (d != 64 && d != 128)) return 0;
    return (size_t)kRopeBwdMaxBlocks * 2 * (size_t)d * sizeof(float);
}

int moa_qk_norm_rope_bwd(const void* Q, const void* K, const void* dQo, const void* dKo,
                         const void* wq, const void* wk, const int64_t* positions,
                         const float* inv_freq, void* dQ, void* dK, float* dwq, float* dwk,
                         int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t rot,
                         const int64_t* q_strides, const int64_t* k_strides,
                         const int64_t* dqo_strides, const int64_t* dko_strides,
                         const int64_t* dq_strides, const int64_t* dk_strides, int axes,
                         const int64_t* sections, int interleaved, float eps, int dtype, int w_dtype,
                         void* workspace, size_t workspace_bytes, void* stream) {
    const Common c{B, Hq, Hk, N, d, rot, positions, inv_freq, axes, sections, interleaved, eps, dtype, w_dtype};
    const void* const w[2] = {wq, wk};
    int st = check_common(c, w);
    if (st) return st;
    float* const dw[2] = {wq ? dwq : nullptr, wk ? dwk : nullptr};
    // without weights the forward's input is not read
    const View x[2] = {{wq ? Q : nullptr, strides_of(q_strides, Hq, c), Hq}, {wk ? K : nullptr, strides_of(k_strides, Hk, c), Hk}};
    const View g[2] = {{dQo, strides_of(dqo_strides, Hq, c), Hq}, {dKo, strides_of(dko_strides, Hk, c), Hk}};
    const View out[2] = {{dQ, strides_of(dq_strides, Hq, c), Hq}, {dK, strides_of(dk_strides, Hk, c), Hk}};
    for (int i = 0; i < 2; ++i) {
        if (w[i] && (st = check_view(x[i], c, i, false))) return st;
        if ((st = check_view(g[i], c, i, false)) || (st = check_view(out[i], c, i, true))) return st;
        if (w[i] && (!dw[i] || !aligned16(dw[i]))) return MOA_ERR_INVALID_ARG;
    }
    if (workspace && !aligned16(workspace)) return MOA_ERR_INVALID_ARG;
    const size_t need = wq || wk ? moa_qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, N, d) : 0;
    if (need && (!workspace || workspace_bytes < need)) return MOA_ERR_WORKSPACE;
    if ((st = check_buffers(out, g, x, true, c, w))) return st;
    // the weights' gradients and the workspace against everything
    struct Buf { const void* p; size_t n; };
    const size_t wn = (size_t)d * (w_dtype == MOA_F32 ? 4 : 2), dn = (size_t)d * 4, tokens = (size_t)(B * N);
    const Buf outs[] = {{dw[0], dw[0] ? dn : 0}, {dw[1], dw[1] ? dn : 0}, {workspace, need}};
    const auto all = [&](const View& v, int i) { return Buf{v.p, v.p && c.any(i) ? bytes(v, c) : 0}; };
    const Buf rest[] = {all(x[0], 0), all(x[1], 1), all(g[0], 0), all(g[1], 1), all(out[0], 0), all(out[1], 1),
                        {wq, wq ? wn : 0}, {wk, wk ? wn : 0}, {positions, positions ? tokens * 8 * axes : 0},
                        {inv_freq, inv_freq ? (size_t)rot * 2 : 0}};
    for (int i = 0; i < 3; ++i) {
        for (const Buf& b : rest)
            if (overlaps(outs[i].p, outs[i].n, b.p, b.n)) return MOA_ERR_INVALID_ARG;
        for (int k = i + 1; k < 3; ++k)
            if (overlaps(outs[i].p, outs[i].n, outs[k].p, outs[k].n)) return MOA_ERR_INVALID_ARG;
    }
    if (!c.any(0) && !c.any(1) && !need) return MOA_OK;
    RopeProblem p{};
    fill(p, c, w);
    for (int i = 0; i < 2; ++i) {
        p.x[i] = x[i].p; p.g[i] = g[i].p; p.y[i] = const_cast<void*>(out[i].p); p.dw[i] = dw[i];
        put(p.xs[i], x[i].s); put(p.gs[i], g[i].s); put(p.ys[i], out[i].s);
    }
    p.ws = static_cast<float*>(workspace);
    return hip_status(launch_rope_bwd(p, static_cast<hipStream_t>(stream)));
}

// Words: the arguments in their order, but 4 for each tensor's strides (the last
// not read), and a flag and 4 for the sections.
int moa_packed_qk_norm_rope(const int64_t* a) {
    using packed::Ptr;
    return moa_qk_norm_rope(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, Ptr{a[6]}, Ptr{a[7]},
                            a[8], a[9], a[10], a[11], a[12], a[13], a + 14, a + 18, a + 22, a + 26, (int)a[30],
                            a[31] ? a + 32 : nullptr, (int)a[36], packed::real(a[37]), (int)a[38], (int)a[39],
                            Ptr{a[40]});
}

int moa_packed_qk_norm_rope_bwd(const int64_t* a) {
    using packed::Ptr;
    return moa_qk_norm_rope_bwd(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, Ptr{a[6]},
                                Ptr{a[7]}, Ptr{a[8]}, Ptr{a[9]}, Ptr{a[10]}, Ptr{a[11]}, a[12], a[13], a[14], a[15],
                                a[16], a[17], a + 18, a + 22, a + 26, a + 30, a + 34, a + 38, (int)a[42],
                                a[43] ? a + 44 : nullptr, (int)a[48], packed::real(a[49]), (int)a[50], (int)a[51],
                                Ptr{a[52]}, (size_t)a[53], Ptr{a[54]});
}

}  // extern "C"
