// Checks of the arguments of the head norms with rotation, for moa_rope.h's entry
// points and the appending to a paged cache (host code only).
#pragma once

#include <cmath>
#include <limits>

#include "api_checks.h"
#include "rope.h"

namespace moa {
namespace rope {

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

inline int check_common(const Common& c, const void* const (&w)[2]) {
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

inline int check_view(const View& v, const Common& c, int i, bool out) {
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

inline size_t bytes(const View& v, const Common& c) { return extent_bytes(v.s, c.B, v.H, c.N, c.d, c.es()); }

// Whether two views certainly share no element: their byte ranges do not meet,
// or they take turns in one buffer: whole batches, or the heads of one token, be
// they [B][N][heads] or [N][B][heads].
inline bool disjoint(const View& a, const View& b, const Common& c) {
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

inline bool same(const View& a, const View& b) {
    return a.p == b.p && a.s.b == b.s.b && a.s.h == b.s.h && a.s.r == b.s.r;
}

// A dimension of size 1 has no stride to keep to.
inline Strides strides_of(const int64_t* s, int64_t H, const Common& c) {
    return s ? Strides{c.B > 1 ? s[0] : 0, H > 1 ? s[1] : 0, c.N > 1 ? s[2] : 0} : contiguous(H, c.N, c.d);
}

// Outputs against every input and each other; out[i] may be its own in[i].
inline int check_buffers(const View (&out)[2], const View (&in)[2], const View (&in2)[2], bool two, const Common& c,
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

inline void fill(RopeProblem& p, const Common& c, const void* const (&w)[2]) {
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

}  // namespace rope
}  // namespace moa
