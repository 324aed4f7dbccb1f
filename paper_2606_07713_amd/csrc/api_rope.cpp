// C-ABI front end of the head norms with rotation (moa_rope.h): argument
// validation and dispatch.  Host code; allocates nothing, never synchronises.
#include "../../include/moa_rope.h"
#include "api_rope.h"
#include "packed.h"

using namespace moa;
using namespace moa::rope;

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
