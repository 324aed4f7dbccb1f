// C-ABI front end of the appending to a paged cache (moa_paged.h): argument
// validation and dispatch.  Host code; allocates nothing, never synchronises.
#include "../../include/moa_paged.h"
#include "api_pools.h"
#include "api_rope.h"
#include "packed.h"
#include "paged.h"

using namespace moa;
using namespace moa::rope;

extern "C" {

int moa_paged_append(const void* Q, const void* K, const void* V, void* Qo, void* k_pool,
                     void* v_pool, const void* wq, const void* wk, const int64_t* positions,
                     const float* inv_freq, const int32_t* seq_lens, const int32_t* new_lens,
                     const int32_t* page_table, int64_t B, int64_t Hq, int64_t Hk, int64_t N,
                     int64_t d, int64_t rot, int64_t page, int64_t num_pages, int64_t max_pages,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* v_strides,
                     const int64_t* qo_strides, const int64_t* k_pool_strides,
                     const int64_t* v_pool_strides, int axes, const int64_t* sections,
                     int interleaved, float eps, int dtype, int w_dtype, void* stream) {
    const Common c{B, Hq, Hk, N, d, rot, positions, inv_freq, axes, sections, interleaved, eps, dtype, w_dtype};
    const Pools pools{page, num_pages, max_pages, seq_lens, new_lens, page_table};
    const void* const w[2] = {wq, wk};
    int st = check_common(c, w);
    if (st) return st;
    // two tensors of Hk heads are walked over
    if (B * N > 0 && Hq + 2 * Hk > std::numeric_limits<int32_t>::max() / (B * N)) return MOA_ERR_UNSUPPORTED;
    const bool any = c.any(0) || c.any(1);
    if ((st = check_pools(pools, B, N, any))) return st;
    const View q{Q, strides_of(q_strides, Hq, c), Hq}, k{K, strides_of(k_strides, Hk, c), Hk}, v{V, strides_of(v_strides, Hk, c), Hk};
    const View qo{Qo, strides_of(qo_strides, Hq, c), Hq};
    Common out = c;   // outputs are bf16
    out.dtype = MOA_BF16;
    if ((st = check_view(q, c, 0, false)) || (st = check_view(k, c, 1, false)) || (st = check_view(v, c, 1, false)) ||
        (st = check_view(qo, out, 0, true)))
        return st;
    const View kp{k_pool, moa::strides_of(k_pool_strides, num_pages, Hk, page, d), Hk};
    const View vp{v_pool, moa::strides_of(v_pool_strides, num_pages, Hk, page, d), Hk};
    if ((st = check_pool(k_pool, kp.s, pools, Hk, d, true)) || (st = check_pool(v_pool, vp.s, pools, Hk, d, true))) return st;
    if (!any) return MOA_OK;
    const Common pool{num_pages, Hk, Hk, page, d, 0, nullptr, nullptr, 1, nullptr, 0, 0, MOA_BF16, MOA_BF16};
    const auto size = [](const View& x, const Common& s, int i) { return Buf{x.p, x.p && s.any(i) ? bytes(x, s) : 0}; };
    const Lists lists(pools, B);
    const size_t wn = (size_t)d * (w_dtype == MOA_F32 ? 4 : 2);
    const Buf to_q = size(qo, out, 0), to_k = size(kp, pool, 1), to_v = size(vp, pool, 1);
    const Buf ins[] = {size(q, c, 0), size(k, c, 1), size(v, c, 1)};
    const Buf small[] = {{wq, wq ? wn : 0}, {wk, wk ? wn : 0}, {positions, positions ? (size_t)(B * N) * 8 * (size_t)axes : 0},
                         {inv_freq, inv_freq ? (size_t)rot * 2 : 0}, lists.b[0], lists.b[1], lists.b[2]};
    for (const Buf& o : {to_q, to_k, to_v})
        for (const Buf& b : small)
            if (meet(o, b)) return MOA_ERR_INVALID_ARG;
    // the pools against the call's tensors and each other
    for (const Buf& o : {to_k, to_v})
        for (const Buf& b : {ins[0], ins[1], ins[2], to_q})
            if (meet(o, b)) return MOA_ERR_INVALID_ARG;
    if (meet(to_k, to_v) && !disjoint(kp, vp, pool)) return MOA_ERR_INVALID_ARG;
    // Qo in Q's place, or beside the inputs in one packed buffer of their type
    if (meet(to_q, ins[0]) && !(dtype == MOA_BF16 && (same(qo, q) || disjoint(qo, q, c)))) return MOA_ERR_INVALID_ARG;
    if (meet(to_q, ins[1]) && !(dtype == MOA_BF16 && disjoint(qo, k, c))) return MOA_ERR_INVALID_ARG;
    if (meet(to_q, ins[2]) && !(dtype == MOA_BF16 && disjoint(qo, v, c))) return MOA_ERR_INVALID_ARG;
    AppendProblem p{};
    fill(p.r, c, w);
    p.r.x[0] = Q; p.r.x[1] = K; p.r.y[0] = Qo;
    put(p.r.xs[0], q.s); put(p.r.xs[1], k.s); put(p.r.ys[0], qo.s);
    p.v = V;
    put(p.vs, v.s);
    p.to = source_of(pools, k_pool, v_pool, kp.s, vp.s);
    return hip_status(launch_paged_append(p, static_cast<hipStream_t>(stream)));
}

// Words: the arguments in their order, but 4 for each tensor's strides (the last
// not read), and a flag and 4 for the sections.
int moa_packed_paged_append(const int64_t* a) {
    using packed::Ptr;
    return moa_paged_append(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, Ptr{a[6]}, Ptr{a[7]},
                            Ptr{a[8]}, Ptr{a[9]}, Ptr{a[10]}, Ptr{a[11]}, Ptr{a[12]}, a[13], a[14], a[15], a[16], a[17],
                            a[18], a[19], a[20], a[21], a + 22, a + 26, a + 30, a + 34, a + 38, a + 42, (int)a[46],
                            a[47] ? a + 48 : nullptr, (int)a[52], packed::real(a[53]), (int)a[54], (int)a[55], Ptr{a[56]});
}

}  // extern "C"
