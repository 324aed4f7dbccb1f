// C-ABI front end of the four-bit key/value cache (moa_kv4.h): argument
// validation, split choice and dispatch.  Host code; allocates nothing, never
// synchronises.
#include <cmath>
#include <limits>

#include "../../include/moa_kv4.h"
#include "api_checks.h"
#include "kv4.h"
#include "packed.h"

namespace {

using namespace moa;

constexpr int64_t kLim = std::numeric_limits<int32_t>::max();
constexpr int64_t kMaxPage = int64_t(1) << 20;
constexpr int kMaxSplits = 256;
constexpr float kMaxScale = 0x1p127f;   // times log2(e) is still finite
// Workgroups of 256 threads in one launch: its threads are counted in 32 bits.
constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;

struct Dims {
    int64_t B, Hk, N, d, page, num_pages, max_pages;
    const void* cache;
    const int32_t *seq_lens, *new_lens, *table;
    bool any() const { return B > 0 && Hk > 0 && N > 0; }
    size_t cache_bytes() const { return (size_t)num_pages * (size_t)Hk * moa_kv4_page_bytes(page, d); }
};

int check_dims(const Dims& s) {
    if (s.B < 0 || s.Hk < 0 || s.N < 0 || s.d < 1 || s.page < 1 || s.num_pages < 0 || s.max_pages < 0)
        return MOA_ERR_INVALID_ARG;
    if (s.d != 64 && s.d != 128) return MOA_ERR_UNSUPPORTED;
    if (!moa_kv4_page_bytes(s.page, s.d)) return MOA_ERR_UNSUPPORTED;
    if (s.B > kLim || s.Hk > kLim || s.N > kLim - 6 || s.num_pages > kLim || s.max_pages > kLim / s.page)
        return MOA_ERR_UNSUPPORTED;
    if (s.B * s.Hk > kLim || (s.B * s.Hk > 0 && s.N + 6 > kLim / 2 / (s.B * s.Hk))) return MOA_ERR_UNSUPPORTED;
    if (s.num_pages > 0 && s.Hk > (int64_t(1) << 46) / s.num_pages / (int64_t)moa_kv4_page_bytes(s.page, s.d))
        return MOA_ERR_UNSUPPORTED;
    if (!s.table && s.any() && (s.max_pages != 1 || s.num_pages < s.B)) return MOA_ERR_INVALID_ARG;
    if (s.any() && !s.seq_lens) return MOA_ERR_INVALID_ARG;
    if (s.any() && !s.cache && s.num_pages > 0) return MOA_ERR_INVALID_ARG;
    if (!aligned16(s.cache)) return MOA_ERR_INVALID_ARG;
    for (const void* p : {s.seq_lens, s.new_lens, s.table})
        if (reinterpret_cast<uintptr_t>(p) & 3) return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

// The arrays that tell where tokens are.
struct Lists {
    Buf b[3];
    explicit Lists(const Dims& s)
        : b{{s.seq_lens, (size_t)s.B * 4}, {s.new_lens, s.new_lens ? (size_t)s.B * 4 : 0},
            {s.table, s.table ? (size_t)s.B * (size_t)s.max_pages * 4 : 0}} {}
    bool meet(const Buf& x) const {
        for (const Buf& y : b)
            if (overlaps(x.p, x.n, y.p, y.n)) return true;
        return false;
    }
};

Kv4Cache cache_of(const Dims& s) {
    Kv4Cache c;
    c.base = static_cast<unsigned char*>(const_cast<void*>(s.cache));
    c.seq_lens = s.seq_lens; c.new_lens = s.new_lens; c.table = s.table;
    c.page_bytes = (long long)moa_kv4_page_bytes(s.page, s.d);
    c.B = (int)s.B; c.hk = (int)s.Hk; c.n = (int)s.N; c.d = (int)s.d;
    c.page = (int)s.page; c.num_pages = (int)s.num_pages; c.max_pages = (int)s.max_pages;
    return c;
}

// Key splits of the attention.  A workgroup's four waves take its 64-key tiles
// in steps of four; starting and ending it costs about two steps, and the
// second pass about three, one more for every 16 splits and for every 6 MB of
// partial states.  `wave` workgroups run at a time: one per compute unit where
// up to 16 rows of d = 128 leave it to the memory, two where a tile is half as
// large or its work twice (measured, splits:us, 32 heads on 8: one query, 4097
// keys, d = 128 1:26.1 8:11.3 17:9.1 64:11.4; 16384 1:85 16:13.3 32:11.1 64:14.3;
// 48 queries of 8192 1:79.0 2:75.9 4:78.1, 64 of them 1:94.0 2:96.3; 200 queries
// of one sequence on 20011 keys 1:143 2:124 4:123 5:106 8:115, 512 on 8192 1:98
// 2:108).
int pick_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t max_len, int requested) {
    if (requested > 0) return requested;
    const int64_t rows = N * (Hq / Hk), per = kv4_rows_per_block((int)rows);
    const int64_t blocks = B * Hk * ((rows + per - 1) / per), tiles = (max_len + 63) / 64;
    const int64_t wave = rows <= 16 && d == 128 ? 256 : 512;
    const double states = (double)(B * Hq * N) * (double)d * sizeof(float) / 6e6;
    int best = 1;
    double least = 0;
    for (int64_t s = 1; s <= kMaxSplits && s <= tiles && (s == 1 || s * blocks <= 4 * wave); ++s) {
        const int64_t rounds = (s * blocks + wave - 1) / wave, steps = ((tiles + s - 1) / s + 3) / 4;
        const double cost = (double)(rounds * (steps + 2)) + (s > 1 ? 3 + (double)s / 16 + (double)s * states : 0);
        if (s == 1 || cost < least) {
            best = (int)s;
            least = cost;
        }
    }
    return best;
}

bool attn_sizes_ok(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page, int64_t max_pages,
                   int64_t max_len, int num_splits) {
    if (B < 0 || Hq < 0 || Hk < 1 || N < 0 || max_pages < 0 || max_len < 0 || Hq % Hk) return false;
    if (num_splits < 0 || num_splits > kMaxSplits || !moa_kv4_page_bytes(page, d)) return false;
    if (B > kLim || Hq > kLim || N > kLim || max_pages > kLim / page) return false;
    if (B * Hq > kLim || (B * Hq > 0 && N > (kMaxBlocks * 4) / (B * Hq))) return false;   // four rows a workgroup in the second pass
    const int64_t rows = N * (Hq / Hk), per = kv4_rows_per_block((int)rows);
    return B * Hk * ((rows + per - 1) / per) <= kMaxBlocks / (num_splits > 0 ? num_splits : 1);
}

// Partial states of a call with these splits (none with one).
size_t states_bytes(int64_t B, int64_t Hq, int64_t N, int64_t d, int splits) {
    if (splits <= 1) return 0;
    return align256((size_t)(B * Hq * N) * (size_t)splits * (size_t)(d + 2) * sizeof(float));
}

}  // namespace

extern "C" {

size_t moa_kv4_page_bytes(int64_t page, int64_t d) {
    if ((d != 64 && d != 128) || page < 64 || page % 64 || page > kMaxPage) return 0;
    return (size_t)page * (size_t)(d + d / 16);
}

int moa_kv4_write(const void* K, const void* V, void* cache, const int32_t* seq_lens,
                  const int32_t* new_lens, const int32_t* page_table, int64_t B, int64_t Hk,
                  int64_t N, int64_t d, int64_t page, int64_t num_pages, int64_t max_pages,
                  const int64_t* k_strides, const int64_t* v_strides, int in_dtype, void* stream) {
    const Dims s{B, Hk, N, d, page, num_pages, max_pages, cache, seq_lens, new_lens, page_table};
    if (in_dtype != MOA_F32 && in_dtype != MOA_BF16) return MOA_ERR_INVALID_ARG;
    int st = check_dims(s);
    if (st) return st;
    if (s.any() && kv4_row_blocks(B, Hk, N, d) > kMaxBlocks) return MOA_ERR_UNSUPPORTED;
    const size_t es = in_dtype == MOA_F32 ? 4 : 2;
    const Strides sk = strides_of(k_strides, B, Hk, N, d), sv = strides_of(v_strides, B, Hk, N, d);
    if ((st = check_tensor(K, sk, B, Hk, N, d, es, false)) || (st = check_tensor(V, sv, B, Hk, N, d, es, false))) return st;
    if (!s.any() || num_pages == 0) return MOA_OK;
    const Buf pool{cache, s.cache_bytes()};
    if (Lists(s).meet(pool) || meet(pool, {K, extent_bytes(sk, B, Hk, N, d, es)}) ||
        meet(pool, {V, extent_bytes(sv, B, Hk, N, d, es)}))
        return MOA_ERR_INVALID_ARG;
    Kv4Rows p{};
    p.c = cache_of(s);
    p.kin = K; p.vin = V;
    put(p.ks, sk); put(p.vs, sv);
    p.bf16 = in_dtype == MOA_BF16;
    return hip_status(launch_kv4_write(p, static_cast<hipStream_t>(stream)));
}

int moa_kv4_read(const void* cache, void* K, void* V, const int32_t* seq_lens,
                 const int32_t* new_lens, const int32_t* page_table, int64_t B, int64_t Hk,
                 int64_t N, int64_t d, int64_t page, int64_t num_pages, int64_t max_pages,
                 const int64_t* k_strides, const int64_t* v_strides, int out_dtype, void* stream) {
    const Dims s{B, Hk, N, d, page, num_pages, max_pages, cache, seq_lens, new_lens, page_table};
    if (out_dtype != MOA_F32 && out_dtype != MOA_BF16) return MOA_ERR_INVALID_ARG;
    int st = check_dims(s);
    if (st) return st;
    if (s.any() && kv4_row_blocks(B, Hk, N, d) > kMaxBlocks) return MOA_ERR_UNSUPPORTED;
    const size_t es = out_dtype == MOA_F32 ? 4 : 2;
    const Strides sk = strides_of(k_strides, B, Hk, N, d), sv = strides_of(v_strides, B, Hk, N, d);
    if ((st = check_tensor(K, sk, B, Hk, N, d, es, true)) || (st = check_tensor(V, sv, B, Hk, N, d, es, true))) return st;
    if (!s.any() || num_pages == 0) return MOA_OK;
    const Buf pool{cache, s.cache_bytes()}, k{K, extent_bytes(sk, B, Hk, N, d, es)}, v{V, extent_bytes(sv, B, Hk, N, d, es)};
    const Lists lists(s);
    if (meet(k, v) || meet(k, pool) || meet(v, pool) || lists.meet(k) || lists.meet(v)) return MOA_ERR_INVALID_ARG;
    Kv4Rows p{};
    p.c = cache_of(s);
    p.kout = K; p.vout = V;
    put(p.ks, sk); put(p.vs, sv);
    p.bf16 = out_dtype == MOA_BF16;
    return hip_status(launch_kv4_read(p, static_cast<hipStream_t>(stream)));
}

int moa_kv4_attn_num_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page,
                            int64_t max_pages, int64_t max_len, int num_splits) {
    if (!attn_sizes_ok(B, Hq, Hk, N, d, page, max_pages, max_len, num_splits) || B * Hq * N == 0) return 1;
    const int64_t cap = max_pages * page;
    return pick_splits(B, Hq, Hk, N, d, max_len > 0 && max_len < cap ? max_len : cap, num_splits);
}

size_t moa_kv4_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d,
                                    int64_t page, int64_t max_pages, int64_t max_len,
                                    int num_splits) {
    return states_bytes(B, Hq, N, d, moa_kv4_attn_num_splits(B, Hq, Hk, N, d, page, max_pages, max_len, num_splits));
}

int moa_kv4_attn_fwd(const void* Q, const void* cache, void* O, float* LSE, const int32_t* seq_lens,
                     const int32_t* new_lens, const int32_t* page_table, int64_t B, int64_t Hq,
                     int64_t Hk, int64_t N, int64_t d, int64_t page, int64_t num_pages,
                     int64_t max_pages, int64_t max_len, const int64_t* q_strides,
                     const int64_t* o_strides, float scale, int causal, int out_dtype,
                     void* workspace, size_t workspace_bytes, int num_splits, void* stream) {
    const Dims s{B, Hk, N, d, page, num_pages, max_pages, cache, seq_lens, new_lens, page_table};
    if (out_dtype != MOA_F32 && out_dtype != MOA_BF16) return MOA_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || (causal != 0 && causal != 1)) return MOA_ERR_INVALID_ARG;
    if (num_splits < 0 || num_splits > kMaxSplits || max_len < 0) return MOA_ERR_INVALID_ARG;
    if (Hq < 0 || Hk < 1 || Hq % Hk) return MOA_ERR_INVALID_ARG;
    int st = check_dims(s);
    if (st) return st;
    if (!attn_sizes_ok(B, Hq, Hk, N, d, page, max_pages, max_len, num_splits)) return MOA_ERR_UNSUPPORTED;
    if (std::fabs(scale) > kMaxScale) return MOA_ERR_UNSUPPORTED;
    const Strides sq = strides_of(q_strides, B, Hq, N, d), so = strides_of(o_strides, B, Hq, N, d);
    const size_t oes = out_dtype == MOA_F32 ? 4 : 2;
    if ((st = check_tensor(Q, sq, B, Hq, N, d, 2, false)) || (st = check_tensor(O, so, B, Hq, N, d, oes, true))) return st;
    if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(LSE) & 3)) return MOA_ERR_INVALID_ARG;
    if (!s.any() || Hq == 0) return MOA_OK;
    const int splits = moa_kv4_attn_num_splits(B, Hq, Hk, N, d, page, max_pages, max_len, num_splits);
    const size_t need = states_bytes(B, Hq, N, d, splits);
    if (need && (!workspace || workspace_bytes < need)) return MOA_ERR_WORKSPACE;
    const Buf ins[] = {{Q, extent_bytes(sq, B, Hq, N, d, 2)}, {cache, s.cache_bytes()}};
    const Buf outs[] = {{O, extent_bytes(so, B, Hq, N, d, oes)}, {LSE, LSE ? (size_t)(B * Hq * N) * 4 : 0}, {workspace, need}};
    const Lists lists(s);
    for (int i = 0; i < 3; ++i) {
        for (const Buf& x : ins)
            if (meet(outs[i], x)) return MOA_ERR_INVALID_ARG;
        if (lists.meet(outs[i])) return MOA_ERR_INVALID_ARG;
        for (int k = i + 1; k < 3; ++k)
            if (meet(outs[i], outs[k])) return MOA_ERR_INVALID_ARG;
    }
    Kv4Attn p{};
    p.c = cache_of(s);
    p.q = Q; p.o = O; p.lse = LSE;
    put(p.qs, sq); put(p.os, so);
    p.hq = (int)Hq;
    p.scale = scale;
    p.causal = causal != 0;
    p.out_bf16 = out_dtype == MOA_BF16;
    p.splits = splits;
    p.ws = static_cast<float*>(workspace);
    return hip_status(launch_kv4_attn(p, static_cast<hipStream_t>(stream)));
}

// Words: the arguments in their order, but 4 for each tensor's strides (the last
// not read).
int moa_packed_kv4_write(const int64_t* a) {
    using packed::Ptr;
    return moa_kv4_write(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, a[6], a[7], a[8], a[9],
                         a[10], a[11], a[12], a + 13, a + 17, (int)a[21], Ptr{a[22]});
}

int moa_packed_kv4_read(const int64_t* a) {
    using packed::Ptr;
    return moa_kv4_read(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, a[6], a[7], a[8], a[9],
                        a[10], a[11], a[12], a + 13, a + 17, (int)a[21], Ptr{a[22]});
}

int moa_packed_kv4_attn_fwd(const int64_t* a) {
    using packed::Ptr;
    return moa_kv4_attn_fwd(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, Ptr{a[6]}, a[7], a[8],
                            a[9], a[10], a[11], a[12], a[13], a[14], a[15], a + 16, a + 20, packed::real(a[24]),
                            (int)a[25], (int)a[26], Ptr{a[27]}, (size_t)a[28], (int)a[29], Ptr{a[30]});
}

}  // extern "C"
