// C-ABI front end of the attention with a window, on whole tensors (moa_window.h)
// and over the paged cache (moa_paged.h): argument validation, split choice and
// dispatch.  Host code; allocates nothing, never synchronises.
#include <algorithm>
#include <cmath>

#include "../../include/moa_paged.h"
#include "../../include/moa_window.h"
#include "api_pools.h"
#include "packed.h"
#include "win.h"

namespace {

using namespace moa;

constexpr int64_t kMaxRows = int64_t(1) << 26;          // B * Hq * N
constexpr int64_t kMaxStageStride = int64_t(1) << 23;   // 64 rows' bytes stay in 32 bits
constexpr float kMaxScale = 0x1p127f;           // times log2(e) is still finite
// Workgroups of 256 threads in one launch: its threads are counted in 32 bits.
constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;
constexpr int64_t kMaxJoinedRows = 4 * kMaxBlocks;      // four rows a workgroup where splits are joined

// The sizes of an attention call; Nk: keys of a sequence, at most; left, right: -1
// where there is no limit, below kMost else, so that sums of them hold.
struct Sizes {
    int64_t B, Hq, Hk, N, Nk, d, left, right, sinks;
    Sizes(int64_t B_, int64_t Hq_, int64_t Hk_, int64_t N_, int64_t Nk_, int64_t d_, int64_t left_, int64_t right_, int64_t sinks_)
        : B(B_), Hq(Hq_), Hk(Hk_), N(N_), Nk(Nk_), d(d_), left(limit(left_)), right(limit(right_)), sinks(std::min(sinks_, kMost)) {}
    static int64_t limit(int64_t x) { return x < 0 || x >= kMost ? -1 : x; }
    int64_t rows() const { return N * (Hq / Hk); }
    int64_t per() const { return win_rows_per_block(rows()); }
    int64_t tiles() const { return (rows() + per() - 1) / per(); }
    int64_t groups() const { return B * Hk * tiles(); }
    bool any() const { return B > 0 && Hq > 0 && N > 0; }
};

// MOA_OK, or what is wrong.
int check_sizes(const Sizes& s, int num_splits) {
    if (s.B < 0 || s.Hq < 0 || s.Hk < 1 || s.N < 0 || s.Nk < 0 || s.d < 1 || s.Hq % s.Hk || s.sinks < 0) return MOA_ERR_INVALID_ARG;
    if (num_splits < 0 || num_splits > kMaxSplits) return MOA_ERR_INVALID_ARG;
    if (s.d != 64 && s.d != 128) return MOA_ERR_UNSUPPORTED;
    if (s.B >= kMaxRows || s.Hq >= kMaxRows || s.Hk >= kMaxRows || s.N > kMost || s.Nk > kMost) return MOA_ERR_UNSUPPORTED;
    if (s.B * std::max(s.Hq, s.Hk) >= kMaxRows) return MOA_ERR_UNSUPPORTED;
    if (s.B * s.Hq > 0 && s.N >= (kMaxRows + s.B * s.Hq - 1) / (s.B * s.Hq)) return MOA_ERR_UNSUPPORTED;
    if (s.any() && s.groups() > kMaxBlocks / std::max(num_splits, 1)) return MOA_ERR_UNSUPPORTED;
    if (num_splits > 1 && s.any() && s.B * s.Hq * s.N > kMaxJoinedRows) return MOA_ERR_UNSUPPORTED;   // (by itself none splits so many)
    return MOA_OK;
}

// Keys that one row tile walks over, at most.
int64_t span(const Sizes& s) {
    if (s.left < 0) return s.Nk;
    const int64_t positions = std::min(s.N, s.per() / std::max<int64_t>(1, s.Hq / s.Hk) + 1);
    const int64_t ahead = s.right < 0 ? s.Nk : s.right;
    return std::min(s.Nk, s.left + ahead + positions + std::min(s.sinks, s.Nk));
}

// Key splits, by an estimate of the call's microseconds.  A workgroup walks over
// `steps` tiles (of 64 keys with many rows; of 128, four waves' 32, with few), and
// beginning and ending cost it two more.  A tile takes the longer the more workgroups
// share a compute unit; more than `most` run one after the other.  With many rows and
// one workgroup for a unit its two key streams take a tile each at a time.  Few rows
// also wait for the memory.  The join reads what the splits wrote, a latency more
// beyond 32 of them.  (Measured, splits:us.  Many rows: 32 heads on 8, 200 of 20011
// keys, d = 128 1:310 4:95 8:94 9:89 12:110; 8 on 2, 4 x 1000, d = 64 1:16 2:30 4:29;
// 8 heads, 500 of 4096, d = 128 4:31 8:25 12:33; 12 on 4, 2 x 700 of 5000, d = 64 1:58
// 3:50 5:46 8:51; 32 on 8, 300 in a window of 1024 1:25 3:27 5:26.  Few: 32 on 8, one
// query of 4097, d = 128 1:42 8:16 16:13 32:11 64:13; of 16384 1:195 16:24 32:17 48:21;
// 8 on 1, 32 x 3 of 9000 4:46 8:34 16:43; 12 on 4, 16 x 4 in a window of 1024, d = 64
// 1:11.3 4:10.6 6:12.7 16:14.)
int pick_splits(const Sizes& s, int requested) {
    if (!s.any()) return 1;
    if (requested > 0) return requested;
    const bool few = s.per() < 128, wide = s.d == 128;
    const int64_t blocks = s.groups(), keys = few ? 128 : 64, all = std::max<int64_t>(1, (span(s) + keys - 1) / keys);
    const int64_t most = few ? (s.per() == 32 ? (wide ? 1 : 2) : (wide ? 2 : 4)) : wide ? 2 : 3;
    const double one = few ? 1.3 : wide ? 2.2 : 1.5, more = few ? 0.4 : wide ? 0.27 : 0.23;   // us, and share of it for each further workgroup
    const double rows = (double)(s.B * s.Hq * s.N), memory = few ? (double)(s.B * s.Hk * span(s)) * (double)s.d * 4 / 6.5e6 : 0;
    const auto tile = [&](int64_t at_once) { return at_once ? one * (1 + more * (double)(at_once - 1)) : 0.0; };
    int best = 1;
    double least = 0;
    for (int64_t k = 1; k <= 128 && k <= all && (k == 1 || k * blocks <= 1024); ++k) {
        const int64_t each = (k * blocks + 255) / 256;   // workgroups of a compute unit
        const double walk = (double)(each / most) * tile(most) + tile(each % most);
        const int64_t steps = (all + k - 1) / k;
        double cost = few ? walk * ((double)all / (double)k + 2.5) + memory
                    : each == 1 ? tile(2) * (double)((steps + 1) / 2 + 2)   // two key streams
                                : walk * (double)(steps + 2);
        if (k > 1) cost += 3 + rows * ((double)k * (double)(s.d + 2) * 8 / 5e6 + 1.0 / 8000) + 3 * (double)((k - 1) / 32);
        if (k == 1 || cost < least) {
            best = (int)k;
            least = cost;
        }
    }
    return best;
}

// Partial states of a call with these splits (none with one).
size_t states_bytes(const Sizes& s, int splits) {
    if (splits <= 1) return 0;
    return align256((size_t)(s.B * s.Hq * s.N) * (size_t)splits * (size_t)(s.d + 2) * sizeof(float));
}

int limit(int64_t x) { return x < 0 ? kNoLimit : (int)x; }

Window window_of(const Sizes& s) { return {limit(s.left), limit(s.right), (int)s.sinks}; }

// What both entry points check and do once their keys are known.  `keys`: the
// ranges that the call reads besides Q.
struct Call {
    const void* Q;
    void* O;
    float* LSE;
    Strides sq, so;
    float scale;
    int out_dtype;
    void* ws;
    size_t ws_bytes;
    int splits;
    void* stream;
};

int check_call(const Call& c, const Sizes& s) {
    const size_t es = c.out_dtype == MOA_F32 ? 4 : 2;
    int st;
    if ((st = check_tensor(c.Q, c.sq, s.B, s.Hq, s.N, s.d, 2, false)) || (st = check_tensor(c.O, c.so, s.B, s.Hq, s.N, s.d, es, true))) return st;
    if (!aligned16(c.ws) || (reinterpret_cast<uintptr_t>(c.LSE) & 3)) return MOA_ERR_INVALID_ARG;
    if (std::fabs(c.scale) > kMaxScale) return MOA_ERR_UNSUPPORTED;
    return MOA_OK;
}

int run(const Call& c, const Sizes& s, const KeySource& src, const Buf* keys, int n_keys) {
    const size_t es = c.out_dtype == MOA_F32 ? 4 : 2, need = states_bytes(s, c.splits);
    if (need && (!c.ws || c.ws_bytes < need)) return MOA_ERR_WORKSPACE;
    const Buf q{c.Q, extent_bytes(c.sq, s.B, s.Hq, s.N, s.d, 2)};
    const Buf outs[] = {{c.O, extent_bytes(c.so, s.B, s.Hq, s.N, s.d, es)},
                        {c.LSE, c.LSE ? (size_t)(s.B * s.Hq * s.N) * 4 : 0}, {c.ws, need}};
    for (int i = 0; i < 3; ++i) {
        if (meet(outs[i], q)) return MOA_ERR_INVALID_ARG;
        for (int k = 0; k < n_keys; ++k)
            if (meet(outs[i], keys[k])) return MOA_ERR_INVALID_ARG;
        for (int k = i + 1; k < 3; ++k)
            if (meet(outs[i], outs[k])) return MOA_ERR_INVALID_ARG;
    }
    WinAttn p{};
    p.s = src;
    p.w = window_of(s);
    p.q = c.Q; p.o = c.O; p.lse = c.LSE;
    put(p.qs, c.sq); put(p.os, c.so);
    p.B = (int)s.B; p.hq = (int)s.Hq; p.hk = (int)s.Hk; p.n = (int)s.N; p.d = (int)s.d;
    p.scale = c.scale;
    p.out_bf16 = c.out_dtype == MOA_BF16;
    p.splits = c.splits;
    p.ws = static_cast<float*>(c.ws);
    return hip_status(launch_win_attn(p, static_cast<hipStream_t>(c.stream)));
}

// Chunks of the queries that see only the first keys of a sequence, 0 if there are
// none: as many as fill the GPU once, of six stages at least, and at most 64.
int far_chunks(const Sizes& s) {
    if (s.left < 0 || !s.any() || s.Nk == 0) return 0;
    const int64_t tiles = win_sink_tiles(window_of(s), (int)s.Nk);
    if (tiles == 0) return 0;
    // the first tile's windows end here
    const int64_t near = std::clamp<int64_t>(std::min<int64_t>(kWinKeyTile, s.Nk) - (s.Nk - s.N) + s.left, 0, s.N);
    const int64_t behind = (s.N - near + kWinStage - 1) / kWinStage * (s.Hq / s.Hk);
    if (behind == 0) return 0;
    const int64_t fill = 256 / (s.B * s.Hk * tiles);
    return (int)std::clamp<int64_t>(std::min(fill, behind / 6), 1, std::max<int64_t>(1, 64 / tiles));
}

// Parts of the queries of the key tiles, where the tiles alone do not fill the GPU: so
// many for the tile with most of them, and as long ones for the others.  A workgroup
// takes a stage of 64 queries in about 1.5 us (256 run at a time), starting and ending
// it costs about four of these, joining about two and one for every 12 MB of partial
// sums.  (Where tiles differ, parts of one length are 7 for the first tile of 4 x 1000
// causal tokens, 8 heads on 2, d = 64, and 1 for the last: 25 us where 4 for each take 31.)
struct Parts {
    int most, stages;
};
Parts near_parts(const Sizes& s) {
    if (!s.any() || s.Nk == 0) return {1, 0};
    const int64_t tiles = (s.Nk + kWinKeyTile - 1) / kWinKeyTile, heads = s.B * s.Hk, G = s.Hq / s.Hk;
    if (heads * tiles > 512) return {1, 0};
    const Window w = window_of(s);
    const bool chunks = far_chunks(s) > 0;
    int64_t each[512], longest = 0, all = 0;
    for (int64_t t = 0; t < tiles; ++t) {
        each[t] = near_stages(w, (int)s.N, (int)s.Nk, chunks, (int)t).each * G;
        longest = std::max(longest, each[t]);
        all += each[t];
    }
    Parts best{1, 0};
    double least = 0;
    for (int64_t k = 1; k <= 16 && k <= longest; ++k) {
        const int64_t stages = (longest + k - 1) / k;   // at most, in a part
        int64_t count = 0;
        for (int64_t t = 0; t < tiles; ++t) count += parts_of((int)k, (int)each[t], (int)stages);
        count *= heads;
        const int64_t rounds = (count + 255) / 256;
        const double mean = (double)(all * heads) / (double)count, last = (double)stages;
        double cost = rounds == 1 ? last + 4 : (double)rounds * (mean + 4) + (last - mean) / 2;
        if (k > 1) cost += 2 + (double)count * kWinKeyTile * (double)s.d * 8 / 12e6;
        if (k == 1 || cost < least) {
            best = {(int)k, (int)stages};
            least = cost;
        }
    }
    return best;
}

size_t part_bytes(const Sizes& s, int parts, int chunks) {
    const int64_t tiles = (s.Nk + kWinKeyTile - 1) / kWinKeyTile, sinks = chunks ? win_sink_tiles(window_of(s), (int)s.Nk) : 0;
    const int64_t sums = sinks * (parts + chunks) + (parts > 1 ? (tiles - sinks) * parts : 0);
    return (size_t)(s.B * s.Hk) * (size_t)sums * 2 * kWinKeyTile * (size_t)s.d * 4;
}

// Sizes of a gradient call.
int check_bwd(const Sizes& s) {
    int st = check_sizes(s, 0);
    if (st) return st;
    if (s.B * s.Hk > 0 && s.Nk >= (kMaxRows + s.B * s.Hk - 1) / (s.B * s.Hk)) return MOA_ERR_UNSUPPORTED;
    const int64_t tiles = (s.Nk + kWinKeyTile - 1) / kWinKeyTile;
    const int64_t more = s.left < 0 ? 0 : 64 + tiles;   // chunks, of one tile or of many with one each
    const int parts = near_parts(s).most;
    if (s.B * s.Hk * (tiles * parts + more) > kMaxBlocks / 2) return MOA_ERR_UNSUPPORTED;   // of 512 threads
    const int64_t joined = parts > 1 ? tiles : far_chunks(s) ? win_sink_tiles(window_of(s), (int)s.Nk) : 0;
    if (s.B * s.Hk * joined > kMaxBlocks / (s.d / 4)) return MOA_ERR_UNSUPPORTED;   // d/4 of them for a tile's two sums
    return MOA_OK;
}

}  // namespace

extern "C" {

int moa_win_attn_num_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk, int64_t d,
                            int64_t left, int64_t right, int64_t sinks, int num_splits) {
    const Sizes s{B, Hq, Hk, Nq, Nk, d, left, right, sinks};
    return check_sizes(s, num_splits) ? 1 : pick_splits(s, num_splits);
}

size_t moa_win_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk,
                                    int64_t d, int64_t left, int64_t right, int64_t sinks,
                                    int num_splits) {
    const Sizes s{B, Hq, Hk, Nq, Nk, d, left, right, sinks};
    return check_sizes(s, num_splits) ? 0 : states_bytes(s, pick_splits(s, num_splits));
}

int moa_win_attn_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int64_t B,
                     int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk, int64_t d,
                     const int64_t* q_strides, const int64_t* k_strides, const int64_t* v_strides,
                     const int64_t* o_strides, int64_t left, int64_t right, int64_t sinks,
                     float scale, int out_dtype, void* workspace, size_t workspace_bytes,
                     int num_splits, void* stream) {
    const Sizes s{B, Hq, Hk, Nq, Nk, d, left, right, sinks};
    if (out_dtype != MOA_F32 && out_dtype != MOA_BF16) return MOA_ERR_INVALID_ARG;
    if (!std::isfinite(scale)) return MOA_ERR_INVALID_ARG;
    int st = check_sizes(s, num_splits);
    if (st) return st;
    const Strides sk = strides_of(k_strides, B, Hk, Nk, d), sv = strides_of(v_strides, B, Hk, Nk, d);
    if ((st = check_tensor(K, sk, B, Hk, Nk, d, 2, false)) || (st = check_tensor(V, sv, B, Hk, Nk, d, 2, false))) return st;
    if (sk.r > kMaxRowStride || sv.r > kMaxRowStride) return MOA_ERR_UNSUPPORTED;
    const Call c{Q, O, LSE, strides_of(q_strides, B, Hq, Nq, d), strides_of(o_strides, B, Hq, Nq, d), scale, out_dtype,
                 workspace, workspace_bytes, pick_splits(s, num_splits), stream};
    if ((st = check_call(c, s))) return st;
    if (!s.any()) return MOA_OK;
    KeySource src{};
    src.k = K; src.v = V;
    put(src.ks, sk); put(src.vs, sv);
    src.len = (int)Nk;
    src.shift = 31;
    src.num_pages = (int)B;
    src.max_pages = 1;
    const Buf keys[] = {{K, extent_bytes(sk, B, Hk, Nk, d, 2)}, {V, extent_bytes(sv, B, Hk, Nk, d, 2)}};
    return run(c, s, src, keys, 2);
}

size_t moa_win_attn_bwd_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t Nq, int64_t Nk,
                                        int64_t d, int64_t left, int64_t right, int64_t sinks) {
    const Sizes s{B, Hq, Hk, Nq, Nk, d, left, right, sinks};
    return check_bwd(s) ? 0 : align256((size_t)(B * Hq * Nq) * 4) + part_bytes(s, near_parts(s).most, far_chunks(s));
}

int moa_win_attn_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                     const float* LSE, void* dQ, void* dK, void* dV, int64_t B, int64_t Hq,
                     int64_t Hk, int64_t Nq, int64_t Nk, int64_t d, const int64_t* q_strides,
                     const int64_t* k_strides, const int64_t* v_strides, const int64_t* o_strides,
                     const int64_t* do_strides, const int64_t* dq_strides,
                     const int64_t* dk_strides, const int64_t* dv_strides, int64_t left,
                     int64_t right, int64_t sinks, float scale, int o_dtype, void* workspace,
                     size_t workspace_bytes, void* stream) {
    const Sizes s{B, Hq, Hk, Nq, Nk, d, left, right, sinks};
    if (o_dtype != MOA_F32 && o_dtype != MOA_BF16) return MOA_ERR_INVALID_ARG;
    if (!std::isfinite(scale)) return MOA_ERR_INVALID_ARG;
    int st = check_bwd(s);
    if (st) return st;
    if (std::fabs(scale) > kMaxScale) return MOA_ERR_UNSUPPORTED;
    struct Tensor {
        const void* p;
        const int64_t* strides;
        int64_t H, N;
        size_t es;
        bool out;
        Strides s;
    } t[] = {{Q, q_strides, Hq, Nq, 2, false, {}}, {K, k_strides, Hk, Nk, 2, false, {}}, {V, v_strides, Hk, Nk, 2, false, {}},
             {O, o_strides, Hq, Nq, o_dtype == MOA_F32 ? size_t(4) : size_t(2), false, {}}, {dO, do_strides, Hq, Nq, 2, false, {}},
             {dQ, dq_strides, Hq, Nq, 2, true, {}}, {dK, dk_strides, Hk, Nk, 2, true, {}}, {dV, dv_strides, Hk, Nk, 2, true, {}}};
    for (Tensor& x : t) {
        x.s = strides_of(x.strides, B, x.H, x.N, d);
        if ((st = check_tensor(x.p, x.s, B, x.H, x.N, d, x.es, x.out))) return st;
        if (x.s.r > kMaxStageStride) return MOA_ERR_UNSUPPORTED;
    }
    if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(LSE) & 3)) return MOA_ERR_INVALID_ARG;
    if (s.any() && !LSE) return MOA_ERR_INVALID_ARG;
    if (B == 0 || (!s.any() && Nk == 0)) return MOA_OK;
    const size_t stats = (size_t)(B * Hq * Nq) * 4;
    const Parts parts = near_parts(s);
    const int chunks = far_chunks(s);
    const size_t need = align256(stats) + part_bytes(s, parts.most, chunks);
    if (need && (!workspace || workspace_bytes < need)) return MOA_ERR_WORKSPACE;
    Buf all[10];
    for (int i = 0; i < 8; ++i) all[i] = {t[i].p, extent_bytes(t[i].s, B, t[i].H, t[i].N, d, t[i].es)};
    all[8] = {LSE, stats};
    all[9] = {workspace, need};
    for (int i : {5, 6, 7, 9})
        for (int k = 0; k < 10; ++k)
            if (k != i && meet(all[i], all[k])) return MOA_ERR_INVALID_ARG;
    WinGrad p{};
    p.w = window_of(s);
    p.q = Q; p.k = K; p.v = V; p.o = O; p.dout = dO; p.lse = LSE;
    p.dq = dQ; p.dk = dK; p.dv = dV;
    put(p.qs, t[0].s); put(p.ks, t[1].s); put(p.vs, t[2].s); put(p.os, t[3].s); put(p.gs, t[4].s);
    put(p.dqs, t[5].s); put(p.dks, t[6].s); put(p.dvs, t[7].s);
    p.B = (int)B; p.hq = (int)Hq; p.hk = (int)Hk; p.nq = (int)Nq; p.nk = (int)Nk; p.d = (int)d;
    p.scale = scale;
    p.o_bf16 = o_dtype == MOA_BF16;
    p.dsum = static_cast<float*>(workspace);
    p.part = need > align256(stats) ? reinterpret_cast<float*>(static_cast<char*>(workspace) + align256(stats)) : nullptr;
    p.parts = parts.most;
    p.part_stages = parts.stages;
    p.chunks = chunks;
    return hip_status(launch_win_bwd(p, static_cast<hipStream_t>(stream)));
}

int moa_paged_attn_num_splits(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page,
                              int64_t max_pages, int64_t max_len, int64_t left, int64_t right,
                              int64_t sinks, int num_splits) {
    const Pools c{page, 0, max_pages, nullptr, nullptr, nullptr};
    if (max_len < 0 || check_pools(c, B, N, false)) return 1;
    const int64_t cap = capacity(c);
    const Sizes s{B, Hq, Hk, N, max_len > 0 && max_len < cap ? max_len : cap, d, left, right, sinks};
    return check_sizes(s, num_splits) ? 1 : pick_splits(s, num_splits);
}

size_t moa_paged_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d,
                                      int64_t page, int64_t max_pages, int64_t max_len,
                                      int64_t left, int64_t right, int64_t sinks, int num_splits) {
    const int splits = moa_paged_attn_num_splits(B, Hq, Hk, N, d, page, max_pages, max_len, left, right, sinks, num_splits);
    return splits <= 1 ? 0 : states_bytes({B, Hq, Hk, N, 0, d, 0, 0, 0}, splits);
}

int moa_paged_attn_fwd(const void* Q, const void* k_pool, const void* v_pool, void* O, float* LSE,
                       const int32_t* seq_lens, const int32_t* new_lens, const int32_t* page_table,
                       int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int64_t page,
                       int64_t num_pages, int64_t max_pages, int64_t max_len,
                       const int64_t* q_strides, const int64_t* k_strides,
                       const int64_t* v_strides, const int64_t* o_strides, int64_t left,
                       int64_t right, int64_t sinks, float scale, int out_dtype, void* workspace,
                       size_t workspace_bytes, int num_splits, void* stream) {
    const Pools pools{page, num_pages, max_pages, seq_lens, new_lens, page_table};
    if (out_dtype != MOA_F32 && out_dtype != MOA_BF16) return MOA_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || max_len < 0) return MOA_ERR_INVALID_ARG;
    int st = check_sizes({B, Hq, Hk, N, 0, d, left, right, sinks}, num_splits);
    if (st) return st;
    const bool any = B > 0 && Hq > 0 && N > 0;
    if ((st = check_pools(pools, B, N, any))) return st;
    const int64_t cap = capacity(pools);
    const Sizes s{B, Hq, Hk, N, max_len > 0 && max_len < cap ? max_len : cap, d, left, right, sinks};
    const Strides sk = strides_of(k_strides, num_pages, Hk, page, d), sv = strides_of(v_strides, num_pages, Hk, page, d);
    if ((st = check_pool(k_pool, sk, pools, Hk, d, false)) || (st = check_pool(v_pool, sv, pools, Hk, d, false))) return st;
    const Call c{Q, O, LSE, strides_of(q_strides, B, Hq, N, d), strides_of(o_strides, B, Hq, N, d), scale, out_dtype,
                 workspace, workspace_bytes, pick_splits(s, num_splits), stream};
    if ((st = check_call(c, s))) return st;
    if (!any) return MOA_OK;
    const Lists lists(pools, B);
    const Buf keys[] = {{k_pool, extent_bytes(sk, num_pages, Hk, page, d, 2)}, {v_pool, extent_bytes(sv, num_pages, Hk, page, d, 2)},
                        lists.b[0], lists.b[1], lists.b[2]};
    return run(c, s, source_of(pools, k_pool, v_pool, sk, sv), keys, 5);
}

// Words: the arguments in their order, but 4 for each tensor's strides (the last
// not read).
int moa_packed_win_attn_fwd(const int64_t* a) {
    using packed::Ptr;
    return moa_win_attn_fwd(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, a[5], a[6], a[7], a[8], a[9], a[10],
                            a + 11, a + 15, a + 19, a + 23, a[27], a[28], a[29], packed::real(a[30]), (int)a[31], Ptr{a[32]},
                            (size_t)a[33], (int)a[34], Ptr{a[35]});
}

int moa_packed_win_attn_bwd(const int64_t* a) {
    using packed::Ptr;
    return moa_win_attn_bwd(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, Ptr{a[6]}, Ptr{a[7]}, Ptr{a[8]},
                            a[9], a[10], a[11], a[12], a[13], a[14], a + 15, a + 19, a + 23, a + 27, a + 31, a + 35, a + 39,
                            a + 43, a[47], a[48], a[49], packed::real(a[50]), (int)a[51], Ptr{a[52]}, (size_t)a[53], Ptr{a[54]});
}

int moa_packed_paged_attn_fwd(const int64_t* a) {
    using packed::Ptr;
    return moa_paged_attn_fwd(Ptr{a[0]}, Ptr{a[1]}, Ptr{a[2]}, Ptr{a[3]}, Ptr{a[4]}, Ptr{a[5]}, Ptr{a[6]}, Ptr{a[7]},
                              a[8], a[9], a[10], a[11], a[12], a[13], a[14], a[15], a[16], a + 17, a + 21, a + 25, a + 29,
                              a[33], a[34], a[35], packed::real(a[36]), (int)a[37], Ptr{a[38]}, (size_t)a[39], (int)a[40],
                              Ptr{a[41]});
}

}  // extern "C"
