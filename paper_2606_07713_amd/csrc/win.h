// Internal launch interface of the attention with a window and first visible
// tokens, on whole tensors (moa_window.h) and over the paged cache (moa_paged.h).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace moa {

// Where the keys and values of (sequence, head) are.  Token t is row t mod 2^shift
// of page table[b][t >> shift]; without a table sequence b is page b, and shift is
// 31 on whole tensors, whose batches are the pages.
struct KeySource {
    const void *k, *v;
    long long ks[3], vs[3];    // element strides (page, head, row)
    const int* seq_lens;       // or null: len tokens each
    const int* new_lens;       // or null: all rows of the call
    const int* table;          // [B][max_pages], or null
    int len, shift, num_pages, max_pages;
};

// Limits of what one row sees: keys j < hi with j >= lo or j < sinks, where
// hi = position + right + 1 and lo = position - left.
struct Window {
    int left, right, sinks;    // left, right: kNoLimit where there is none
};
constexpr int kNoLimit = 1 << 30;

// Division by n of numbers below 2^31, as a product: x / n = (2 x m) >> (32 + shift).
struct Div {
    uint32_t n, m;
    int shift, unused;
};
inline Div div_by(long long n) {
    Div d{(uint32_t)n, 0, 0, 0};
    while ((1ll << d.shift) < n) ++d.shift;
    d.m = (uint32_t)(((1ull << (31 + d.shift)) + (uint64_t)n - 1) / (uint64_t)n);
    return d;
}

struct WinAttn {
    KeySource s;
    Window w;
    const void* q;
    void* o;
    float* lse;                // nullable
    long long qs[3], os[3];    // element strides (batch, head, row)
    int B, hq, hk, n, d;
    float scale;
    bool out_bf16;
    // set by the launchers: query heads of a key/value head; workgroups of a row tile
    Div group, per_tile, per_head, heads;
    // Key splits (1 = none) and their partial states: [B][hq][n][splits][d]
    // fp32, then [B][hq][n][splits][2] (reference in log2 units, sum).
    int splits;
    float* ws;
};

inline void set_divisions(WinAttn& p) {
    p.group = div_by(p.hq / p.hk);
    p.per_tile = div_by((long long)p.B * p.hk * p.splits);
    p.per_head = div_by(p.splits);
    p.heads = div_by(p.hk);
}

// The states of up to kMaxSplits splits are added: none of them is larger than the
// largest number over that, or it is done by the definition, whose states are 2^-40 of
// the sums (of weights of at most 1).
constexpr int kMaxSplits = 256;
constexpr float kStateShift = 40.0f;
// From here on an fp32 reference would be off by more than 8 log2 units.
constexpr double kLargestReference = 0x1p28;

// Rows (queries times the query heads of a key/value head) that a workgroup
// takes: 16 or 32 in the kernel of few rows, 128 in that of many.
inline int win_rows_per_block(long long rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 128; }

hipError_t launch_win_attn(const WinAttn& p, hipStream_t stream);
// The two kernels behind it.
hipError_t launch_win_few(const WinAttn& p, hipStream_t stream);
hipError_t launch_win_many(const WinAttn& p, hipStream_t stream);

// Gradients on whole tensors.
struct WinGrad {
    Window w;
    const void *q, *k, *v, *o, *dout;
    const float* lse;
    void *dq, *dk, *dv;
    // element strides (batch, head, row)
    long long qs[3], ks[3], vs[3], os[3], gs[3], dqs[3], dks[3], dvs[3];
    int B, hq, hk, nq, nk, d;
    float scale;
    bool o_bf16;
    Div group, per_item, heads;   // set by the launcher, as in WinAttn
    float* dsum;               // [B][hq][nq]: <dO, O> of every row
    float* part;               // partial sums of dK and dV
    int parts;                 // of a key tile's queries at most (1: whole)
    int part_stages;           // stages that a part has at most
    int near_items;            // set by the launcher: parts of all tiles
    int chunks;                // of the queries behind the first keys' windows (0: none)
};

// Keys of a workgroup of the dK, dV kernel, and queries of one of its stages.
constexpr int kWinKeyTile = 128, kWinStage = 64;

// Key tiles that hold first keys which stay visible behind the window.
inline int win_sink_tiles(const Window& w, int nk) {
    const int sinks = w.sinks < nk ? w.sinks : nk;
    return w.left == kNoLimit ? 0 : (sinks + kWinKeyTile - 1) / kWinKeyTile;
}

// The stages of one head whose queries see a key of tile kt, but for those that see
// only first keys of it and have chunks of their own; near_hi: the last query of those
// whose windows reach the tile.
struct Near {
    int first, each, near_hi;
};
constexpr Near near_stages(const Window& w, int nq, int nk, bool chunks, int kt) {
    const long long off = (long long)nk - nq, last = nq - 1;
    const int k0 = kt * kWinKeyTile, k1 = (k0 + kWinKeyTile < nk ? k0 + kWinKeyTile : nk) - 1;
    const long long from = w.right == kNoLimit ? 0 : k0 - off - w.right, to = w.left == kNoLimit ? last : k1 - off + w.left;
    const int lo = (int)(from < 0 ? 0 : from > nq ? nq : from);
    const int near_hi = (int)(to < -1 ? -1 : to > last ? last : to);
    const int hi = k0 < w.sinks && !chunks ? (int)last : near_hi, first = lo / kWinStage;
    return {first, hi < lo ? 0 : hi / kWinStage + 1 - first, near_hi};
}
// Into how many parts these stages of all heads are cut: long lists into more, so that
// all workgroups take about as long.
constexpr int parts_of(int most, int stages, int part_stages) {
    if (most == 1) return 1;
    const int n = (stages + part_stages - 1) / part_stages;
    return n < 1 ? 1 : n > most ? most : n;
}

hipError_t launch_win_bwd(const WinGrad& p, hipStream_t stream);

}  // namespace moa
