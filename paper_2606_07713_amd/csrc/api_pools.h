// Checks of the arguments that say where a paged cache's tokens are (host code only).
#pragma once

#include "api_checks.h"
#include "win.h"

namespace moa {

constexpr int64_t kMost = int64_t(1) << 30;           // positions and sizes: sums of two stay in 32 bits
constexpr int64_t kMaxRowStride = int64_t(1) << 25;   // 16 rows' bytes stay in 32 bits

// The two pools of a paged cache.
struct Pools {
    int64_t page, num_pages, max_pages;
    const int32_t *seq_lens, *new_lens, *table;
};

inline int64_t capacity(const Pools& c) { return c.max_pages * c.page; }

inline int log2_of(int64_t page) {
    int k = 0;
    while ((int64_t(1) << k) < page) ++k;
    return k;
}

inline int check_pools(const Pools& c, int64_t B, int64_t N, bool any) {
    if (c.page < 1 || c.num_pages < 0 || c.max_pages < 0) return MOA_ERR_INVALID_ARG;
    if (c.page < 16 || c.page > (int64_t(1) << 20) || (c.page & (c.page - 1))) return MOA_ERR_UNSUPPORTED;
    if (c.num_pages >= kMost || c.max_pages > kMost / c.page || N > kMost) return MOA_ERR_UNSUPPORTED;
    if (!c.table && any && (c.max_pages != 1 || c.num_pages < B)) return MOA_ERR_INVALID_ARG;
    if (any && !c.seq_lens) return MOA_ERR_INVALID_ARG;
    for (const void* p : {c.seq_lens, c.new_lens, c.table})
        if (reinterpret_cast<uintptr_t>(p) & 3) return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

// A pool of keys or values.
inline int check_pool(const void* p, const Strides& s, const Pools& c, int64_t Hk, int64_t d, bool out) {
    if (s.r > kMaxRowStride) return MOA_ERR_UNSUPPORTED;
    return check_tensor(p, s, c.num_pages, Hk, c.page, d, 2, out);
}

// Tokens, and where they are.
inline KeySource source_of(const Pools& c, const void* k, const void* v, const Strides& sk, const Strides& sv) {
    KeySource s{};
    s.k = k; s.v = v;
    put(s.ks, sk); put(s.vs, sv);
    s.seq_lens = c.seq_lens; s.new_lens = c.new_lens; s.table = c.table;
    s.shift = log2_of(c.page);
    s.num_pages = (int)c.num_pages;
    s.max_pages = (int)c.max_pages;
    return s;
}

// The arrays that tell where tokens are.
struct Lists {
    Buf b[3];
    Lists(const Pools& c, int64_t B)
        : b{{c.seq_lens, (size_t)B * 4}, {c.new_lens, c.new_lens ? (size_t)B * 4 : 0},
            {c.table, c.table ? (size_t)B * (size_t)c.max_pages * 4 : 0}} {}
};

}  // namespace moa
