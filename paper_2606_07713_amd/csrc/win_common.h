// Device-side pieces of the attention with a window: which keys a row sees, the
// walk over the key tiles that any of some rows see, and a row's result by its
// definition.
#pragma once

#include "device_common.h"
#include "win.h"

namespace moa {
namespace win {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Max and sum over the four lanes with the same lane % 16.
__device__ __forceinline__ float column_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const bf16x2 t = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, t);
}

// a and b as sums of TERMS bf16 numbers each, every one the nearest to what the ones
// before it leave: at most 2^-8 or 2^-17 of a weight is lost with one or two, and nothing of
// an fp32 number with three.
template <int TERMS>
__device__ __forceinline__ void bf16_terms(float a, float b, uint32_t (&w)[TERMS]) {
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        w[t] = pack2(a, b);
        if (t + 1 < TERMS) {
            a -= bf16lo_to_f32(w[t]);
            b -= bf16hi_to_f32(w[t]);
        }
    }
}

__device__ __forceinline__ int over(const Div& d, int x) { return (int)(__umulhi((uint32_t)x << 1, d.m) >> d.shift); }

// New tokens of sequence b, its length, and the tokens that the pages have room
// for at most.
__device__ __forceinline__ int new_tokens(const int* new_lens, int b, int n) {
    return new_lens ? min(max(new_lens[b], 0), n) : n;
}
__device__ __forceinline__ int length(const KeySource& s, int b) { return s.seq_lens ? s.seq_lens[b] : s.len; }
__device__ __forceinline__ int capacity(const KeySource& s) {
    return s.seq_lens ? (s.num_pages ? s.max_pages << s.shift : 0) : s.len;
}

// The page of key `key` of sequence b, or -1.
__device__ __forceinline__ int page_of(const KeySource& s, int b, int key) {
    if (!s.table) return b;
    const int index = key >> s.shift;
    if (index >= s.max_pages) return -1;
    const int id = s.table[(size_t)b * s.max_pages + index];
    return id >= 0 && id < s.num_pages ? id : -1;
}

// Element offset of key `key` in its page of a pool with strides st.
__device__ __forceinline__ long long key_offset(const long long (&st)[3], int shift, int page, int head, int key) {
    const int row = shift < 31 ? key & ((1 << shift) - 1) : key;
    return page * st[0] + head * st[1] + row * st[2];
}

// Keys that a row sees: j < hi with j >= lo or j < sinks (0 <= lo).
struct Seen {
    int lo, hi;
};

// Of a row at position pos of a sequence with `end` keys.
__device__ __forceinline__ Seen seen_from(const Window& w, long long pos, int end) {
    Seen s;
    s.hi = w.right == kNoLimit ? end : (int)max(0ll, min((long long)end, pos + w.right + 1));
    s.lo = w.left == kNoLimit ? 0 : (int)min((long long)end, max(0ll, pos - w.left));
    return s;
}
__device__ __forceinline__ bool sees(const Seen& s, int sinks, int key) {
    return key < s.hi && (key >= s.lo || key < sinks);
}
__device__ __forceinline__ bool sees_any(const Seen& s, int sinks) { return s.hi > 0 && (s.lo < s.hi || sinks > 0); }

// Bits 0 .. n - 1.
__device__ __forceinline__ uint32_t ones(int n) { return (uint32_t)(0xffffffffull >> (32 - min(max(n, 0), 32))); }

// Bit k: the row sees key k0 + k.
__device__ __forceinline__ uint32_t seen_bits(const Seen& s, int sinks, int k0) {
    return ones(s.hi - k0) & (~ones(s.lo - k0) | ones(sinks - k0));
}

// Of rows the first of which sees wl and the last wh (uniform): whether all of them see
// all of the 32 keys from k0 on, and whether any of them sees one.
__device__ __forceinline__ bool all_see(const Seen& wl, const Seen& wh, int sinks, int k0) {
    return k0 + 32 <= wl.hi && (k0 >= wh.lo || k0 + 32 <= sinks);
}
__device__ __forceinline__ bool any_sees(const Seen& wl, const Seen& wh, int sinks, int k0) {
    return k0 < wh.hi && (k0 + 32 > wl.lo || k0 < sinks);
}

// x, or -inf where bit n is not set: two instructions.  (Written as comparisons these
// became a branch per element.)
__device__ __forceinline__ float keep_bit(float x, uint32_t bits, int n) {
    const uint32_t all = (uint32_t)((int)(bits << (31 - n)) >> 31);
    return __uint_as_float((__float_as_uint(x) & all) | (0xff800000u & ~all));
}

// The scores in a 32x32 accumulator; element i is bit 8 (i / 4) + 4 half + i % 4.
__device__ __forceinline__ void keep(f32x16& x, uint32_t bits, int half) {
    bits >>= 4 * half;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = keep_bit(x[i], bits, 8 * (i >> 2) + (i & 3));
}

// The launch's arguments once more, from where they came: what is used behind a loop
// then need not be kept in scalar registers during it.  T: the kernel's first argument.
template <typename T>
__device__ __forceinline__ T arguments_again() {
    static_assert(sizeof(T) % 8 == 0, "read as words");
    typedef const __attribute__((address_space(4))) unsigned long long* words;
    words w = (words)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(w));
    struct { unsigned long long x[sizeof(T) / 8]; } raw;
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 8; ++i) raw.x[i] = w[i];
    return __builtin_bit_cast(T, raw);
}

// The tiles of T keys that any of the rows from `first` to `last` (positions in
// order) see: those of the first keys, then those of the windows.
template <int T>
struct Tiles {
    int head, skip, count;
    __device__ __forceinline__ Tiles(const Seen& first, const Seen& last, int sinks) {
        const int end = (last.hi + T - 1) / T, from = first.lo / T;
        head = (min(sinks, last.hi) + T - 1) / T;
        const int begin = max(from, head);
        skip = begin - head;
        count = head + max(0, end - begin);
    }
    __device__ __forceinline__ int at(int v) const { return v < head ? v : v + skip; }
};

// <a, b> of two rows of D elements as T sums it, in one order; a is the same row in all
// lanes.  (The loads of U pieces are in flight together.)
template <int D, int U, typename T>
__device__ __forceinline__ T dot_as(const u16* a, const u16* b) {
#pragma clang fp contract(off)
    T x = 0;
    const uint64_t at = reinterpret_cast<uint64_t>(a);
    const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
    const u32x4* q = reinterpret_cast<const u32x4*>(uniform);
#pragma unroll 1
    for (int e = 0; e < D; e += 8 * U) {
        u32x4 u[U], v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            u[i] = q[e / 8 + i];
            v[i] = *reinterpret_cast<const u32x4*>(b + e + 8 * i);
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x = __builtin_elementwise_fma((T)bf16lo_to_f32(u[i][j]), (T)bf16lo_to_f32(v[i][j]), x);
                x = __builtin_elementwise_fma((T)bf16hi_to_f32(u[i][j]), (T)bf16hi_to_f32(v[i][j]), x);
            }
    }
    return x;
}
// In fp32, or in fp64 what that does not hold.
template <int D, int U = 8>
__device__ __forceinline__ double dot(const u16* a, const u16* b) {
    const float x = dot_as<D, U, float>(a, b);
    return __builtin_isfinite(x) ? (double)x : dot_as<D, U, double>(a, b);
}

// Adds the lanes' w times their rows to o, this lane's elements D/64 lane ..; row(j):
// lane j's row, only taken where its bit of `which` is set.  U at a time are in flight.
template <int D, int U = 8, typename F>
__device__ __forceinline__ void add_rows(float (&o)[D / 64], uint64_t which, float w, F row) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    while (which) {
        uint32_t bits[U];
        float f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool one = which != 0;
            const int j = one ? __builtin_ctzll(which) : 0;
            f[u] = one ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j)) : 0.0f;
            bits[u] = 0;
            if (one) {
                const u16* at = row(j);
                if constexpr (E == 2) bits[u] = *reinterpret_cast<const uint32_t*>(at + 2 * lane);
                else bits[u] = at[lane];
            }
            which &= which - 1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            o[0] = __builtin_fmaf(f[u], bf16lo_to_f32(bits[u]), o[0]);
            if constexpr (E == 2) o[1] = __builtin_fmaf(f[u], bf16hi_to_f32(bits[u]), o[1]);
        }
    }
}

// One row by its definition, by one wave, over the keys of tiles begin .. end - 1:
// scores of any size, weights of at most 1, nothing of a key that the row does not
// see.  For the rows whose sums in the tile kernels did not come out finite: a
// value that is infinite or NaN (which a product with a weight of 0 spreads to
// rows that do not see it), or a score or a sum beyond fp32.  o: this lane's
// elements D/64 lane ..; without `partial` divided by the sum, with it the state
// of a split: its weights count against the fp32 number that its reference is.  Where
// that would leave fp32 too, or there is none, the reference is NaN, and the join does
// the whole row (RowsAgain).
template <int D, int T, int U = 8>
__device__ void row_by_definition(const WinAttn& p, int b, int h, const u16* q, const Seen& seen, const Tiles<T>& tiles,
                                  int begin, int end, bool partial, float (&o)[D / 64], float& ref, float& sum) {
    // Both walks have to see the same scores, bit for bit: of one of 2^100 a single
    // rounding is 2^47.
#pragma clang fp contract(off)
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    // (the factor of the tile kernels: states of both kinds meet)
    const double c = p.scale * kLog2e;
    const auto score = [&](int key, int page) {
        return dot<D, U>(q, static_cast<const u16*>(p.s.k) + key_offset(p.s.ks, p.s.shift, page, h, key)) * c;
    };
    const auto walk = [&](auto f) {
#pragma unroll 1
        for (int v = begin; v < end; ++v) {
            const int k0 = tiles.at(v) * T, key = k0 + lane;
            const int page = lane < T && sees(seen, p.w.sinks, key) ? page_of(p.s, b, key) : -1;
            if (wave_any(page >= 0)) f(k0, key, page);
        }
    };
    double M = -__builtin_inf(), L = 0.0;
    bool any = false;
    walk([&](int, int key, int page) {
#pragma clang fp contract(off)
        const double x = page >= 0 ? score(key, page) : -__builtin_inf();
        double m = x;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) m = fmax(m, __shfl_xor(m, s));
        any = true;
        const double top = fmax(M, m);
        // A score that is NaN is not in M, but makes L one; one of -inf counts nothing,
        // also where there is no other yet.
        double w = x == -__builtin_inf() ? 0.0 : (double)exp2_hw((float)(x - top));
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) w += __shfl_xor(w, s);
        L = (M == -__builtin_inf() ? L : L * (double)exp2_hw((float)(M - top))) + w;
        M = top;
    });
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    ref = kNegInf;
    sum = 0.0f;
    if (!any) return;
    double inv = 1.0 / L;
    ref = (float)M;
    if (partial) {
        ref = (float)(M + (double)kStateShift);
        if (!(__builtin_fabs(M) < kLargestReference)) {
            ref = sum = __builtin_nanf("");
            return;
        }
        const double rest = M - (double)ref, whole = __builtin_rint(rest);
        inv = __builtin_ldexp((double)exp2_hw((float)(rest - whole)), (int)whole);
    }
    sum = (float)(partial ? L * inv : L);
    walk([&](int k0, int key, int page) {
#pragma clang fp contract(off)
        const float w = page >= 0 ? (float)((double)exp2_hw((float)(score(key, page) - M)) * inv) : 0.0f;
        add_rows<D, U>(o, __ballot(page >= 0), w, [&](int j) {
            return static_cast<const u16*>(p.s.v) + key_offset(p.s.vs, p.s.shift, __builtin_amdgcn_readlane(page, j), h, k0 + j);
        });
    });
}

// Stores such a row: O and LSE.
template <int D>
__device__ __forceinline__ void store_output(const WinAttn& p, int b, int hh, int qi, const float (&o)[D / 64], float ref, float sum) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const long long to = b * p.os[0] + hh * p.os[1] + qi * p.os[2] + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (p.out_bf16) static_cast<__bf16*>(p.o)[to + e] = (__bf16)o[e];
        else static_cast<float*>(p.o)[to + e] = o[e];
    }
    // (a sum of 0 without a reference: -inf; NaN: NaN)
    if (p.lse && lane == 0) p.lse[((size_t)b * p.hq + hh) * p.n + qi] = (ref + __log2f(sum)) * kLn2;
}

// The same, or the state of split sp.
template <int D>
__device__ __forceinline__ void store_row(const WinAttn& p, int b, int hh, int qi, int sp, const float (&o)[D / 64],
                                          float ref, float sum) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    if (p.splits == 1) return store_output<D>(p, b, hh, qi, o, ref, sum);
    const size_t at = ((size_t)b * p.hq + hh) * p.n + qi;
    float* ml = p.ws + (size_t)p.B * p.hq * p.n * p.splits * D + (at * p.splits + sp) * 2;
#pragma unroll
    for (int e = 0; e < E; ++e) p.ws[(at * p.splits + sp) * D + E * lane + e] = o[e];
    if (lane == 0) {
        ml[0] = ref;
        ml[1] = sum;
    }
}

// The join's rows with a state that asks for it: all splits at once by the definition.
struct RowsAgain {
    static constexpr bool any = true;
    WinAttn p;
    template <int D>
    __device__ __forceinline__ void row(int b, int hh, int qi) const {
        const KeySource& src = p.s;
        const int len = length(src, b);
        const Seen seen = seen_from(p.w, (long long)len - new_tokens(src.new_lens, b, p.n) + qi, max(0, min(len, capacity(src))));
        const Tiles<64> tiles(seen, seen, p.w.sinks);
        float f[D / 64], M, L;
        // (two loads in flight: the join of all others keeps its registers)
        row_by_definition<D, 64, 2>(p, b, over(p.group, hh), static_cast<const u16*>(p.q) + b * p.qs[0] + hh * p.qs[1] + qi * p.qs[2],
                                 seen, tiles, 0, tiles.count, false, f, M, L);
        store_output<D>(p, b, hh, qi, f, M, L);
    }
};

}  // namespace win
}  // namespace moa
