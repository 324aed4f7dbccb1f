// Attention over the four-bit cache (moa_kv4.h).
//
// A workgroup takes RT tiles of 16 rows of one key/value head -- a row is a
// query and one of the G = Hq/Hk heads that share the stored head, query by
// query -- over a range of keys; its four waves take the range's 64-key tiles
// in turn, each with a softmax state of its own, and join them at the end.
//
// The codes go from memory to registers in the order in which the matrix
// instruction takes them, without LDS: for S^T = K Q^T a lane holds 32 (16 at
// d = 64) successive elements of a key, its part of a wave-wide read of whole
// rows; for O^T += V^T P^T it holds, of every four keys, the elements d/16 c ..
// of its column c.  One v_cvt_scalef32_pk_bf16_fp4 makes two bf16 of a byte and
// their power of two, exactly.  The S^T accumulators leave a lane with the four
// keys 16 t + 4 g .. of row n = lane % 16 -- and since the order of the keys
// in a product is free, two such accumulators, packed to bf16, are the B
// operand of the second product as they are.  That product is taken twice, with
// the weights' nearest bf16 numbers and with those of what these leave: one
// bf16 number per weight (2^-8) would be off by as much as a bf16 output is by
// itself, and by far more than an fp32 output.
//
// Softmax: a running reference per row, the maximum of the first tile that the
// row sees; later tiles are weighed against it without looking for their own
// maximum, and only a sum beyond 2^20 (scores 16 and more log2 units above the
// reference; fp32 and bf16 hold such weights as well as small ones) raises it,
// for the whole wave at once, and so does a tile with values of 2^65 and more.
// fp32 sums of the unrounded weights per lane, joined over the lanes once at the
// end.
//
// What bounds it: with few rows the memory (64 sequences of 8192 keys, 8 stored
// heads of d = 128 for 32: 571 MB in 91 us, 6.2 TB/s; reading alone reaches 6.9),
// with many the sum of vector and matrix instructions, which hardly overlap as
// they are ordered here (a tile of 16 rows takes a SIMD 2600 cycles from the
// caches, one of 32 rows 3800; 2100 and 2900 with one bf16 number per weight): 32
// heads on 8, 8192 causal queries, d = 128, 748 us, 0.74 PFLOP/s.  Short calls are
// chains of latencies.
#include <cfloat>
#include <limits>

#include "kv4_common.h"
#include "prefill_bf16_common.h"
#include "split_join.h"

namespace moa {
namespace {

using namespace kv4;

constexpr int WAVES = 4;
constexpr float kLargeSum = 1048576.0f;   // a lane's sum of one tile's weights that raises the reference

// Max over the four lanes with the same lane % 16.
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

// a and b as two bf16 numbers each: the nearest, and the nearest to the rest.
// Together they hold 17 bits, 2^-18 of a weight at most is lost.
__device__ __forceinline__ void two_terms(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack2(a, b);
    lo = pack2(a - bf16lo_to_f32(hi), b - bf16hi_to_f32(hi));
}

template <int B>
__device__ __forceinline__ uint32_t values2(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

// Eight successive elements of a key.
__device__ __forceinline__ bf16x8 key8(uint32_t w, float scale) {
    const uint4 r = make_uint4(values2<0>(w, scale), values2<1>(w, scale), values2<2>(w, scale), values2<3>(w, scale));
    return __builtin_bit_cast(bf16x8, r);
}

// The power of two of byte I of w.  One instruction for each byte: left to
// itself the compiler takes a shift and a mask for bytes 0 to 2.
template <int I>
__device__ __forceinline__ float scale_byte(uint32_t w) {
    float r;
    if constexpr (I == 0)
        asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(23), "v"(w));
    else if constexpr (I == 1)
        asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(23), "v"(w));
    else if constexpr (I == 2)
        asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(23), "v"(w));
    else
        r = scale_of(w >> 24);
    return r;
}

// One 64-key tile's codes and scales of one lane.  ONCE: no other workgroup
// reads them, so they need not stay in the caches.
template <int D, bool ONCE>
struct Tile {
    uint32_t k[4][D / 32], v[4][D / 32];   // [16-key group][dwords]
    uint32_t ks, vs[4];

    __device__ __forceinline__ void load(const unsigned char* head, int page, int in, int lane) {
        const int r = lane & 15, g = lane >> 4;
        const unsigned char* kc = head + in * 32 * D;
        const unsigned char* vc = head + val_codes(page, D) + in * 32 * D;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            read(kc + (16 * t + r) * (D / 2) + g * (D / 8), k[t]);
            read(vc + (4 * t + g) * 2 * D + r * (D / 8), v[t]);
        }
        // key scales: of this lane's 32 (16) elements; value scales: of its column
        constexpr int LANES_PER_BLOCK = D == 128 ? 1 : 2, COLS_PER_BLOCK = D == 128 ? 4 : 8;
        ks = *reinterpret_cast<const uint32_t*>(head + key_scales(page, D) + in * 2 * D + (g / LANES_PER_BLOCK) * 64 + r * 4);
        const uint4 s = *reinterpret_cast<const uint4*>(head + val_scales(page, D) + in * 2 * D + (r / COLS_PER_BLOCK) * 64 + g * 16);
        vs[0] = s.x; vs[1] = s.y; vs[2] = s.z; vs[3] = s.w;
    }
    static __device__ __forceinline__ void read(const unsigned char* p, uint32_t (&w)[D / 32]) {
        typedef uint32_t vec __attribute__((ext_vector_type(D / 32)));
        const vec* at = reinterpret_cast<const vec*>(p);
        vec x;
        if constexpr (ONCE) x = __builtin_nontemporal_load(at);
        else x = *at;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) w[i] = x[i];
    }
    // S^T of 16-key group t: 4 keys 16 t + 4 g .. of row lane % 16.
    template <int T>
    __device__ __forceinline__ void keys(bf16x8 (&a)[D / 32]) const {
        const float s = scale_byte<T>(ks);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) a[i] = key8(k[T][i], s);
    }
    // V^T operands of the 32 keys of groups 2 U and 2 U + 1 for elements 4 F .. of
    // the column's D/16.
    template <int U, int F>
    __device__ __forceinline__ void values(bf16x8 (&a)[4]) const {
        uint32_t r[4][4];
        quad<0>(v[2 * U][2 * F], v[2 * U][2 * F + 1], vs[2 * U], r);
        quad<1>(v[2 * U + 1][2 * F], v[2 * U + 1][2 * F + 1], vs[2 * U + 1], r);
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = __builtin_bit_cast(bf16x8, make_uint4(r[e][0], r[e][1], r[e][2], r[e][3]));
    }
    // w01: keys 0, 1 of four elements, w23: keys 2, 3
    template <int H>
    static __device__ __forceinline__ void quad(uint32_t w01, uint32_t w23, uint32_t s, uint32_t (&r)[4][4]) {
        pair(w01, scale_byte<0>(s), scale_byte<1>(s), r[0][2 * H], r[1][2 * H], r[2][2 * H], r[3][2 * H]);
        pair(w23, scale_byte<2>(s), scale_byte<3>(s), r[0][2 * H + 1], r[1][2 * H + 1], r[2][2 * H + 1], r[3][2 * H + 1]);
    }
    static __device__ __forceinline__ void pair(uint32_t w, float sa, float sb, uint32_t& e0, uint32_t& e1, uint32_t& e2, uint32_t& e3) {
        const uint32_t a01 = values2<0>(w, sa), a23 = values2<1>(w, sa), b01 = values2<2>(w, sb), b23 = values2<3>(w, sb);
        e0 = __builtin_amdgcn_perm(b01, a01, 0x05040100);
        e1 = __builtin_amdgcn_perm(b01, a01, 0x07060302);
        e2 = __builtin_amdgcn_perm(b23, a23, 0x05040100);
        e3 = __builtin_amdgcn_perm(b23, a23, 0x07060302);
    }
    // Whether a value's scale is 2^65 or more (a byte of 192 and more).
    __device__ __forceinline__ bool large_values() const {
        uint32_t x = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) x |= vs[t] & (vs[t] << 1);
        return (x & 0x80808080u) != 0;
    }
    // Value scales that no written block has (255: the block held a NaN; unset
    // memory) become 2^-127, a finite factor for keys that a row does not see.
    // Returns those bytes, one bit per key of the lane: bit 4 t + j.
    __device__ __forceinline__ uint32_t tame() {
        uint32_t bad = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (((vs[t] >> (8 * j)) & 255u) > 252u) {
                    bad |= 1u << (4 * t + j);
                    vs[t] &= ~(255u << (8 * j));
                }
        return bad;
    }
};

template <int D, int RT, bool ONCE>
__global__ __launch_bounds__(WAVES * 64, 2) void kv4_attn_kernel(Kv4Attn p, float c, bool flip, int row_tiles) {
    constexpr int E = D / 16, ROWS = 16 * RT, LD = D + 4;
    __shared__ __attribute__((aligned(16))) float part[WAVES][ROWS][LD];
    __shared__ float part_m[WAVES][ROWS], part_l[WAVES][ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const Kv4Cache& kc = p.c;
    const int G = p.hq / kc.hk;
    // Row tiles last, the last ones first: those of one head and split, which read
    // the same keys, mostly go to one XCD (successive workgroups go to the eight
    // in turn), and under the causal mask the longest begin first (16 heads of 2
    // sequences of 4096, d = 128: 266 us with row tiles next to each other, 210
    // so, 233 first to last).
    int blk = blockIdx.x;
    const int groups = kc.B * kc.hk * p.splits, rt = row_tiles - 1 - blk / groups;
    blk %= groups;
    const int sp = blk % p.splits; blk /= p.splits;
    const int h = blk % kc.hk, b = blk / kc.hk;

    const int count = new_tokens(kc, b), rows = count * G, row0 = rt * ROWS;
    if (row0 >= rows) return;
    const long long len = kc.seq_lens[b], cap = kc.num_pages ? (long long)kc.max_pages * kc.page : 0;
    const long long first = len - count;   // position of query 0
    // A row sees keys 0 .. sees(row) - 1; rows behind the last one are computed
    // as it is, with queries of zero, and not stored.
    const auto sees = [&](int row) -> int {
        const long long s = p.causal ? first + row / G + 1 : len;
        return (int)max(0ll, min(s, cap));
    };
    int seen[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) seen[i] = sees(min(row0 + 16 * i + n, rows - 1));
    const int most = __builtin_amdgcn_readfirstlane(sees(min(row0 + ROWS, rows) - 1));
    const int whole = __builtin_amdgcn_readfirstlane(sees(row0)) >> 6;   // tiles below it need no mask
    const int tiles = (most + 63) >> 6, per = (tiles + p.splits - 1) / p.splits;
    const int begin = sp * per, end = min(tiles, begin + per);

    bf16x8 q[RT][D / 32];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int row = row0 + 16 * i + n;
        const bool in = row < rows;
        const int qi = in ? row / G : 0, hh = h * G + (in ? row - qi * G : 0);
        const u16* src = static_cast<const u16*>(p.q) + b * p.qs[0] + hh * p.qs[1] + qi * p.qs[2] + g * (D / 4);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            uint4 w = in ? *reinterpret_cast<const uint4*>(src + 8 * k) : make_uint4(0, 0, 0, 0);
            if (flip) { w.x ^= 0x80008000u; w.y ^= 0x80008000u; w.z ^= 0x80008000u; w.w ^= 0x80008000u; }
            q[i][k] = __builtin_bit_cast(bf16x8, w);
        }
    }

    f32x4 o[RT][E];
    float ref[RT], l[RT];   // reference in log2 units, -inf before the first visible key
    bool ready = false;     // every row has one
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        ref[i] = kNegInf;
        l[i] = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[i][e] = f32x4{0, 0, 0, 0};
    }
    const int tpp = kc.page >> 6;   // tiles per page
    int at = begin + wave, index = at / tpp, in = at - index * tpp;
    // Loads the tile at `at` and moves on; false: there is none (no more tiles,
    // or its page is not in the pool).  Something is loaded in any case, so that
    // the number of loads in flight is known where a tile's own are waited for:
    // with loads on one side of a branch every wait was for all of them.
    const auto fetch = [&](Tile<D, ONCE>& tile) -> bool {
        const unsigned char* head = nullptr;
        int tile_in = 0;
        if (at < end) {
            while (in >= tpp) { in -= tpp; ++index; }
            head = page_of(kc, b, h, index);
            tile_in = head ? in : 0;
        }
        tile.load(head ? head : kc.base + (size_t)h * kc.page_bytes, kc.page, tile_in, lane);
        at += WAVES;
        in += WAVES;
        return head != nullptr;
    };
    const auto attend = [&](Tile<D, ONCE>& tile, int t) {
        f32x4 s[RT][4];
        const auto score = [&](auto T) {
            bf16x8 a[D / 32];
            tile.template keys<decltype(T)::value>(a);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < D / 32; ++k) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[k], q[i][k], x, 0, 0, 0);
                s[i][decltype(T)::value] = x;
            }
        };
        score(std::integral_constant<int, 0>{});
        score(std::integral_constant<int, 1>{});
        score(std::integral_constant<int, 2>{});
        score(std::integral_constant<int, 3>{});

        uint32_t bad = 0;
        const bool masked = t >= whole;
        if (masked) {
            bad = tile.tame();
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (64 * t + 16 * u + 4 * g + j >= seen[i]) s[i][u][j] = kNegInf;
        }

        // The weights 2^(s c - ref), each as two bf16 numbers, and their sums.
        bf16x8 pt[RT][2], rest[RT][2];
        float sum[RT];
        const auto weights = [&]() {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const float shift = ref[i] == kNegInf ? 0.0f : -ref[i];
                float w[4][4], x = 0.0f;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        w[u][j] = exp2_hw(__builtin_fmaf(s[i][u][j], c, shift));
                        x += w[u][j];
                    }
                sum[i] = x;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) two_terms(w[2 * u + k / 2][2 * (k % 2)], w[2 * u + k / 2][2 * (k % 2) + 1], hi[k], lo[k]);
                    pt[i][u] = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
                    rest[i][u] = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
                }
            }
        };
        // Against the present references, without a maximum, unless the tile is
        // masked, a row has seen nothing yet, a sum comes out too large or the
        // values are so large themselves (2^22 of weight a tile, 2^25 tiles: below
        // 2^65 the products stay in fp32) that weights above 1 are not for them.
        bool raise = masked || !ready;
        if (!raise) {
            weights();
            bool large = tile.large_values();
#pragma unroll
            for (int i = 0; i < RT; ++i) large |= sum[i] > kLargeSum;
            raise = wave_any(large);
        }
        if (raise) {
            ready = true;
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float x = kNegInf;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x = fmaxf(x, s[i][u][j]);
                // Finite for a row that sees a key of the tile, whatever its scores: -inf
                // is the mark of rows that have seen none.  A score beyond fp32 leaves an
                // infinite weight or none at all, and the row NaN.
                x = fminf(column_max(x) * c, FLT_MAX);
                if (64 * t < seen[i]) x = fmaxf(x, -FLT_MAX);
                x = fmaxf(ref[i], x);
                const float a = ref[i] == kNegInf ? 0.0f : exp2_hw(ref[i] - x);
                ref[i] = x;
                l[i] *= a;
#pragma unroll
                for (int e = 0; e < E; ++e) o[i][e] *= a;
                ready &= !wave_any(x == kNegInf);
            }
            weights();
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) l[i] += sum[i];

        // The products of four elements follow their unpacking at once, so that the next
        // four are unpacked while the matrix unit works.
        const auto product = [&](auto U, auto F) {
            constexpr int u = decltype(U)::value, f = decltype(F)::value;
            if constexpr (f < D / 64) {
                bf16x8 a[4];
                tile.template values<u, f>(a);
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[i][4 * f + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[e], pt[i][u], o[i][4 * f + e], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[i][4 * f + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[e], rest[i][u], o[i][4 * f + e], 0, 0, 0);
            }
        };
        constexpr std::integral_constant<int, 0> zero;
        constexpr std::integral_constant<int, 1> one;
        product(zero, zero);
        product(zero, one);
        product(one, zero);
        product(one, one);

        // A masked tile with blocks that hold a NaN: their elements become NaN
        // in the rows that see the key, counted by a product of ones.
        if (masked && wave_any(bad != 0)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t va[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int at = 4 * (2 * u + k / 2) + 2 * (k % 2);
                    va[k] = ((bad >> at) & 1u ? 0x3f80u : 0u) | ((bad >> (at + 1)) & 1u ? 0x3f800000u : 0u);
                }
                const bf16x8 a = __builtin_bit_cast(bf16x8, make_uint4(va[0], va[1], va[2], va[3]));
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    uint32_t vb[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int key = 64 * t + 16 * (2 * u + k / 2) + 4 * g + 2 * (k % 2);
                        vb[k] = (key < seen[i] ? 0x3f80u : 0u) | (key + 1 < seen[i] ? 0x3f800000u : 0u);
                    }
                    f32x4 hit = {0, 0, 0, 0};
                    hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, make_uint4(vb[0], vb[1], vb[2], vb[3])), hit, 0, 0, 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (hit[j] > 0.0f)
#pragma unroll
                            for (int e = 0; e < E; ++e) o[i][e][j] = __builtin_nanf("");
                }
            }
        }
    };
    // Two tiles in registers: the next one's loads are in flight while one is
    // worked on.
    if (at < end) {
        Tile<D, ONCE> tile0, tile1;
        bool have0 = fetch(tile0);
        for (int t = begin + wave; t < end; t += 2 * WAVES) {
            const bool have1 = fetch(tile1);
            if (have0) attend(tile0, t);
            have0 = fetch(tile0);
            if (have1) attend(tile1, t + WAVES);
        }
    }

    // Join the waves' states: a common reference per row, then sums.
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        l[i] = column_sum(l[i]);
        if (g == 0) part_m[wave][16 * i + n] = ref[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int row = 16 * i + n;
        float M = kNegInf;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, part_m[w][row]);
        const float a = ref[i] == kNegInf ? 0.0f : exp2_hw(ref[i] - M);
        if (g == 0) part_l[wave][row] = l[i] * a;
        // column 4 g + j of the wave's O^T: elements E (4 g + j) + e of the row
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<float4*>(&part[wave][row][E * (4 * g + j) + e]) =
                    make_float4(o[i][e][j] * a, o[i][e + 1][j] * a, o[i][e + 2][j] * a, o[i][e + 3][j] * a);
    }
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS * (D / 8); x += WAVES * 64) {
        const int r = x / (D / 8), d8 = (x % (D / 8)) * 8, row = row0 + r;
        if (row >= rows) break;
        float f[8], L = 0.0f, M = kNegInf;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            M = fmaxf(M, part_m[w][r]);
            L += part_l[w][r];
            const float4 u = *reinterpret_cast<const float4*>(&part[w][r][d8]), v = *reinterpret_cast<const float4*>(&part[w][r][d8 + 4]);
            f[0] += u.x; f[1] += u.y; f[2] += u.z; f[3] += u.w;
            f[4] += v.x; f[5] += v.y; f[6] += v.z; f[7] += v.w;
        }
        const int qi = row / G, hh = h * G + row - qi * G;
        const size_t at = ((size_t)b * p.hq + hh) * kc.n + qi;
        if (p.splits > 1) {
            float* acc = p.ws + (at * p.splits + sp) * D + d8;
            reinterpret_cast<float4*>(acc)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(acc)[1] = make_float4(f[4], f[5], f[6], f[7]);
            if (d8 == 0) {
                float* ml = p.ws + (size_t)kc.B * p.hq * kc.n * p.splits * D + (at * p.splits + sp) * 2;
                ml[0] = M;
                ml[1] = L;
            }
            continue;
        }
        const bool none = M == kNegInf;   // no visible key
        const float inv = none ? 0.0f : 1.0f / L;
        const long long to = b * p.os[0] + hh * p.os[1] + qi * p.os[2] + d8;
        if (p.out_bf16) {
            *reinterpret_cast<uint4*>(static_cast<u16*>(p.o) + to) =
                make_uint4(pack2(f[0] * inv, f[1] * inv), pack2(f[2] * inv, f[3] * inv), pack2(f[4] * inv, f[5] * inv), pack2(f[6] * inv, f[7] * inv));
        } else {
            float4* dst = reinterpret_cast<float4*>(static_cast<float*>(p.o) + to);
            dst[0] = make_float4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
            dst[1] = make_float4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
        }
        if (p.lse && d8 == 0) p.lse[at] = none ? kNegInf : (M + __log2f(L)) * kLn2;
    }
}

template <int D, int RT>
hipError_t go(const Kv4Attn& p, hipStream_t stream) {
    const int rows = p.c.n * (p.hq / p.c.hk), tiles = (rows + 16 * RT - 1) / (16 * RT);
    // A negative scale goes into the queries' signs; a factor of zero becomes the
    // smallest one there is (kernels here keep subnormal numbers), whose weights
    // round to 1 as well, so that masked scores keep the weight 0.
    float c = p.scale * kLog2e;
    const bool flip = c < 0.0f;
    c = flip ? -c : c;
    if (c == 0.0f) c = std::numeric_limits<float>::denorm_min();
    const long long blocks = (long long)p.c.B * p.c.hk * tiles * p.splits;
    const auto run = [&](auto kernel) {
        return launch_kernel(kernel, dim3((unsigned)blocks), dim3(WAVES * 64), stream, p, c, flip, tiles);
    };
    const hipError_t e = tiles == 1 ? run(kv4_attn_kernel<D, RT, true>) : run(kv4_attn_kernel<D, RT, false>);
    if (e != hipSuccess || p.splits == 1) return e;
    const SplitJoin j{p.ws, p.o, p.lse, p.c.new_lens, {p.os[0], p.os[1], p.os[2]}, p.c.B, p.hq, p.c.n, p.splits, p.out_bf16};
    return launch_split_join<D>(j, stream);
}

}  // namespace

int kv4_rows_per_block(int rows) { return rows <= 16 ? 16 : 32; }

hipError_t launch_kv4_attn(const Kv4Attn& p, hipStream_t stream) {
    const bool one = kv4_rows_per_block(p.c.n * (p.hq / p.c.hk)) == 16;
    if (p.c.d == 64) return one ? go<64, 1>(p, stream) : go<64, 2>(p, stream);
    return one ? go<128, 1>(p, stream) : go<128, 2>(p, stream);
}

}  // namespace moa
