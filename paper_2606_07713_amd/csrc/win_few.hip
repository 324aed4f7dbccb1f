// Attention with a window for few rows: up to 32 of one key/value head, a row
// being a query and one of the G = Hq/Hk heads that share it, query by query
// (moa_window.h, moa_paged.h).
//
// A workgroup takes RT tiles of 16 rows over a range of keys; its four waves take
// the range's 32-key steps in turn, each with a softmax state of its own, and join
// them at the end.  Keys and values go from memory to registers, without LDS: for
// S^T = K Q^T a lane holds chunks of a key's row as they are stored.  For O^T +=
// V^T P^T it needs eight keys of one element; since which element is whose is
// free, lane r of 16 takes elements D/16 r .. of its eight keys, a wave's load
// covers four whole rows, and turning the eight pieces inside the lane is one
// v_perm for each register.  The S^T accumulators leave a lane with the keys
// 4 g .. 4 g + 3 of two groups of 16 for its row, which is the second product's
// operand when the values are taken in the same order: no weight crosses a lane.
// A weight meets V as two bf16 numbers, 17 bits together, or as three, all of its bits,
// for an fp32 output, whose rounding is far below two; the sums are of the fp32 weights.
//
// What bounds it: HBM.  64 sequences of 8192 tokens, 32 heads on 8, d = 128: 316 us,
// 6.8 TB/s, the matrix cores 0.06 busy.  One sequence of 4097: 8 us in 256 workgroups and
// 4 for the join, latencies.
#include <limits>

#include "split_join.h"
#include "win_common.h"

namespace moa {
namespace {

using namespace win;

constexpr int WAVES = 4;
constexpr int T = 32;                     // keys of a step
constexpr float kLargeSum = 1048576.0f;   // a lane's sum of one step's weights that raises the reference
constexpr int kNonTemporal = 2;

// The keys and values of 32 keys that one lane holds.  ONCE: no other workgroup
// reads them, so they need not stay in the caches.
template <int D, bool ONCE>
struct Step {
    typedef uint32_t vec __attribute__((ext_vector_type(D / 32)));
    u32x4 k[2][D / 32];
    vec v[8];

    // Group t of 16 keys; rows behind the descriptors' ends are zeros.
    __device__ __forceinline__ void load(int t, __amdgpu_buffer_rsrc_t rk, __amdgpu_buffer_rsrc_t rv, uint32_t koff,
                                         const uint32_t (&voff)[4]) {
        constexpr int AUX = ONCE ? kNonTemporal : 0;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) k[t][s] = __builtin_amdgcn_raw_buffer_load_b128(rk, koff + 64 * s, 0, AUX);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (D == 128) v[4 * t + j] = __builtin_amdgcn_raw_buffer_load_b128(rv, voff[j], 0, AUX);
            else v[4 * t + j] = __builtin_amdgcn_raw_buffer_load_b64(rv, voff[j], 0, AUX);
        }
    }
    // V^T operand of elements 2 W (LOW) or 2 W + 1 of the lane's D/16.
    __device__ __forceinline__ bf16x8 values(int w, bool low) const {
        const uint32_t which = low ? 0x05040100u : 0x07060302u;
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_perm(v[2 * i + 1][w], v[2 * i][w], which);
        return __builtin_bit_cast(bf16x8, r);
    }
};

template <int D, int RT, int TERMS, bool ONCE>
__global__ __launch_bounds__(WAVES * 64, RT == 1 ? 2 : 1) void win_few_kernel(WinAttn p, float c, bool flip, int row_tiles) {
    constexpr int E = D / 16, ROWS = 16 * RT, LD = D + 4;
    __shared__ __attribute__((aligned(16))) float part[WAVES][ROWS][LD];
    __shared__ float part_m[WAVES][ROWS], part_l[WAVES][ROWS];
    __shared__ int again[ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const KeySource& src = p.s;
    const int G = (int)p.group.n;
    // Row tiles last, those of the highest positions first.
    const int up = over(p.per_tile, blockIdx.x), rt = row_tiles - 1 - up, in_tile = blockIdx.x - up * (int)p.per_tile.n;
    const int bh = over(p.per_head, in_tile), sp = in_tile - bh * p.splits, b = over(p.heads, bh), h = bh - b * p.hk;

    const int count = new_tokens(src.new_lens, b, p.n), rows = count * G, row0 = rt * ROWS;
    if (row0 >= rows) return;
    const int len = length(src, b), end = max(0, min(len, capacity(src)));
    const long long first = (long long)len - count;   // position of query 0
    const auto seen_of = [&](int row) { return seen_from(p.w, first + over(p.group, row), end); };
    // Rows behind the last one are computed as it is, with queries of zero, and not stored.
    Seen seen[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) seen[i] = seen_of(min(row0 + 16 * i + n, rows - 1));
    Seen low = seen_of(row0), high = seen_of(min(row0 + ROWS, rows) - 1);
    low.lo = __builtin_amdgcn_readfirstlane(low.lo); low.hi = __builtin_amdgcn_readfirstlane(low.hi);
    high.lo = __builtin_amdgcn_readfirstlane(high.lo); high.hi = __builtin_amdgcn_readfirstlane(high.hi);
    const Tiles<T> steps(low, high, p.w.sinks);
    const int per = (steps.count + p.splits - 1) / p.splits, begin = sp * per, stop = min(steps.count, begin + per);

    bf16x8 q[RT][D / 32];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int row = row0 + 16 * i + n;
        const bool in = row < rows;
        const int qi = in ? over(p.group, row) : 0, hh = h * G + (in ? row - qi * G : 0);
        const u16* at = static_cast<const u16*>(p.q) + b * p.qs[0] + hh * p.qs[1] + qi * p.qs[2] + g * 8;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            uint4 w = in ? *reinterpret_cast<const uint4*>(at + 32 * k) : make_uint4(0, 0, 0, 0);
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
    const uint32_t krb = (uint32_t)src.ks[2] * 2u, vrb = (uint32_t)src.vs[2] * 2u, koff = n * krb + g * 16;
    uint32_t voff[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) voff[j] = (4 * g + j) * vrb + n * (D / 8);

    // Lane 2 i + t holds the page of group t of this wave's i-th step from `known` on.
    int pages = 0, known = begin + wave, at = begin + wave;
    const auto look = [&]() {
        const int v = known + WAVES * (lane >> 1), key = steps.at(v) * T + 16 * (lane & 1);
        pages = v < stop && key < end ? page_of(src, b, key) : -1;
    };
    // Loads the step at `at` and moves on; bit t: group t has a page.  Something is
    // loaded in any case, so that the number of loads in flight is known where a
    // step's own are waited for.
    const auto fetch = [&](Step<D, ONCE>& x) -> int {
        if (at - known == 32 * WAVES) {
            known = at;
            look();
        }
        const int i = (at - known) / WAVES, k0 = steps.at(at) * T;
        int have = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * i + t), key = k0 + 16 * t;
            const int in = page >= 0 ? max(0, min(16, end - key)) : 0;
            have |= page >= 0 ? 1 << t : 0;
            const u16* kb = static_cast<const u16*>(src.k) + (in ? key_offset(src.ks, src.shift, page, h, key) : 0);
            const u16* vb = static_cast<const u16*>(src.v) + (in ? key_offset(src.vs, src.shift, page, h, key) : 0);
            x.load(t, make_rsrc(kb, rows_extent(in, krb, 2 * D)), make_rsrc(vb, rows_extent(in, vrb, 2 * D)), koff, voff);
        }
        at += WAVES;
        return have;
    };
    const auto attend = [&](Step<D, ONCE>& x, int v, int have) {
        const int k0 = steps.at(v) * T;
        f32x4 s[RT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                f32x4 a = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < D / 32; ++k)
                    a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[t][k]), q[i][k], a, 0, 0, 0);
                s[i][t] = a;
            }
        const bool masked = have != 3 || !all_see(low, high, p.w.sinks, k0);
        if (masked) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                uint32_t bits = seen_bits(seen[i], p.w.sinks, k0);
                if (have != 3) bits &= (have & 1 ? 0x0000ffffu : 0u) | (have & 2 ? 0xffff0000u : 0u);
                bits >>= 4 * g;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[i][t][j] = keep_bit(s[i][t][j], bits, 16 * t + j);
            }
        }
        // The weights 2^(s c - ref), each as TERMS bf16 numbers, and their sums.
        u32x4 pt[RT][TERMS];
        float sum[RT];
        const auto weights = [&]() {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const float shift = ref[i] == kNegInf ? 0.0f : -ref[i];
                float w[8], total = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = exp2_hw(__builtin_fmaf(s[i][j / 4][j % 4], c, shift));
                    total += w[j];
                }
                sum[i] = total;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t x[TERMS];
                    bf16_terms<TERMS>(w[2 * j], w[2 * j + 1], x);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) pt[i][k][j] = x[k];
                }
            }
        };
        // Against the present references, without a maximum, unless the step is
        // masked, a row has seen nothing yet or a sum comes out too large.
        bool raise = masked || !ready;
        if (!raise) {
            weights();
            bool large = false;
#pragma unroll
            for (int i = 0; i < RT; ++i) large |= !(sum[i] <= kLargeSum);
            raise = wave_any(large);
        }
        if (raise) {
            ready = true;
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float m = kNegInf;
#pragma unroll
                for (int j = 0; j < 8; ++j) m = fmaxf(m, s[i][j / 4][j % 4]);
                m = fmaxf(ref[i], column_max(m) * c);
                const float a = ref[i] == kNegInf ? 0.0f : exp2_hw(ref[i] - m);
                ref[i] = m;
                l[i] *= a;
#pragma unroll
                for (int e = 0; e < E; ++e) o[i][e] *= a;
                ready &= !wave_any(m == kNegInf);
            }
            weights();
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) l[i] += sum[i];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bf16x8 a = x.values(e / 2, e % 2 == 0);
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int k = 0; k < TERMS; ++k)
                    o[i][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, pt[i][k]), o[i][e], 0, 0, 0);
        }
    };
    // Two steps in registers: the next one's loads are in flight while one is worked on.
    if (at < stop) {
        look();
        Step<D, ONCE> x0, x1;
        int have0 = fetch(x0);
        for (int v = begin + wave; v < stop; v += 2 * WAVES) {
            const int have1 = fetch(x1);
            if (have0) attend(x0, v, have0);
            have0 = fetch(x0);
            if (have1) attend(x1, v + WAVES, have1);
        }
    }

    // Join the waves' states: a common reference per row, then sums.
    if (threadIdx.x < ROWS) again[threadIdx.x] = 0;
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
        if (g == 0) part_l[wave][row] = ref[i] == kNegInf ? l[i] : l[i] * a;
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
        const int qi = over(p.group, row), hh = h * G + row - qi * G;
        // Sums that are not finite, or none at all in a row that sees keys: by the definition.
        const float most = p.splits > 1 ? (float)kMaxSplits : 1.0f;
        float zero = 0.0f * (L * most);
#pragma unroll
        for (int e = 0; e < 8; ++e) zero = __builtin_fmaf(f[e] * most, 0.0f, zero);
        if (!(zero == 0.0f) || (L == 0.0f && begin < stop && sees_any(seen_of(row), p.w.sinks))) again[r] = 1;
        const size_t to_row = ((size_t)b * p.hq + hh) * p.n + qi;
        if (p.splits > 1) {
            float* acc = p.ws + (to_row * p.splits + sp) * D + d8;
            reinterpret_cast<float4*>(acc)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(acc)[1] = make_float4(f[4], f[5], f[6], f[7]);
            if (d8 == 0) {
                float* ml = p.ws + (size_t)p.B * p.hq * p.n * p.splits * D + (to_row * p.splits + sp) * 2;
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
        if (p.lse && d8 == 0) p.lse[to_row] = none ? kNegInf : (M + __log2f(L)) * kLn2;
    }
    __syncthreads();
    for (int r = wave; r < ROWS; r += WAVES) {
        if (!again[r]) continue;
        const int row = row0 + r, qi = over(p.group, row), hh = h * G + row - qi * G;
        float f[D / 64], M, L;
        row_by_definition<D, T>(p, b, h, static_cast<const u16*>(p.q) + b * p.qs[0] + hh * p.qs[1] + qi * p.qs[2],
                                seen_of(row), steps, begin, stop, p.splits > 1, f, M, L);
        store_row<D>(p, b, hh, qi, sp, f, M, L);
    }
}

template <int D, int RT>
hipError_t go(WinAttn p, hipStream_t stream) {
    set_divisions(p);
    const int rows = p.n * (p.hq / p.hk), tiles = (rows + 16 * RT - 1) / (16 * RT);
    // A negative scale goes into the queries' signs; a factor of zero becomes the
    // smallest one there is (kernels here keep subnormal numbers), whose weights
    // round to 1 as well, so that masked scores keep the weight 0.
    float c = p.scale * kLog2e;
    const bool flip = c < 0.0f;
    c = flip ? -c : c;
    if (c == 0.0f) c = std::numeric_limits<float>::denorm_min();
    const long long blocks = (long long)p.B * p.hk * tiles * p.splits;
    const auto run = [&](auto kernel) {
        return launch_kernel(kernel, dim3((unsigned)blocks), dim3(WAVES * 64), stream, p, c, flip, tiles);
    };
    constexpr int BF16 = 2, F32 = 3;   // terms of a weight
    hipError_t e;
    if (p.out_bf16) e = tiles == 1 ? run(win_few_kernel<D, RT, BF16, true>) : run(win_few_kernel<D, RT, BF16, false>);
    else e = tiles == 1 ? run(win_few_kernel<D, RT, F32, true>) : run(win_few_kernel<D, RT, F32, false>);
    if (e != hipSuccess || p.splits == 1) return e;
    const SplitJoin j{p.ws, p.o, p.lse, p.s.new_lens, {p.os[0], p.os[1], p.os[2]}, p.B, p.hq, p.n, p.splits, p.out_bf16};
    return launch_split_join<D>(j, stream, RowsAgain{p});
}

}  // namespace

hipError_t launch_win_few(const WinAttn& p, hipStream_t stream) {
    const bool one = p.n * (p.hq / p.hk) <= 16;
    if (p.d == 64) return one ? go<64, 1>(p, stream) : go<64, 2>(p, stream);
    return one ? go<128, 1>(p, stream) : go<128, 2>(p, stream);
}

hipError_t launch_win_attn(const WinAttn& p, hipStream_t stream) {
    const long long rows = (long long)p.n * (p.hq / p.hk);
    return win_rows_per_block(rows) < 128 ? launch_win_few(p, stream) : launch_win_many(p, stream);
}

}  // namespace moa
