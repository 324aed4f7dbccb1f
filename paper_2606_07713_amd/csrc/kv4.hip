// Quantising keys and values into the pages of the four-bit cache, and reading
// them back (moa_kv4.h has the format).
//
// Both move 2.53 bytes per element (fp32: 4.53) and do little else, so device
// memory bounds them (8192 tokens, 16 heads, d = 128, bf16, 85 MB: written in 17.6
// us, 4.8 TB/s, read back in 15, 5.6, where copies of that mix reach 6.5; fp32, 152
// MB: 36 and 75).  A group of d/8 lanes takes the four tokens of an aligned quad: a
// lane has the same eight elements of all four, which makes its value codes one
// 16-byte piece of the page ([d/4][4][2] of the quad) and its key codes 4 bytes of
// four rows.  A quad of which only some tokens belong to the call (a single
// decoded token) writes 2-byte pieces of the quad, never a byte of another
// token: no read-modify-write, so different calls may fill one quad.
#include "kv4_common.h"

namespace moa {
namespace {

using namespace kv4;

constexpr int THREADS = 256;   // as kv4_row_blocks counts them

// The quad of one lane group: tokens 4 * quad + j of sequence b, head h.
template <int D>
struct Quad {
    int b, h, lane8;        // lane8: this lane's elements are 8 lane8 ..
    int row0;               // row of token j = 0 (may be negative)
    int count;              // new tokens of the sequence
    unsigned char* page;    // null: nothing to do
    int at;                 // quad within the page
    __device__ __forceinline__ bool row_in(int j) const { return row0 + j >= 0 && row0 + j < count; }
};

// Groups are numbered over (b, h, quad), the quads of one head fastest; a
// sequence's n new tokens touch at most `quads` of them.
template <int D>
__device__ __forceinline__ Quad<D> quad_of(const Kv4Cache& c, int quads) {
    constexpr int LPR = D / 8;
    Quad<D> q;
    q.page = nullptr;
    q.lane8 = threadIdx.x % LPR;
    const long long g = (long long)blockIdx.x * (THREADS / LPR) + threadIdx.x / LPR;
    const int bh = (int)(g / quads), i = (int)(g - (long long)bh * quads);
    if (bh >= c.B * c.hk) return q;
    q.b = bh / c.hk;
    q.h = bh - q.b * c.hk;
    q.count = new_tokens(c, q.b);
    const long long first = (long long)c.seq_lens[q.b] - q.count;   // position of row 0
    const long long quad = (first >> 2) + i, capacity = (long long)c.max_pages * c.page;
    if (quad < 0 || 4 * quad >= capacity) return q;
    q.row0 = (int)(4 * quad - first);
    if (q.row0 >= q.count) return q;
    const int pos = (int)(4 * quad), index = pos / c.page;
    q.page = page_of(c, q.b, q.h, index);
    q.at = (pos - index * c.page) >> 2;
    return q;
}

// Offsets of a quad's parts: key codes of token j, key scale of token j (block
// blk), value codes of the lane's eight elements, value scales of block blk.
template <int D>
__device__ __forceinline__ int key_code_at(int quad, int j, int lane8) { return (4 * quad + j) * (D / 2) + 4 * lane8; }
template <int D>
__device__ __forceinline__ int key_scale_at(int page, int quad, int j, int blk) {
    const int tile = quad >> 4, t = (quad >> 2) & 3, r = 4 * (quad & 3) + j;
    return key_scales(page, D) + tile * 2 * D + blk * 64 + r * 4 + t;
}
template <int D>
__device__ __forceinline__ int val_code_at(int page, int quad, int lane8) { return val_codes(page, D) + quad * 2 * D + lane8 * 16; }
template <int D>
__device__ __forceinline__ int val_scale_at(int page, int quad, int blk) {
    const int tile = quad >> 4, t = (quad >> 2) & 3, g = quad & 3;
    return val_scales(page, D) + tile * 2 * D + blk * 64 + g * 16 + t * 4;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        f[0] = bf16lo_to_f32(w.x); f[1] = bf16hi_to_f32(w.x);
        f[2] = bf16lo_to_f32(w.y); f[3] = bf16hi_to_f32(w.y);
        f[4] = bf16lo_to_f32(w.z); f[5] = bf16hi_to_f32(w.z);
        f[6] = bf16lo_to_f32(w.w); f[7] = bf16hi_to_f32(w.w);
    } else {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
}

// Codes of eight elements (element e at bits 4 e) and the scale byte of their
// block, which four neighbouring lanes hold.
__device__ __forceinline__ uint32_t quantise8(const float (&f)[8], uint32_t& byte) {
    uint32_t top = 0;   // of the magnitudes' bits: NaN and infinity are above all numbers
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, kDppQuadXor1, 0xf, 0xf, false));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, kDppQuadXor2, 0xf, 0xf, false));
    // a = 1.f * 2^(E-127) <= 1.75 * 2^2 * 2^(byte-127)
    const int exponent = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    byte = top >= 0x7f800000u ? 255u : (uint32_t)min(max(exponent, 2), 252);
    const float scale = scale_of(byte);
    uint32_t w = 0;   // nearest value, ties to the even code, at most 6
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
    return w;
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void kv4_write_kernel(Kv4Rows p, int quads) {
    const Quad<D> q = quad_of<D>(p.c, quads);
    if (!q.page) return;
    const int page = p.c.page, blk = q.lane8 >> 2;
    const bool first = (q.lane8 & 3) == 0;
    const T* k = static_cast<const T*>(p.kin) + q.b * p.ks[0] + q.h * p.ks[1] + 8 * q.lane8;
    const T* v = static_cast<const T*>(p.vin) + q.b * p.vs[0] + q.h * p.vs[1] + 8 * q.lane8;
    uint32_t codes[4], bytes = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        codes[j] = 0;
        if (!q.row_in(j)) continue;
        float f[8];
        uint32_t byte;
        load8(k + (long long)(q.row0 + j) * p.ks[2], f);
        *reinterpret_cast<uint32_t*>(q.page + key_code_at<D>(q.at, j, q.lane8)) = quantise8(f, byte);
        if (first) q.page[key_scale_at<D>(page, q.at, j, blk)] = (unsigned char)byte;
        load8(v + (long long)(q.row0 + j) * p.vs[2], f);
        codes[j] = quantise8(f, byte);
        bytes |= byte << (8 * j);
    }
    unsigned char* vc = q.page + val_code_at<D>(page, q.at, q.lane8);
    unsigned char* vs = q.page + val_scale_at<D>(page, q.at, blk);
    if (q.row_in(0) && q.row_in(3)) {
        uint4 w;   // [two fours of elements][4 tokens][2 bytes]
        w.x = __builtin_amdgcn_perm(codes[1], codes[0], 0x05040100);
        w.y = __builtin_amdgcn_perm(codes[3], codes[2], 0x05040100);
        w.z = __builtin_amdgcn_perm(codes[1], codes[0], 0x07060302);
        w.w = __builtin_amdgcn_perm(codes[3], codes[2], 0x07060302);
        *reinterpret_cast<uint4*>(vc) = w;
        if (first) *reinterpret_cast<uint32_t*>(vs) = bytes;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (!q.row_in(j)) continue;
        *reinterpret_cast<u16*>(vc + 2 * j) = (u16)codes[j];
        *reinterpret_cast<u16*>(vc + 8 + 2 * j) = (u16)(codes[j] >> 16);
        if (first) vs[j] = (unsigned char)(bytes >> (8 * j));
    }
}

// Two codes of byte B of w, times the scale: exact in bf16.
template <int B>
__device__ __forceinline__ uint32_t values2(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

// Four times as much is written as read: past the caches (4 sequences of up to
// 16384 tokens, 8 heads, d = 128, 282 MB: 59.4 -> 42.5 us, 6.6 TB/s).
__device__ __forceinline__ void store_past(void* p, u32x4 v) { __builtin_nontemporal_store(v, static_cast<u32x4*>(p)); }

template <typename T>
__device__ __forceinline__ void store8(T* p, uint32_t codes, float scale) {
    const uint4 w = make_uint4(values2<0>(codes, scale), values2<1>(codes, scale), values2<2>(codes, scale),
                               values2<3>(codes, scale));
    if constexpr (sizeof(T) == 2) {
        store_past(p, u32x4{w.x, w.y, w.z, w.w});
    } else {
        store_past(p, u32x4{w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u});
        store_past(p + 4, u32x4{w.z << 16, w.z & 0xffff0000u, w.w << 16, w.w & 0xffff0000u});
    }
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void kv4_read_kernel(Kv4Rows p, int quads) {
    const Quad<D> q = quad_of<D>(p.c, quads);
    if (!q.page) return;
    const int page = p.c.page, blk = q.lane8 >> 2;
    T* k = static_cast<T*>(p.kout) + q.b * p.ks[0] + q.h * p.ks[1] + 8 * q.lane8;
    T* v = static_cast<T*>(p.vout) + q.b * p.vs[0] + q.h * p.vs[1] + 8 * q.lane8;
    uint32_t kc[4], kb[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        kc[j] = *reinterpret_cast<const uint32_t*>(q.page + key_code_at<D>(q.at, j, q.lane8));
        kb[j] = q.page[key_scale_at<D>(page, q.at, j, blk)];
    }
    const uint4 w = *reinterpret_cast<const uint4*>(q.page + val_code_at<D>(page, q.at, q.lane8));
    const uint32_t bytes = *reinterpret_cast<const uint32_t*>(q.page + val_scale_at<D>(page, q.at, blk));
    const uint32_t vc[4] = {__builtin_amdgcn_perm(w.z, w.x, 0x05040100), __builtin_amdgcn_perm(w.z, w.x, 0x07060302),
                            __builtin_amdgcn_perm(w.w, w.y, 0x05040100), __builtin_amdgcn_perm(w.w, w.y, 0x07060302)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (!q.row_in(j)) continue;
        store8(k + (long long)(q.row0 + j) * p.ks[2], kc[j], scale_of(kb[j]));
        store8(v + (long long)(q.row0 + j) * p.vs[2], vc[j], scale_of((bytes >> (8 * j)) & 255u));
    }
}

template <typename K>
hipError_t go(K kernel, const Kv4Rows& p, hipStream_t stream) {
    const long long blocks = kv4_row_blocks(p.c.B, p.c.hk, p.c.n, p.c.d);
    return launch_kernel(kernel, dim3((unsigned)blocks), dim3(THREADS), stream, p, kv4_quads(p.c.n));
}

}  // namespace

hipError_t launch_kv4_write(const Kv4Rows& p, hipStream_t stream) {
    if (p.bf16) return p.c.d == 64 ? go(kv4_write_kernel<u16, 64>, p, stream) : go(kv4_write_kernel<u16, 128>, p, stream);
    return p.c.d == 64 ? go(kv4_write_kernel<float, 64>, p, stream) : go(kv4_write_kernel<float, 128>, p, stream);
}

hipError_t launch_kv4_read(const Kv4Rows& p, hipStream_t stream) {
    if (p.bf16) return p.c.d == 64 ? go(kv4_read_kernel<u16, 64>, p, stream) : go(kv4_read_kernel<u16, 128>, p, stream);
    return p.c.d == 64 ? go(kv4_read_kernel<float, 64>, p, stream) : go(kv4_read_kernel<float, 128>, p, stream);
}

}  // namespace moa
