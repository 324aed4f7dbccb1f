// Device-side layout of the four-bit key/value cache.
#pragma once

#include "device_common.h"
#include "kv4.h"

namespace moa {
namespace kv4 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Where the parts of one head's page begin, in bytes: key codes at 0.
__device__ __forceinline__ int key_scales(int page, int d) { return page * (d / 2); }
__device__ __forceinline__ int val_codes(int page, int d) { return page * (d / 2 + d / 32); }
__device__ __forceinline__ int val_scales(int page, int d) { return page * (d + d / 32); }

// New tokens of sequence b: how many, and the position of the first (which
// may lie before 0 or behind the capacity).
__device__ __forceinline__ int new_tokens(const Kv4Cache& c, int b) {
    return c.new_lens ? min(max(c.new_lens[b], 0), c.n) : c.n;
}

// One head's page, or null where there is none.
__device__ __forceinline__ unsigned char* page_of(const Kv4Cache& c, int b, int head, int index) {
    const int id = c.table ? c.table[(size_t)b * c.max_pages + index] : b;
    if (id < 0 || id >= c.num_pages) return nullptr;
    return c.base + ((size_t)id * c.hk + head) * c.page_bytes;
}

// The power of two of a scale byte.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace kv4
}  // namespace moa
