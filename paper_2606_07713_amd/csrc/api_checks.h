// Checks of arguments that the entry points share (host code only).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace moa {

// MOA_OK, or MOA_ERR_HIP with the error's name kept for this thread.
int hip_status(hipError_t e);

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool overlaps(const void* a, size_t an, const void* b, size_t bn) {
    if (an == 0 || bn == 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + bn && b0 < a0 + an;
}

// Element strides of one tensor over (batch, head, row); d is contiguous.
struct Strides {
    int64_t b, h, r;
};

inline Strides contiguous(int64_t H, int64_t N, int64_t d) { return {H * N * d, N * d, d}; }

// Bytes from a tensor's base pointer to the end of its last element.
inline size_t extent_bytes(const Strides& s, int64_t B, int64_t H, int64_t N, int64_t d, size_t es) {
    if (B == 0 || H == 0 || N == 0 || d == 0) return 0;
    return (size_t)((B - 1) * s.b + (H - 1) * s.h + (N - 1) * s.r + d) * es;
}

// True if no two (batch, head, row, element) positions share an address:
// the dimensions of size > 1, by increasing stride, nest without overlap.
inline bool injective(const Strides& s, int64_t B, int64_t H, int64_t N, int64_t d) {
    if (B == 0 || H == 0 || N == 0) return true;   // nothing is written
    struct Dim { int64_t stride, count; } dims[3] = {{s.b, B}, {s.h, H}, {s.r, N}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (dims[j].stride < dims[i].stride) { Dim t = dims[i]; dims[i] = dims[j]; dims[j] = t; }
    int64_t span = d;   // elements covered by the inner dimensions so far
    for (int i = 0; i < 3; ++i) {
        if (dims[i].count <= 1) continue;
        if (dims[i].stride < span) return false;
        span = dims[i].stride * dims[i].count;
    }
    return true;
}

}  // namespace moa
