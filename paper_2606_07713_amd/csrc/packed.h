// Entry points that take the arguments of one call as a record of 8-byte words
// (host code only).  They serve this package's Python binding, whose foreign
// calls pay for every argument: the 25 of moa_qk_norm_rope take 1.9 us to hand
// over, a packed record 0.5, of a call of 12 us.
#pragma once

#include <stdint.h>
#include <string.h>

namespace moa {
namespace packed {

// A word that is a pointer of any type.
struct Ptr {
    int64_t word;
    template <typename T>
    operator T*() const { return reinterpret_cast<T*>(word); }
};

// A word that is a double, as Python packs its numbers.
inline float real(int64_t word) {
    double d;
    memcpy(&d, &word, sizeof d);
    return static_cast<float>(d);
}

}  // namespace packed
}  // namespace moa
