// Internal launch interface of the appending to a paged cache (paged.hip).
#pragma once

#include "rope.h"
#include "win.h"

namespace moa {

// New tokens: queries and keys (r: inputs, norms, rotation, the rotated queries) and
// values, and where they go.
struct AppendProblem {
    RopeProblem r;
    const void* v;
    long long vs[3];   // element strides (batch, head, row)
    KeySource to;
};

hipError_t launch_paged_append(const AppendProblem& p, hipStream_t stream);

}  // namespace moa
