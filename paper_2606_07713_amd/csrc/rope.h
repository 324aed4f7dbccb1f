// Internal launch interface of the head norms with rotation (rope.hip).
#pragma once

#include <hip/hip_runtime_api.h>

namespace moa {

constexpr int kRopeMaxAxes = 4;
// Workgroups of the gradient kernel at most: each writes a partial sum of the
// weights' gradients (both tensors, d floats each).
constexpr int kRopeBwdMaxBlocks = 1024;

// Index 0 is Q, 1 is K.  Strides in elements over (batch, head, row).
struct RopeProblem {
    const void* x[2];      // the forward's inputs
    const void* g[2];      // gradients of its outputs (backward)
    void* y[2];            // outputs: the rotated rows, or the gradients of x
    const void* w[2];      // norm weights, or null: no norm
    long long xs[2][3], gs[2][3], ys[2][3];
    const long long* pos;  // [axes][B*N], or null
    const float* freq;     // [rot/2]
    float* dw[2];          // gradients of w (backward)
    float* ws;             // [blocks][2][d] partial sums (backward)
    int B, N, H[2], d, rot;
    int axes, first[kRopeMaxAxes];   // first[a]: pairs before axis a's
    float eps;
    bool interleaved, bf16, w_bf16;
};

hipError_t launch_rope_fwd(const RopeProblem& p, hipStream_t stream);
hipError_t launch_rope_bwd(const RopeProblem& p, hipStream_t stream);

}  // namespace moa
