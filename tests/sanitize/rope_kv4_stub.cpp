// Stand-ins for the kernel launchers behind moa_rope.h and moa_kv4.h, for the
// sanitizer build of their C-ABI front ends; see launch_stub.cpp.
#include "../../paper_2606_07713_amd/csrc/kv4.h"
#include "../../paper_2606_07713_amd/csrc/rope.h"

namespace moa {

hipError_t launch_rope_fwd(const RopeProblem&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_rope_bwd(const RopeProblem&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv4_write(const Kv4Rows&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv4_read(const Kv4Rows&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv4_attn(const Kv4Attn&, hipStream_t) { return hipErrorNoDevice; }
int kv4_rows_per_block(int rows) { return rows <= 16 ? 16 : 32; }

}  // namespace moa
