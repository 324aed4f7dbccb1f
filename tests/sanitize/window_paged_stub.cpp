// Stand-ins for the kernel launchers behind moa_window.h and moa_paged.h, for the
// sanitizer build of their C-ABI front ends; see launch_stub.cpp.
#include "../../paper_2606_07713_amd/csrc/paged.h"
#include "../../paper_2606_07713_amd/csrc/win.h"

namespace moa {

hipError_t launch_win_attn(const WinAttn&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_win_bwd(const WinGrad&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_paged_append(const AppendProblem&, hipStream_t) { return hipErrorNoDevice; }

}  // namespace moa
