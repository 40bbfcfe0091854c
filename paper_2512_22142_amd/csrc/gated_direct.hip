// The bf16 fast path of cleave_linear_gated.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_gated_direct_kernels() { return configure_all<kBf16, GatedEpilogue>(); }

hipError_t launch_gated_direct(const ExecuteArgs& args, const GatedArgs& epi, DirectShape shape, bool tails, int grid,
                               hipStream_t stream) {
  return launch_with<kBf16>(args, GatedEpilogue{epi}, shape, tails, grid, stream);
}

}  // namespace cleave
