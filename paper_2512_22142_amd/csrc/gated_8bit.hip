// cleave_linear_gated with 8-bit operands and more than a few rows.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_gated_8bit_kernels() { return configure_all<kE4M3, GatedEpilogue>(); }

hipError_t launch_gated_8bit(const ExecuteArgs& args, const GatedArgs& epi, DirectShape shape, bool tails, int grid,
                             hipStream_t stream) {
  return launch_with<kE4M3>(args, GatedEpilogue{epi}, shape, tails, grid, stream);
}

}  // namespace cleave
