// The fast path of cleave_linear with 8-bit operands.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_linear_8bit_kernels() { return configure_all<kE4M3, LinearEpilogue>(); }

hipError_t launch_linear_8bit(const ExecuteArgs& args, const LinearArgs& epi, DirectShape shape, bool tails, int grid,
                              hipStream_t stream) {
  return launch_with<kE4M3>(args, LinearEpilogue{epi}, shape, tails, grid, stream);
}

}  // namespace cleave
