// The bf16 fast path of cleave_linear.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_linear_direct_kernels() { return configure_all<kBf16, LinearEpilogue>(); }

hipError_t launch_linear_direct(const ExecuteArgs& args, const LinearArgs& epi, DirectShape shape, bool tails, int grid,
                                hipStream_t stream) {
  return launch_with<kBf16>(args, LinearEpilogue{epi}, shape, tails, grid, stream);
}

}  // namespace cleave
