// The bf16 fast path of cleave_linear_gated_grad.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_gated_grad_kernels() { return configure_all<kBf16, GatedGradEpilogue>(); }

hipError_t launch_gated_grad_direct(const ExecuteArgs& args, const GatedArgs& epi, DirectShape shape, bool tails, int grid,
                                    hipStream_t stream) {
  return launch_with<kBf16>(args, GatedGradEpilogue{epi}, shape, tails, grid, stream);
}

}  // namespace cleave
