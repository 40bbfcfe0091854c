// The bf16 fast path of cleave_execute and cleave_execute_assemble.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_execute_direct_kernels() { return configure_all<kBf16, NoEpilogue>(); }

hipError_t launch_execute_direct(const ExecuteArgs& args, DirectShape shape, bool tails, int grid, hipStream_t stream) {
  return launch_with<kBf16>(args, NoEpilogue{}, shape, tails, grid, stream);
}

}  // namespace cleave
