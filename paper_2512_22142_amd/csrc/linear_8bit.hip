// The fast path of cleave_linear with 8-bit operands.
#include "execute_direct.h"

namespace cleave {

hipError_t configure_linear_8bit_kernels() {
  const hipError_t e = configure_all<kE4M3, LinearEpilogue>();
  return e == hipSuccess ? configure_all<kE4M3Exact, LinearEpilogue>() : e;
}

hipError_t launch_linear_8bit(const ExecuteArgs& args, const LinearArgs& epi, DirectShape shape, bool tails, int grid,
                              hipStream_t stream) {
  return args.C && args.c_bf16 ? launch_with<kE4M3>(args, LinearEpilogue{epi}, shape, tails, grid, stream)
                               : launch_with<kE4M3Exact>(args, LinearEpilogue{epi}, shape, tails, grid, stream);
}

}  // namespace cleave
