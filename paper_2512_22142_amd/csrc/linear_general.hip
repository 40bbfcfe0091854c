// The general path of cleave_linear: any element type, size and alignment.
#include "execute_general.h"

namespace cleave {

namespace {

// Of the tiles that cleave_execute has, the two that serve every size with the registers an epilogue needs (two waves to a
// SIMD; with four it spills: 3001 x 2500 x 1000 with bias and residual 53 us).
template <int EB>
using ElementTile = Shape<EB, 64, 64, 2, 2, 1, 2>;

template <int EB>
hipError_t configure_type() {
  hipError_t e = configure_layouts<Wide4<EB>, LinearEpilogue>();
  if (e == hipSuccess) e = configure_layouts<Lone<EB>, LinearEpilogue>();
  if (e == hipSuccess) e = configure_elements<ElementTile<EB>, LinearEpilogue>();
  return e;
}

template <int EB>
hipError_t launch_type(const ExecuteArgs& args, const LinearEpilogue& epi, int tile_class, const GeneralLoads& how,
                       hipStream_t stream) {
  if (how.a_elements || how.b_elements) return launch_elements<ElementTile<EB>>(args, epi, tile_class, how, stream);
  return how.tile == kTileLone ? launch_layouts<Lone<EB>>(args, epi, tile_class, how, stream)
                               : launch_layouts<Wide4<EB>>(args, epi, tile_class, how, stream);
}

}  // namespace

hipError_t configure_linear_general_kernels() {
  const hipError_t e = configure_type<2>();
  return e != hipSuccess ? e : configure_type<4>();
}

hipError_t launch_linear_general(const ExecuteArgs& args, const LinearArgs& epi, int dtype, int tile_class,
                                 const GeneralLoads& how, hipStream_t stream) {
  return dtype == CLEAVE_BF16 ? launch_type<2>(args, LinearEpilogue{epi}, tile_class, how, stream)
                              : launch_type<4>(args, LinearEpilogue{epi}, tile_class, how, stream);
}

}  // namespace cleave
