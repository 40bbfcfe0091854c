// The general path of cleave_linear: any element type, size and alignment.
#include "execute_general.h"

namespace cleave {

namespace {

// Of the tiles that cleave_execute has, the two that serve every size.
template <int EB>
hipError_t configure_type() {
  hipError_t e = configure_layouts<Wide<EB>, LinearEpilogue>();
  if (e == hipSuccess) e = configure_layouts<Narrow<EB>, LinearEpilogue>();
  if (e == hipSuccess) e = configure_elements<ByElement<EB>, LinearEpilogue>();
  return e;
}

template <int EB>
hipError_t launch_type(const ExecuteArgs& args, const LinearEpilogue& epi, int tile_class, const GeneralLoads& how,
                       hipStream_t stream) {
  if (how.a_elements || how.b_elements) return launch_elements<ByElement<EB>>(args, epi, tile_class, how, stream);
  return how.tile == kTileNarrow ? launch_layouts<Narrow<EB>>(args, epi, tile_class, how, stream)
                                 : launch_layouts<Wide<EB>>(args, epi, tile_class, how, stream);
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
