// The general path of cleave_execute and cleave_execute_assemble.
#include "execute_general.h"

namespace cleave {

namespace {

template <int EB>
hipError_t configure_type() {
  hipError_t e = configure_layouts<Wide<EB>, NoEpilogue>();
  if (e == hipSuccess) e = configure_layouts<Narrow<EB>, NoEpilogue>();
  if (e == hipSuccess) e = configure_layouts<Lone<EB>, NoEpilogue>();
  if (e == hipSuccess) e = configure_elements<ByElement<EB>, NoEpilogue>();
  if (EB == 4 && e == hipSuccess) e = configure_layouts<Quarter, NoEpilogue>();
  if (EB == 2 && e == hipSuccess) e = configure_one<Large, kByK, kByK, NoEpilogue>();
  if (e == hipSuccess) e = configure_one<Wide4<EB>, kByK, kByK, NoEpilogue>();
  if (e == hipSuccess) e = configure_one<Wide4<EB>, kByRow, kByRow, NoEpilogue>();
  if (EB == 4 && e == hipSuccess) e = configure_one<Wide4<4>, kByRow, kByK, NoEpilogue>();
  return e;
}

template <int EB>
hipError_t launch_type(const ExecuteArgs& args, int tile_class, const GeneralLoads& how, hipStream_t stream) {
  if (how.a_elements || how.b_elements)
    return launch_elements<ByElement<EB>>(args, NoEpilogue{}, tile_class, how, stream);
  if (EB == 2 && how.tile == kTileHuge) {   // large items, both operands K-contiguous
    ExecuteArgs whole = args;
    const int grid = cut_items<Large>(&whole, tile_class, how);
    return launch_one<Large, kByK, kByK>(whole, NoEpilogue{}, grid, stream);
  }
  if (how.tile == kTileWide4) {   // NT, TN and, fp32 only, TT
    ExecuteArgs cut = args;
    const int grid = cut_items<Wide4<EB>>(&cut, tile_class, how);
    if (!args.transA) return launch_one<Wide4<EB>, kByK, kByK>(cut, NoEpilogue{}, grid, stream);
    if (EB == 4 && args.transB) return launch_one<Wide4<4>, kByRow, kByK>(cut, NoEpilogue{}, grid, stream);
    return launch_one<Wide4<EB>, kByRow, kByRow>(cut, NoEpilogue{}, grid, stream);
  }
  if (EB == 4 && how.tile == kTileQuarter) return launch_layouts<Quarter>(args, NoEpilogue{}, tile_class, how, stream);
  if (how.tile == kTileLone) return launch_layouts<Lone<EB>>(args, NoEpilogue{}, tile_class, how, stream);
  return how.tile == kTileNarrow ? launch_layouts<Narrow<EB>>(args, NoEpilogue{}, tile_class, how, stream)
                                 : launch_layouts<Wide<EB>>(args, NoEpilogue{}, tile_class, how, stream);
}

}  // namespace

hipError_t configure_execute_kernels() {
  const hipError_t e = configure_type<2>();
  return e != hipSuccess ? e : configure_type<4>();
}

hipError_t launch_execute(const ExecuteArgs& args, int dtype, int tile_class, const GeneralLoads& how,
                          hipStream_t stream) {
  return dtype == CLEAVE_BF16 ? launch_type<2>(args, tile_class, how, stream)
                              : launch_type<4>(args, tile_class, how, stream);
}

}  // namespace cleave
