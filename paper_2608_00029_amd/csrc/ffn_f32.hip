// Gated projections in float32: the forms of the tile kernel (ffn_tile.h; which one a
// product takes: ffn_sched.h).
#include "ffn_tile.h"

namespace cattn {

template <int MODE> struct LaunchF32 {
  static hipError_t run(TileArgs<float> g, hipStream_t st) {
    const FfnPlan plan = ffn_plan(MODE, g.M, g.N, g.K, false);
    g.parts = plan.parts;
    switch (plan.form) {
      case F128: return launch_form<float, MODE, 2, 2, 2, 2, 2, 1>(g, st);
      case F64X128: return launch_form<float, MODE, 2, 2, 1, 2, 2, 1>(g, st);
      case F64:  // (a gate and an up column in one wave: two waves beside each other, so two sets)
        if constexpr (MODE == FWD) return launch_form<float, MODE, 2, 1, 1, 2, 2, 1, 2>(g, st);
        else return launch_form<float, MODE, 2, 2, 1, 1, 2, 1>(g, st);
    }
    return hipErrorInvalidValue;
  }
};

hipError_t launch_gated_fwd_f32(const GatedFwd& a, hipStream_t st) { return tiles_fwd<float, LaunchF32>(a, st); }
hipError_t launch_gated_bwd_f32(const GatedBwd& a, hipStream_t st) { return tiles_bwd<float, LaunchF32>(a, st); }

}  // namespace cattn
