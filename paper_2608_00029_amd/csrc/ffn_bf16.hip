// Gated projections in bfloat16: the forms of the tile kernel (ffn_tile.h; which one a
// product takes: ffn_sched.h).
#include "ffn_tile.h"

namespace cattn {

template <int MODE> struct LaunchBf16 {
  static hipError_t run(TileArgs<bf16> g, hipStream_t st) {
    const FfnPlan plan = ffn_plan(MODE, g.M, g.N, g.K, true);
    g.parts = plan.parts;
    switch (plan.form) {
      case F256: return launch_form<bf16, MODE, 4, 2, 2, 4, 2, 1>(g, st);
      case F192: return launch_form<bf16, MODE, 2, 4, 3, 2, 2, 1>(g, st);
      case F256X128: return launch_form<bf16, MODE, 4, 2, 2, 2, 2, 1>(g, st);
      case F64: return launch_form<bf16, MODE, 2, 1, 1, 2, 4, 1, 2>(g, st);
      case F128X64:
        if constexpr (MODE == FWD) return launch_form<bf16, MODE, 4, 1, 1, 2, 3, 1, 2>(g, st);
        break;
      case F128: return launch_form<bf16, MODE, 4, 2, 1, 2, 4, 3>(g, st);
    }
    return hipErrorInvalidValue;
  }
};

hipError_t launch_gated_fwd_bf16(const GatedFwd& a, hipStream_t st) { return tiles_fwd<bf16, LaunchBf16>(a, st); }
hipError_t launch_gated_bwd_bf16(const GatedBwd& a, hipStream_t st) { return tiles_bwd<bf16, LaunchBf16>(a, st); }

}  // namespace cattn
