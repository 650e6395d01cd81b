// The residual norm's backward, float rows.
#include "fno_rownorm_bwd.h"

namespace fno {

hipError_t launch_row_norm_bwd_f32(const RowNormArgs& a, bool post, bool pre, const RowLaunchSize& l,
                                hipStream_t s) {
  return launch_form<float>(a, post, pre, l, s);
}

}  // namespace fno
