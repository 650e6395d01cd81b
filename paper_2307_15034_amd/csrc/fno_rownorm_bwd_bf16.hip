// The residual norm's backward, __bf16 rows.
#include "fno_rownorm_bwd.h"

namespace fno {

hipError_t launch_row_norm_bwd_bf16(const RowNormArgs& a, bool post, bool pre, const RowLaunchSize& l,
                                hipStream_t s) {
  return launch_form<__bf16>(a, post, pre, l, s);
}

}  // namespace fno
