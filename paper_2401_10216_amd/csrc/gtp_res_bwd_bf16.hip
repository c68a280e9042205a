// The residual step's gradient: bf16 rows.
#include "gtp_res_bwd.hpp"

namespace gtp {

hipError_t launch_res_backward_bf16(const ResArgs& a, const ResLay& y, hipStream_t s) {
  const Backward f{a, y, s};
  return a.L == 0 ? res_with_team<uint16_t, 4, true>(y, f) : res_with_team<uint16_t, 4, false>(y, f);
}

}  // namespace gtp
