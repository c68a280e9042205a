// The residual step's gradient: fp32 rows, and the choice of a way.
#include "gtp_res_bwd.hpp"

namespace gtp {

hipError_t launch_res_backward_f32(const ResArgs& a, const ResLay& y, hipStream_t s) {
  const Backward f{a, y, s};
  return a.L == 0 ? res_with_team<float, 4, true>(y, f) : res_with_team<float, 4, false>(y, f);
}

int64_t residual_work_floats(const ResArgs& a) {
  ResLay y;
  if (residual_layout(a, false, true, &y)) return res_grid(a.N, y) * res_columns(a.L, a.C);
  return residual_is_long(a) ? residual_long_floats(a) : residual_any_floats(a);
}

hipError_t launch_residual_backward(const ResArgs& a, hipStream_t s) {
  if (a.N == 0) return a.weights() ? launch_residual_sum(a, nullptr, 0, s) : hipSuccess;
  ResLay y;
  if (!residual_layout(a, false, true, &y))
    return residual_is_long(a) ? launch_residual_long_backward(a, s) : launch_residual_any_backward(a, s);
  const hipError_t e = a.bf16 ? launch_res_backward_bf16(a, y, s) : launch_res_backward_f32(a, y, s);
  return e == hipSuccess && a.weights() ? launch_residual_sum(a, a.work, res_grid(a.N, y), s) : e;
}

}  // namespace gtp
