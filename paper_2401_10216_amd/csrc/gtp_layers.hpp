// Launchers of the layers around the product: normalisation of SH features
// (gtp_norm.hip), the residual step (gtp_res_*.hip), dropout (gtp_drop.hip).  Arguments are validated by the C
// entries (gtp_layers.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/gtp.h"

namespace gtp {

// The message of the calling thread's last failed call (kept by gtp_api.hip).
gtp_status set_error(gtp_status s, const char* msg) noexcept;

struct NormArgs {
  const void *x, *dy;          // [N, C, K] of `bf16`'s type
  const float *w, *b;          // [L + 1, C], [C] or null (ones, zeros)
  const float *mean_in, *rstd_in;
  void* y;                     // y, or dx (may be null in the backward)
  float *mean, *rstd;          // [N], [N, L + 1] or null
  float *dw, *db;              // [L + 1, C], [C] or null
  float* partial;              // norm_partial_floats, for dw and db
  int64_t N, C;
  int L;
  bool bf16;
  float eps;
};
hipError_t launch_norm(const NormArgs& a, hipStream_t s);
int64_t norm_partial_floats(int L, int64_t N, int64_t C, bool bf16);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);

// The residual step r = x + scale sigmoid(gate) t, t = post ? norm(a) w_post + b_post : a,
// h = norm(r) w_pre + b_pre, and its gradient.
struct ResArgs {
  const void *x, *a, *gate;    // [N, C, K], the gate [N, C] or null (x: r in the backward)
  const void *dh, *dr;         // backward; dr null: zeros
  const float *scale, *w1, *b1, *w2, *b2;  // [L + 1, C] and [C], each may be null (ones, zeros); 1: post, 2: pre
  void *r, *h;
  float *mean1, *rstd1, *mean2, *rstd2;    // [N], [N, L + 1]: written by the forward (each may be null), read by the backward
  void *dx, *da, *dgate;       // each may be null
  float *dscale, *dw1, *db1, *dw2, *db2;
  float *work;                 // residual_work_floats
  int64_t N, C;
  int L;
  bool bf16, post;
  float eps;
  bool weights() const { return dscale || dw1 || db1 || dw2 || db2; }
};
hipError_t launch_residual(const ResArgs& a, hipStream_t s);
// floats of work of the backward, whichever gradients are asked for
int64_t residual_work_floats(const ResArgs& a);
hipError_t launch_residual_backward(const ResArgs& a, hipStream_t s);

// y = res + keep x scale over `groups` groups of K elements, one draw a group.
hipError_t launch_dropout(const void* x, const void* res, bool bf16, uint32_t threshold, float scale,
                          const uint64_t* rng, int64_t groups, int64_t K, void* y, hipStream_t s);

}  // namespace gtp
