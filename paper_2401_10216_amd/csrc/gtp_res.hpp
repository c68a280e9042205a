// The residual step between two parts of a block (gtp_res_*.hip): what its kernels share.
//
//   t = post ? xh1 w1 + b1 d_l0 : a,  xh1 = (a - mu1 d_l0) r1_l,
//   r = x + s[l, c] sig(gate[c]) t,  h = xh2 w2 + b2 d_l0,  xh2 = (r - mu2 d_l0) r2_l,
// mu and r_l the mean and 1 / size of a degree of a row, as in gtp_norm.hip; sig(v) =
// 1 / (1 + e^-v).  Gradient for dh and dr, with g2 = dh w2:
//   D = dr + r2_l (g2 - xh2 mean(g2 xh2) - d_l0 mean g2)      (dx = D),
//   g1 = D sig s w1,  da = r1_l (g1 - xh1 mean(g1 xh1) - d_l0 mean g1)   (post; else D sig s),
//   dgate[c] = sig (1 - sig) sum_{l,m} D s t,
// and from four sums over the rows (and m), E1 = sum D sig xh1 (xh1 = a without post), E2 = sum
// dh xh2, F = sum D sig and G = sum dh at degree 0:
//   dw1 = s E1,  db1 = s_0 F,  ds = w1 E1 + b1 F d_l0,  dw2 = E2,  db2 = G.
// Degrees share nothing but the gate.
#pragma once

#include "gtp_layers.hpp"

namespace gtp {

// The weights of a row's degree l, channel c, ones and zeros where there are none.
struct ResWeights {
  const float *scale, *w1, *b1, *w2, *b2;
  int64_t C;
  bool post;
  __host__ explicit ResWeights(const ResArgs& a)
      : scale(a.scale), w1(a.post ? a.w1 : nullptr), b1(a.post ? a.b1 : nullptr), w2(a.w2), b2(a.b2), C(a.C), post(a.post) {}
  __device__ float s(int l, int64_t c) const { return scale ? scale[l * C + c] : 1.0f; }
  __device__ float post_w(int l, int64_t c) const { return w1 ? w1[l * C + c] : 1.0f; }
  __device__ float post_b(int l, int64_t c) const { return l == 0 && b1 ? b1[c] : 0.0f; }
  __device__ float pre_w(int l, int64_t c) const { return w2 ? w2[l * C + c] : 1.0f; }
  __device__ float pre_b(int l, int64_t c) const { return l == 0 && b2 ? b2[c] : 0.0f; }
};

// 1 / (1 + e^-v): 0 and 1 at the infinities, e^-v may overflow.
__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }

// Columns of a part of the weight sums: E1 and E2 [L + 1, C], F and G [C].
__host__ __device__ inline int64_t res_columns(int L, int64_t C) { return 2 * int64_t(L + 2) * C; }

// Adds `parts` parts of the weight sums, in order, and makes the weights' gradients.
hipError_t launch_residual_sum(const ResArgs& a, const float* partial, int64_t parts, hipStream_t s);

// Rows too long for the registers (gtp_res_long.hip), where residual_is_long says so.
bool residual_is_long(const ResArgs& a);
hipError_t launch_residual_long(const ResArgs& a, hipStream_t s);
int64_t residual_long_floats(const ResArgs& a);
hipError_t launch_residual_long_backward(const ResArgs& a, hipStream_t s);

// Rows of any length (gtp_res_any.hip).
hipError_t launch_residual_any(const ResArgs& a, hipStream_t s);
int64_t residual_any_floats(const ResArgs& a);
hipError_t launch_residual_any_backward(const ResArgs& a, hipStream_t s);

}  // namespace gtp
