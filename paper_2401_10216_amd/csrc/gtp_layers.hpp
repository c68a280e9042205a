// Launchers of the layers around the product: normalisation of SH features
// (gtp_norm.hip), dropout (gtp_drop.hip).  Arguments are validated by the C
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

// y = res + keep x scale over `groups` groups of K elements, one draw a group.
hipError_t launch_dropout(const void* x, const void* res, bool bf16, uint32_t threshold, float scale,
                          const uint64_t* rng, int64_t groups, int64_t K, void* y, hipStream_t s);

}  // namespace gtp
