// The gradients of keys and values without a bias (gtp_attn_dkv.hpp).
#include "gtp_attn_dkv.hpp"

namespace gtp {

hipError_t launch_attn_dkv(const AttnArgs& a, hipStream_t s) {
  if (a.bytes_k)
    launch_attn_dkv_bytes(a, s);
  else if (a.bias)
    launch_attn_dkv_bias(a, s);
  else
    launch_dkv_kernel<kNoBias>(a, s);
  return hipGetLastError();
}

}  // namespace gtp
