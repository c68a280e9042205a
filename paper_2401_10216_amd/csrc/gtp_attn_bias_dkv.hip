// The gradients of keys and values with a bias by distance.
#include "gtp_attn_dkv.hpp"

namespace gtp {

void launch_attn_dkv_bias(const AttnArgs& a, hipStream_t s) { launch_dkv_kernel<kBias>(a, s); }

}  // namespace gtp
