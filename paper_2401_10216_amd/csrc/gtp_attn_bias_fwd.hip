// The attention's forward with a bias by distance.
#include "gtp_attn_fwd.hpp"

namespace gtp {

void launch_attn_fwd_bias(const AttnArgs& a, hipStream_t s) { launch_fwd_kernel<kBias>(a, s); }

}  // namespace gtp
