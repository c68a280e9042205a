// The attention's forward with a bias by distance whose buckets are made ahead.
#include "gtp_attn_fwd.hpp"

namespace gtp {

void launch_attn_fwd_bytes(const AttnArgs& a, hipStream_t s) { launch_fwd_kernel<kBiasBytes>(a, s); }

}  // namespace gtp
