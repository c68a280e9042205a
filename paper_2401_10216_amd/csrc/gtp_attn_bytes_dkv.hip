// The gradients of keys and values with a bias by distance whose buckets are made ahead.
#include "gtp_attn_dkv.hpp"

namespace gtp {

void launch_attn_dkv_bytes(const AttnArgs& a, hipStream_t s) { launch_dkv_kernel<kBiasBytes>(a, s); }

}  // namespace gtp
