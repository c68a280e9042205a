// The gradient of the queries with a bias by distance whose buckets are made ahead.
#include "gtp_attn_dq.hpp"

namespace gtp {

void launch_attn_dq_bytes(const AttnArgs& a, hipStream_t s) { launch_dq_kernel<kBiasBytes>(a, s); }

}  // namespace gtp
