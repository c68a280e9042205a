// The gradient of the queries without a bias (gtp_attn_dq.hpp), and the rows' sums of dout o.
#include "gtp_attn_dq.hpp"

namespace gtp {
namespace {

// delta[t, h] = sum_i dout[t, h, i] o[t, h, i]: 16 lanes a row.  In a
// pass of its own, once for both gradients: dout and o read once, HBM's time for the long
// cases and a launch's (4 us) for the short.
constexpr uint32_t kDeltaGrid = 1u << 20;  // workgroups at most: a launch holds less than 2^32 threads
template <typename T>
__global__ __launch_bounds__(256) void k_attn_delta(const AttnArgs a) {
  const int64_t n = a.Tq * a.H;
  const int i0 = threadIdx.x & 15;
  for (int64_t id = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); id < n; id += int64_t(gridDim.x) * 16) {
    const int64_t t = id / a.H, h = id % a.H;
    const T* o = static_cast<const T*>(a.o.p) + t * a.o.row + h * a.o.head;
    const T* g = static_cast<const T*>(a.dout.p) + t * a.dout.row + h * a.dout.head;
    float s = 0.0f;
    for (int i = i0; i < a.d; i += 16) s = fmaf(to_f32<T>(o[i]), to_f32<T>(g[i]), s);
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) s += __shfl_xor(s, x);  // a row's lanes are in the loop together
    if (i0 == 0) a.delta[id] = s;
  }
}

}  // namespace

hipError_t launch_attn_delta(const AttnArgs& a, hipStream_t s) {
  const int64_t all = (a.Tq * a.H + 15) / 16;
  const uint32_t n = all < kDeltaGrid ? uint32_t(all) : kDeltaGrid;
  if (a.bf16)
    k_attn_delta<uint16_t><<<n, 256, 0, s>>>(a);
  else
    k_attn_delta<float><<<n, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_attn_dq(const AttnArgs& a, hipStream_t s) {
  if (a.bytes)
    launch_attn_dq_bytes(a, s);
  else if (a.bias)
    launch_attn_dq_bias(a, s);
  else
    launch_dq_kernel<kNoBias>(a, s);
  return hipGetLastError();
}

}  // namespace gtp
