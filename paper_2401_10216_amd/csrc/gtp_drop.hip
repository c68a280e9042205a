// Dropout whose mask is never stored: y = res + keep x / (1 - p), the draw of
// group g (K consecutive elements: all coefficients of one channel, so that a
// channel is dropped whole and y turns with x) taken from the generator at
// index g / 8, halfword g mod 8.  The gradient is the same map of dy.
#include "gtp_device.hpp"
#include "gtp_layers.hpp"
#include "gtp_rng.hpp"

namespace gtp {
namespace {

__device__ __forceinline__ float ld(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float ld(const uint16_t* p, int64_t i) { return __uint_as_float(uint32_t(p[i]) << 16); }
__device__ __forceinline__ void st(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st(uint16_t* p, int64_t i, float v) {
  const __bf16 h = static_cast<__bf16>(v);  // to nearest, ties to even
  p[i] = __builtin_bit_cast(uint16_t, h);
}

template <typename T>
__global__ __launch_bounds__(256) void k_dropout(const T* x, const T* res, uint32_t threshold, float scale,
                                                 const uint64_t* __restrict__ rng, int64_t n, int64_t K, T* y) {
  const uint64_t seed = rng[0], offset = rng[1];
  for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < n; e += int64_t(gridDim.x) * 256) {
    const int64_t g = e / K;
    uint32_t bits[4];
    philox(uint64_t(g) >> 3, seed, offset, bits);
    const uint32_t wd = (g & 4) ? ((g & 2) ? bits[3] : bits[2]) : ((g & 2) ? bits[1] : bits[0]);
    const uint32_t draw = (g & 1) ? wd >> 16 : wd & 0xffffu;
    const float v = draw >= threshold ? ld(x, e) * scale : 0.0f;
    st(y, e, res ? v + ld(res, e) : v);
  }
}

}  // namespace

hipError_t launch_dropout(const void* x, const void* res, bool bf16, uint32_t threshold, float scale,
                          const uint64_t* rng, int64_t groups, int64_t K, void* y, hipStream_t s) {
  const int64_t n = groups * K;
  const int64_t blocks = (n + 255) / 256;
  const dim3 grid{uint32_t(blocks < 65536 ? blocks : 65536)};
  if (bf16)
    k_dropout<<<grid, 256, 0, s>>>(static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(res), threshold, scale,
                                   rng, n, K, static_cast<uint16_t*>(y));
  else
    k_dropout<<<grid, 256, 0, s>>>(static_cast<const float*>(x), static_cast<const float*>(res), threshold, scale, rng,
                                   n, K, static_cast<float*>(y));
  return hipGetLastError();
}

}  // namespace gtp
