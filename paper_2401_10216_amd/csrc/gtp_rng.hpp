// Counter-based random bits for dropout.
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", SC 2011): 128 bits from a 128-bit counter and a 64-bit key, by
// ten rounds of two 32 x 32 -> 64 bit products.  A call's counter is (index,
// offset) and its key the seed, low words first, so any element's draw can be
// made again from its index alone and no mask is ever stored.  A draw is 16
// bits of a call (its halfword h: the low, then the high half of word h / 2):
// eight draws a call; an element is kept where its draw is at least the
// threshold round(65536 p).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace gtp {

__host__ __device__ __forceinline__ void philox(uint64_t index, uint64_t seed, uint64_t offset, uint32_t (&out)[4]) {
  uint32_t c0 = uint32_t(index), c1 = uint32_t(index >> 32), c2 = uint32_t(offset), c3 = uint32_t(offset >> 32);
  uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
    c0 = uint32_t(b >> 32) ^ c1 ^ k0;
    c1 = uint32_t(b);
    c2 = uint32_t(a >> 32) ^ c3 ^ k1;
    c3 = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  out[0] = c0;
  out[1] = c1;
  out[2] = c2;
  out[3] = c3;
}

// Threshold of the 16-bit draws for dropping with probability p in [0, 1), and
// the factor 1 / (1 - p) of what is kept, at the p that the threshold stands for.
inline uint32_t drop_threshold(double p) {
  const double t = p * 65536.0 + 0.5;
  return t >= 65535.0 ? 65535u : uint32_t(t);
}
inline float drop_scale(uint32_t threshold) { return float(65536.0 / (65536.0 - double(threshold))); }

}  // namespace gtp
