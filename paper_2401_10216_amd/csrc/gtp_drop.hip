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

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = float4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<float4*>(p + 4) = float4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  bf16x8 o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = static_cast<__bf16>(v[j]);
  *reinterpret_cast<bf16x8*>(p) = o;
}

constexpr int kThreads = 256, kIters = 4, kTile = kThreads * 8 * kIters;

// What bounds it is HBM: a draw costs an eighth of a call of the generator (ten
// rounds of two 32-bit products, most of the work), made once: a workgroup takes
// 8192 elements, its threads first make the calls for the groups that these fall
// into, a call each, and leave a byte of kept-or-not bits in LDS; then each thread
// walks its elements, 8 at a time, 16 bytes an access where the addresses allow.
// 32768 x 128 channels of 49 bf16: 146 us, 5.6 TB/s (the chip's best copy: 5.5); a
// call for every element, as the first version made, took 493.
template <typename T, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_dropout(const T* x, const T* res, uint32_t threshold, float scale,
                                                      const uint64_t* __restrict__ rng, int64_t n, int K,
                                                      uint32_t inv_k, T* y) {
  __shared__ __align__(4) uint8_t bits[kTile / 8 + 8];
  lds_poison(reinterpret_cast<float*>(bits), kTile / 32 + 2);
  const int64_t e0 = int64_t(blockIdx.x) * kTile;
  const int64_t g0 = e0 / K;              // the tile's first group
  const int k0 = int(e0 - g0 * K);        // and the first element's place in it
  const int count = int(n - e0 < kTile ? n - e0 : kTile);
  // local / K for local < kTile + K: with inv_k = floor(2^32 / K) + 1 exact while local K < 2^32; a group as long as a
  // tile or longer can end but once in it
  auto group_of = [&](int64_t local) {
    if (K >= kTile) return local >= K ? 1 : 0;
    return K == 1 ? int(local) : int(__umulhi(uint32_t(local), inv_k));
  };
  const int64_t c0 = g0 >> 3;
  const int calls = int(((g0 + group_of(int64_t(k0) + count - 1)) >> 3) - c0) + 1;
  for (int i = threadIdx.x; i < calls; i += kThreads) {
    uint32_t w[4];
    philox(uint64_t(c0 + i), rng[0], rng[1], w);
    uint32_t b = 0;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      b |= ((w[h] & 0xffffu) >= threshold ? 1u : 0u) << (2 * h);
      b |= ((w[h] >> 16) >= threshold ? 1u : 0u) << (2 * h + 1);
    }
    bits[i] = uint8_t(b);
  }
  if (int(threadIdx.x) == 0) bits[calls] = 0;  // read beside the last call's, never used
  __syncthreads();
  const int gshift = int(g0 & 7);
#pragma unroll
  for (int it = 0; it < kIters; ++it) {
    const int local = (it * kThreads + int(threadIdx.x)) * 8;
    if (local >= count) return;
    const int gl = group_of(int64_t(k0) + local);
    int k = int(int64_t(k0) + local - int64_t(gl) * K);
    const int bit = gl + gshift;
    // the bits of this group and the next eight
    uint32_t keep = (uint32_t(bits[bit >> 3]) | uint32_t(bits[(bit >> 3) + 1]) << 8) >> (bit & 7);
    float v[8], r[8];
    const bool whole = local + 8 <= count;
    if (WIDE && whole) {
      load8(x + e0 + local, v);
      if (res) load8(res + e0 + local, r);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = local + j < count;
        v[j] = in ? ld(x, e0 + local + j) : 0.0f;
        r[j] = in && res ? ld(res, e0 + local + j) : 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = keep & 1u ? v[j] * scale : 0.0f;
      if (res) v[j] += r[j];
      if (++k == K) {
        k = 0;
        keep >>= 1;
      }
    }
    if (WIDE && whole) {
      store8(y + e0 + local, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (local + j < count) st(y, e0 + local + j, v[j]);
    }
  }
}

template <typename T>
hipError_t launch(const void* x, const void* res, uint32_t threshold, float scale, const uint64_t* rng, int64_t n,
                  int64_t K, void* y, hipStream_t s) {
  const uint32_t inv_k = uint32_t((uint64_t(1) << 32) / uint64_t(K)) + 1;
  const bool wide = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(res) | reinterpret_cast<uintptr_t>(y)) & 15) == 0;
  const auto k = wide ? k_dropout<T, true> : k_dropout<T, false>;
  k<<<uint32_t((n + kTile - 1) / kTile), kThreads, 0, s>>>(static_cast<const T*>(x), static_cast<const T*>(res), threshold,
                                                           scale, rng, n, int(K), inv_k, static_cast<T*>(y));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const void* x, const void* res, bool bf16, uint32_t threshold, float scale,
                          const uint64_t* rng, int64_t groups, int64_t K, void* y, hipStream_t s) {
  const int64_t n = groups * K;
  return bf16 ? launch<uint16_t>(x, res, threshold, scale, rng, n, K, y, s)
              : launch<float>(x, res, threshold, scale, rng, n, K, y, s);
}

}  // namespace gtp
