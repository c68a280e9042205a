// What the normalisation (gtp_norm.hip) and the residual step (gtp_res_*.hip) share:
// a row of SH features [C, K] on the threads of a wave or workgroup, its loads and
// stores whatever its alignment, and sums by degree.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "gtp_device.hpp"

namespace gtp {

__device__ __forceinline__ float ld(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float ld(const uint16_t* p, int64_t i) { return __uint_as_float(uint32_t(p[i]) << 16); }
__device__ __forceinline__ void st(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st(uint16_t* p, int64_t i, float v) {
  const __bf16 h = static_cast<__bf16>(v);  // to nearest, ties to even
  p[i] = __builtin_bit_cast(uint16_t, h);
}

template <typename T, int V>
struct Vec {
  typedef T type __attribute__((ext_vector_type(V)));
};
template <typename T>
struct Vec<T, 1> {
  typedef T type;
};

template <typename T, int V>
__device__ __forceinline__ typename Vec<T, V>::type ldv(const T* p, int64_t i) {
  return *reinterpret_cast<const typename Vec<T, V>::type*>(p + i);
}
template <typename T, int V>
__device__ __forceinline__ float get(const typename Vec<T, V>::type& v, int j) {
  T e;
  if constexpr (V == 1)
    e = v;
  else
    e = v[j];
  if constexpr (sizeof(T) == 4)
    return e;
  else
    return __uint_as_float(uint32_t(e) << 16);
}
template <typename T>
__device__ __forceinline__ T narrow(float f) {
  if constexpr (sizeof(T) == 4) {
    return f;
  } else {
    const __bf16 h = static_cast<__bf16>(f);  // to nearest, ties to even
    return __builtin_bit_cast(uint16_t, h);
  }
}
template <typename T, int V>
__device__ __forceinline__ void stv(T* p, int64_t i, const float (&f)[V]) {
  typename Vec<T, V>::type v;
  if constexpr (V == 1) {
    v = narrow<T>(f[0]);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = narrow<T>(f[j]);
  }
  *reinterpret_cast<typename Vec<T, V>::type*>(p + i) = v;
}

// Sum over aligned groups of W lanes, on the data-parallel paths of the VALU (the
// shuffles through LDS took longer than a short row's arithmetic: 65536 rows of
// 256 in 37 us, 19 without any sum); every lane of the group gets it.
template <int W>
__device__ __forceinline__ float lane_sum(float v) {
  auto add = [&](auto ctrl) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if constexpr (W >= 2) add(std::integral_constant<int, 0xb1>{});   // quad_perm 1 0 3 2
  if constexpr (W >= 4) add(std::integral_constant<int, 0x4e>{});   // quad_perm 2 3 0 1
  if constexpr (W >= 8) add(std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (W >= 16) add(std::integral_constant<int, 0x140>{}); // row_mirror
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (W >= 32) {
    const u32x2 p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  if constexpr (W >= 64) {
    const u32x2 p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  return v;
}
__device__ __forceinline__ float wave_sum(float v) { return lane_sum<64>(v); }

// Hides from the compiler that v is what it was: what was computed from it before
// is computed again rather than kept (the rows' 16-bit elements widened to 32 bits
// and normalised would take two to four times the registers of the rows).
template <typename X>
__device__ __forceinline__ void renew(X& v) {
  if constexpr (sizeof(X) == 16) {
    asm volatile("" : "+v"(v));
  } else if constexpr (sizeof(X) == 8) {
    uint64_t u = __builtin_bit_cast(uint64_t, v);
    asm volatile("" : "+v"(u));
    v = __builtin_bit_cast(X, u);
  }
}

// Hides a workgroup-wide number's value: addresses made from it are made again
// rather than kept in registers, one for each element, across the rows.
__device__ __forceinline__ int renewed(int v) {
  v = __builtin_amdgcn_readfirstlane(v);
  asm volatile("" : "+s"(v));
  return v;
}

// What a thread's places hold.  Thread t < A takes, V at a time, the elements V t + i A V
// of its row, i = 0, 1, ..., with A V a multiple of K: so each of its V places always holds
// the same coefficient k, and a step i moves every place on by A V / K channels.
template <int V>
struct Places {
  int deg[V], at[V];  // degree; where in the weights' LDS copy its weight of step 0 is
  int j0, ch;         // the place of a degree-0 coefficient, -1 = none (K > 1: at most one), and its channel at step 0
  int cpc;            // channels a step moves on by
  bool on;
  __device__ __forceinline__ Places(int A, int K, int C, int t) {
    on = t < A;
    cpc = A * V / K;
    j0 = -1;
    ch = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int pos = (on ? V * t : 0) + j, c = pos / K, k = pos - c * K;
      deg[j] = degree_of(k);
      at[j] = deg[j] * (C | 1) + c;
      if (k == 0) j0 = j, ch = c;
    }
  }
};

// Elements at .. at + V - 1 of a row of R >= V, whatever its alignment (16-byte
// accesses to element-aligned memory), zeros past its end.  The load is
// unconditional, from the row's last V elements where it would leave the row, and
// step_fix moves what came into place: a branch around each load made every one
// wait for the one before it.
template <typename T, int V>
__device__ __forceinline__ typename Vec<T, V>::type step_load(const T* row, int at, int R) {
  typename Vec<T, V>::type v;
  __builtin_memcpy(&v, row + (at < R - V ? at : R - V), sizeof(v));
  return v;
}
// EVEN: R is a multiple of V, so that a group is in the row or past its end as a whole.
template <bool EVEN, typename T, int V>
__device__ __forceinline__ void step_fix(typename Vec<T, V>::type& v, int at, int R) {
  if constexpr (EVEN) {
    v = at < R ? v : typename Vec<T, V>::type{};
    return;
  }
  const int shift = at - (R - V);
  if (shift > 0) {
    typename Vec<T, V>::type u = {};
#pragma unroll
    for (int s = 1; s < V; ++s)
      if (shift == s)
#pragma unroll
        for (int j = 0; j + s < V; ++j) u[j] = v[j + s];
    v = u;
  }
}
template <bool EVEN, typename T, int V>
__device__ __forceinline__ void step_store(T* row, int at, int R, const float (&o)[V]) {
  if (at <= R - V) {
    typename Vec<T, V>::type v;
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = narrow<T>(o[j]);
    __builtin_memcpy(row + at, &v, sizeof(v));
  } else if constexpr (!EVEN) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (at + j < R) row[at + j] = narrow<T>(o[j]);
  }
}

// Sums of the places' values by degree: red[pos] holds place pos's value (the
// barrier behind the writes is the caller's).  Wave v takes degrees v, v + waves, ...
template <typename F>
__device__ __forceinline__ void by_degree(const float* red, int K, int cpc, int L, int l_first, F done) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int l = wave; l <= L; l += waves) {
    if (l < l_first) continue;
    float s = 0.0f, u = 0.0f;
    for (int c = lane; c < cpc; c += 64) {
      const float* p = red + c * K + l * l;
      s += p[0];
#pragma unroll 4
      for (int m = 1; m <= l; ++m) {  // two chains
        s += p[2 * m - 1];
        u += p[2 * m];
      }
    }
    done(l, wave_sum(s + u));
  }
}

// Elements of a row of R that thread t takes, V at a time, the steps AV apart.
__device__ __forceinline__ int elements_of(int R, int V, int AV, int t) {
  const int full = R / AV, rest = R - full * AV - V * t;
  return full * V + (rest < 0 ? 0 : rest < V ? rest : V);
}

}  // namespace gtp
