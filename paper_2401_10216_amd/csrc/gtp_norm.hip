// Normalisation of SH features, degree by degree, and its gradient.
//
// x[n, c, (l, m)] of a row n: with v_l = mean over (c, m) of (x - mu d_l0)^2 and
// mu = mean_c x[c, 0],
//   y = (x - mu d_l0) r_l w[l, c] + b[c] d_l0,   r_l = 1 / sqrt(v_l + eps).
// A rotation mixes the m of a degree and leaves v_l and mu alone, so y turns
// with x; L = 0 is the ordinary layer norm over the channels.  Gradient, with
// xh = (x - mu d_l0) r_l and g = dy w:
//   dx = r_l (g - xh mean_{c,m}(g xh) - d_l0 mean_c g),
//   dw[l, c] = sum_{n,m} dy xh,   db[c] = sum_n dy[c, 0].
// All sums in fp32.
//
// HBM bounds both directions: x (and dy) read once, y (dx) written once, a row
// kept in registers between its sums and its results.  A workgroup takes a row at a
// time, 1 to 16 waves by its length; the sums of a degree go through LDS.  Measured:
// 16384 x 128 channels of degree 6, fp32, 156-164 us forward (5.0-5.3 TB/s; the chip's
// best copy 5.5) and 245-263 backward; 65536 rows of 256, 20 and 31 us.
//
// Degree 16 with 64 channels (18496 elements a row, bf16, 8192 rows) runs at 200 us
// forward (3.0 TB/s) and 440-465 backward (2.0): one workgroup a CU cannot load a row
// while it sums another.  Registers allow no second one forward (ten waves of 126); the
// backward's sums of dw by element, 83 of its 103 KB of LDS, do not either, and it keeps
// 56 bytes a lane in scratch memory.  Rows of more than some 24500 elements (forward:
// 32768) do not stay in registers: 4096 rows of degree 16 with 128 channels, as many
// bytes, take 288 us forward and 492 backward (dx 329, a kernel of its own for dw 159).
// Degrees share no sum, so a row could be dealt to workgroups by degrees.
#include <algorithm>
#include <type_traits>

#include "gtp_device.hpp"
#include "gtp_layers.hpp"

namespace gtp {
namespace {

__device__ __forceinline__ float ld(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float ld(const uint16_t* p, int64_t i) { return __uint_as_float(uint32_t(p[i]) << 16); }
__device__ __forceinline__ void st(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st(uint16_t* p, int64_t i, float v) {
  const __bf16 h = static_cast<__bf16>(v);  // to nearest, ties to even
  p[i] = __builtin_bit_cast(uint16_t, h);
}

// A row's elements on the threads.  Thread t < A takes, V at a time, the elements
// V t + i A V of its row, i = 0, 1, ..., with A V a multiple of K: so each of its V
// places always holds the same coefficient k (one degree, one accumulator), and a
// step i moves every place on by A V / K channels.
struct Lay {
  int A, threads, NI;   // NI: steps that a row takes
  int V, steps_reg;     // steps_reg: the instantiation that holds them in registers, 0 = none does
};

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

// What a thread's places hold.
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

// The weights in LDS, a degree's row of C in C | 1 (an odd stride: places of
// several degrees and one channel read different banks), behind them the shifts;
// ones and zeros where there are none, so that every element does the same.  In
// registers, one for each element, they halved the rows in flight; from the cache
// they cost a load an element.
__device__ __forceinline__ void load_weights(const float* w, const float* b, int C, int L, float* tw) {
  for (int l = 0; l <= L; ++l)
    for (int c = threadIdx.x; c < C; c += int(blockDim.x)) tw[l * (C | 1) + c] = w ? w[int64_t(l) * C + c] : 1.0f;
  for (int c = threadIdx.x; c < C; c += int(blockDim.x)) tw[(L + 1) * (C | 1) + c] = b ? b[c] : 0.0f;
}

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

// Forward.  NI > 0: a row of NI steps stays in registers between its sums and its
// results (one read); NI = 0: longer rows, read again for the squares at degree 0 about
// a thread's mean and for the results.  Degree 0 is summed about
// each thread's own mean, the threads' means and sums then joined, so a mean far
// from zero costs no digits.
template <typename T, int V, int NI, bool K1, bool EVEN>
__global__ __launch_bounds__(1024) void k_norm(const T* x, const float* __restrict__ w, const float* __restrict__ b,
                                               float eps, int64_t N, int C, int L, int A, T* y,
                                               float* __restrict__ mean, float* __restrict__ rstd) {
  // [A V] squares (K1: [A]), [A V / K] (K1: [A]) sums, [L + 2] the row's statistics, then load_weights's and room for
  // a row's last step
  extern __shared__ float lds[];
  const int K = (L + 1) * (L + 1), t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const Places<V> pl(A, K, C, t);
  const int slots = K1 ? A : pl.cpc, squares = K1 ? A : A * V;
  float* const red = lds;
  float* const sums = lds + squares;
  float* const stat = sums + slots;
  float* const tw = stat + L + 2;
  const int R = C * K, AV = A * V, steps = NI > 0 ? NI : (R + AV - 1) / AV;
  lds_poison(lds, squares + slots + L + 2 + (L + 2) * (C | 1) + steps * pl.cpc);
  load_weights(w, b, C, L, tw);
  const float* const tb = tw + (L + 1) * (C | 1);
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const T* const xr = x + n * R;
    T* const yr = y + n * R;
    typedef typename Vec<T, V>::type Row;
    Row xv[NI > 0 ? NI : 1];
    // f(i, place of the step's first element, the elements)
    auto each = [&](auto f) {
      if constexpr (NI > 0) {
#pragma unroll
        for (int i = 0; i < NI; ++i) f(i, i * AV + V * t, xv[i]);
      } else {
        for (int i0 = 0; i0 < steps; i0 += 4) {  // four steps' loads at a time
          Row v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = step_load<T, V>(xr, (i0 + i) * AV + V * t, R);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            step_fix<EVEN, T, V>(v[i], (i0 + i) * AV + V * t, R);
            if (i0 + i < steps) f(i0 + i, (i0 + i) * AV + V * t, v[i]);
          }
        }
      }
    };
    if (pl.on) {
      if constexpr (NI > 0) {
#pragma unroll
        for (int i = 0; i < NI; ++i) xv[i] = step_load<T, V>(xr, i * AV + V * t, R);
#pragma unroll
        for (int i = 0; i < NI; ++i) step_fix<EVEN, T, V>(xv[i], i * AV + V * t, R);
      }
      float s2[V], s1 = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) s2[j] = 0.0f;
      each([&](int, int, const Row& v) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float f = get<T, V>(v, j);
          if constexpr (K1) {
            s1 += f;
          } else {
            const bool zero = j == pl.j0;
            s1 += zero ? f : 0.0f;
            s2[j] = fmaf(zero ? 0.0f : f, f, s2[j]);
          }
        }
      });
      // about the thread's own mean at degree 0
      const int mine = K1 ? elements_of(R, V, AV, t) : (C - pl.ch + pl.cpc - 1) / pl.cpc;
      const float own = mine > 0 ? s1 / float(mine) : 0.0f;
      if constexpr (K1) {
        each([&](int, int at, const Row& v) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float f = (EVEN ? at : at + j) < R ? get<T, V>(v, j) - own : 0.0f;
            s2[0] = fmaf(f, f, s2[0]);
          }
        });
        sums[t] = s1;
        red[t] = s2[0];
      } else {
        float q = 0.0f;
        if (pl.j0 >= 0)
          each([&](int, int at, const Row& v) {
            float f = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) f = j == pl.j0 ? get<T, V>(v, j) : f;
            f = (EVEN ? at : at + pl.j0) < R ? f - own : 0.0f;
            q = fmaf(f, f, q);
          });
#pragma unroll
        for (int j = 0; j < V; ++j) red[V * t + j] = j == pl.j0 ? q : s2[j];
        if (pl.j0 >= 0) sums[pl.ch] = s1;
      }
    }
    __syncthreads();
    if (wave == 0) {
      // slot c holds the elements of nc channels (K1: of a thread)
      float s = 0.0f;
      for (int c = lane; c < slots; c += 64) s += sums[c];
      const float mu = wave_sum(s) / float(C);
      float q = 0.0f;
      for (int c = lane; c < slots; c += 64) {
        const int nc = K1 ? elements_of(R, V, AV, c) : (C - c + pl.cpc - 1) / pl.cpc;  // 0 past the last
        if (nc > 0) {
          const float d = sums[c] / float(nc) - mu;
          q += red[K1 ? c : c * K] + float(nc) * d * d;
        }
      }
      const float r = 1.0f / sqrtf(wave_sum(q) / float(C) + eps);
      if (lane == 0) {
        stat[0] = r;
        stat[L + 1] = mu;
        if (mean) mean[n] = mu;
        if (rstd) rstd[n * (L + 1)] = r;
      }
    }
    if constexpr (!K1)
      by_degree(red, K, pl.cpc, L, 1, [&](int l, float s) {
        const float r = 1.0f / sqrtf(s / (float(C) * float(2 * l + 1)) + eps);
        if (lane == 0) {
          stat[l] = r;
          if (rstd) rstd[n * (L + 1) + l] = r;
        }
      });
    __syncthreads();
    if (!pl.on) continue;
    if constexpr (NI > 0)
#pragma unroll
      for (int i = 0; i < NI; ++i) renew(xv[i]);
    const int cpc = renewed(pl.cpc);
    const float mu = stat[L + 1];
    float r[V];
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = stat[K1 ? 0 : pl.deg[j]];
    each([&](int i, int at, const Row& v) {
      float o[V];
      const float shift = K1 ? 0.0f : tb[pl.ch + i * cpc];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float wv = tw[pl.at[j] + i * cpc];
        if constexpr (K1)
          o[j] = fmaf((get<T, V>(v, j) - mu) * r[j], wv, tb[pl.at[j] + i * cpc]);
        else
          o[j] = fmaf((get<T, V>(v, j) - (j == pl.j0 ? mu : 0.0f)) * r[j], wv, j == pl.j0 ? shift : 0.0f);
      }
      step_store<EVEN, T, V>(yr, at, R, o);
    });
  }
}

// Backward: dx and, over all rows that the workgroup takes, its part of dw and db:
// each thread adds to its own elements' sums in LDS (8 bytes of LDS traffic an
// element beside 6..12 of HBM, at a twelfth of the time), and at the end a
// channel's coefficients are added up by degree.  partial[workgroup][(L + 2) C]: L + 1
// rows of dw, then db.  NI = 0 (rows too long for that): dx alone.
template <typename T, int V, int NI, bool K1, bool EVEN, int MAXT>
__global__ __launch_bounds__(MAXT) void k_norm_backward(const T* __restrict__ x, const T* dy,
                                                        const float* __restrict__ w, const float* __restrict__ mean,
                                                        const float* __restrict__ rstd, int64_t N, int C, int L, int A,
                                                        T* dx, float* __restrict__ partial) {
  // [NI A V] dw by element, [NI A V / K] db by channel, then [A V] (K1: [A]) sums of
  // g xh, [A V / K] (K1: [A]) of g, [L + 2] the row's means, load_weights's and room for a row's last step
  extern __shared__ __align__(16) float lds[];
  const int K = (L + 1) * (L + 1), t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const Places<V> pl(A, K, C, t);
  const int slots = K1 ? A : pl.cpc, nred = K1 ? A : A * V;
  float* const aw = lds;
  float* const ab = aw + NI * A * V;
  float* const red = ab + NI * pl.cpc;
  float* const sums = red + nred;
  float* const stat = sums + slots;
  float* const tw = stat + L + 2;
  const int R = C * K, AV = A * V, steps = NI > 0 ? NI : (R + AV - 1) / AV;
  lds_poison(lds, NI * AV + NI * pl.cpc + nred + slots + L + 2 + (L + 2) * (C | 1) + steps * pl.cpc);
  load_weights(w, nullptr, C, L, tw);
  typedef typename Vec<T, V>::type Row;
  typedef typename Vec<float, V>::type Sums;
  if constexpr (NI > 0) {
    if (pl.on)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          aw[i * AV + V * t + j] = 0.0f;
          if (K1 || j == pl.j0) ab[i * pl.cpc + (K1 ? V * t + j : pl.ch)] = 0.0f;
        }
  }
  __syncthreads();
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const T* const xr = x + n * R;
    const T* const gr = dy + n * R;
    Row xv[NI > 0 ? NI : 1], gv[NI > 0 ? NI : 1];
    auto each = [&](auto f) {
      if constexpr (NI > 0) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          f(i, i * AV + V * t, xv[i], gv[i]);
          __builtin_amdgcn_sched_barrier(0);  // a step's LDS reads with the step: all at once they spill
        }
      } else {
        for (int i0 = 0; i0 < steps; i0 += 4) {  // four steps' loads at a time
          Row v[4], g[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = step_load<T, V>(xr, (i0 + i) * AV + V * t, R);
            g[i] = step_load<T, V>(gr, (i0 + i) * AV + V * t, R);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            step_fix<EVEN, T, V>(v[i], (i0 + i) * AV + V * t, R);
            step_fix<EVEN, T, V>(g[i], (i0 + i) * AV + V * t, R);
            if (i0 + i < steps) f(i0 + i, (i0 + i) * AV + V * t, v[i], g[i]);
          }
        }
      }
    };
    float mu = 0.0f, r[V];
    auto xhat = [&](const Row& v, int j) { return (get<T, V>(v, j) - (K1 || j == pl.j0 ? mu : 0.0f)) * r[j]; };
    if (pl.on) {
      if constexpr (NI > 0) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          xv[i] = step_load<T, V>(xr, i * AV + V * t, R);
          gv[i] = step_load<T, V>(gr, i * AV + V * t, R);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          step_fix<EVEN, T, V>(xv[i], i * AV + V * t, R);
          step_fix<EVEN, T, V>(gv[i], i * AV + V * t, R);
        }
      }
      mu = mean[n];
      const int cpc = renewed(pl.cpc);
#pragma unroll
      for (int j = 0; j < V; ++j) r[j] = rstd[n * (L + 1) + (K1 ? 0 : pl.deg[j])];
      float sx[V], sg = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) sx[j] = 0.0f;
      each([&](int i, int at, const Row& xi, const Row& gi) {  // past the row's end gi is zero, and so is g
        Sums old;
        if constexpr (NI > 0) old = *reinterpret_cast<const Sums*>(aw + i * AV + V * t);
        float d0 = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = get<T, V>(gi, j), xh = xhat(xi, j), g = (EVEN ? at : at + j) < R ? d * tw[pl.at[j] + i * cpc] : 0.0f;
          sx[K1 ? 0 : j] = fmaf(g, xh, sx[K1 ? 0 : j]);
          old[j] = fmaf(d, xh, old[j]);
          sg += K1 || j == pl.j0 ? g : 0.0f;
          if constexpr (K1) {
            if constexpr (NI > 0) ab[i * AV + V * t + j] += d;
          } else {
            d0 = j == pl.j0 ? d : d0;
          }
        }
        if constexpr (NI > 0) {
          *reinterpret_cast<Sums*>(aw + i * AV + V * t) = old;
          if (!K1 && pl.j0 >= 0) ab[i * cpc + pl.ch] += d0;
        }
      });
      if constexpr (K1) {
        red[t] = sx[0];
        sums[t] = sg;
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) red[V * t + j] = sx[j];
        if (pl.j0 >= 0) sums[pl.ch] = sg;
      }
    }
    if (!dx) continue;
    __syncthreads();
    if (wave == 0) {
      float s = 0.0f, q = 0.0f;
      for (int c = lane; c < slots; c += 64) {
        s += sums[c];
        if constexpr (K1) q += red[c];
      }
      s = wave_sum(s);
      if constexpr (K1) q = wave_sum(q);
      if (lane == 0) {
        stat[L + 1] = s / float(C);
        if constexpr (K1) stat[0] = q / float(C);
      }
    }
    if constexpr (!K1)
      by_degree(red, K, pl.cpc, L, 0, [&](int l, float s) {
        if (lane == 0) stat[l] = s / (float(C) * float(2 * l + 1));
      });
    __syncthreads();
    if (!pl.on) continue;
    if constexpr (NI > 0)
#pragma unroll
      for (int i = 0; i < NI; ++i) renew(xv[i]), renew(gv[i]);
    const float mg = stat[L + 1];
    const int cpc = renewed(pl.cpc);
    float mx[V];
#pragma unroll
    for (int j = 0; j < V; ++j) mx[j] = stat[K1 ? 0 : pl.deg[j]];
    T* const out = dx + n * R;
    each([&](int i, int at, const Row& xi, const Row& gi) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j)
        o[j] = r[j] * (get<T, V>(gi, j) * tw[pl.at[j] + i * cpc] - (K1 || j == pl.j0 ? mg : 0.0f) -
                       xhat(xi, j) * mx[j]);
      step_store<EVEN, T, V>(out, at, R, o);
    });
  }
  if constexpr (NI > 0) {
    if (!partial) return;
    float* const out = partial + int64_t(blockIdx.x) * (L + 2) * C;
    __syncthreads();
    for (int q = t; q < (L + 2) * C; q += int(blockDim.x)) {
      const int l = q / C, c = q - l * C;
      float s = 0.0f;
      if (l <= L)
        for (int m = 0; m < 2 * l + 1; ++m) s += aw[c * K + l * l + m];
      else
        s = ab[c];
      out[q] = s;
    }
  }
}

// L = 0 with short rows: W lanes take a row (V NI elements each), its sums never
// leave them; a wave takes 64 / W rows at a time.  Forward: mean, then squares
// about it, then the results.
constexpr int kShortThreads = 256;

template <typename T, int V, int NI, int W>
__global__ __launch_bounds__(kShortThreads) void k_norm_short(const T* x, const float* __restrict__ w,
                                                              const float* __restrict__ b, float eps, int64_t N, int C,
                                                              T* y, float* __restrict__ mean,
                                                              float* __restrict__ rstd) {
  const int sub = threadIdx.x % W;
  float wr[NI][V], br[NI][V];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = V * (sub + i * W) + j;
      wr[i][j] = w && c < C ? w[c] : 1.0f;
      br[i][j] = b && c < C ? b[c] : 0.0f;
    }
  constexpr int ROWS = kShortThreads / W;
  for (int64_t n0 = int64_t(blockIdx.x) * ROWS; n0 < N; n0 += int64_t(gridDim.x) * ROWS) {
    const int64_t n = n0 + threadIdx.x / W;
    const bool there = n < N;
    float f[NI][V];
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const bool in = there && V * (sub + i * W) < C;
      typename Vec<T, V>::type v = {};
      if (in) v = ldv<T, V>(x, n * C + V * (sub + i * W));
#pragma unroll
      for (int j = 0; j < V; ++j) {
        f[i][j] = get<T, V>(v, j);
        s += f[i][j];
      }
    }
    const float mu = lane_sum<W>(s) / float(C);
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        f[i][j] -= mu;
        q = V * (sub + i * W) < C ? fmaf(f[i][j], f[i][j], q) : q;
      }
    const float r = 1.0f / sqrtf(lane_sum<W>(q) / float(C) + eps);
    if (!there) continue;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (V * (sub + i * W) < C) {
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = fmaf(f[i][j] * r, wr[i][j], br[i][j]);
        stv<T, V>(y, n * C + V * (sub + i * W), o);
      }
    if (sub == 0) {
      if (mean) mean[n] = mu;
      if (rstd) rstd[n] = r;
    }
  }
}

template <typename T, int V, int NI, int W>
__global__ __launch_bounds__(kShortThreads) void k_norm_short_backward(const T* __restrict__ x, const T* dy,
                                                                       const float* __restrict__ w,
                                                                       const float* __restrict__ mean,
                                                                       const float* __restrict__ rstd, int64_t N, int C,
                                                                       T* dx, float* __restrict__ partial) {
  __shared__ float red[kShortThreads * V];
  lds_poison(red, kShortThreads * V);
  const int sub = threadIdx.x % W;
  float wr[NI][V], aw[NI][V], ab[NI][V];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = V * (sub + i * W) + j;
      wr[i][j] = w && c < C ? w[c] : 1.0f;
      aw[i][j] = ab[i][j] = 0.0f;
    }
  constexpr int ROWS = kShortThreads / W;
  for (int64_t n0 = int64_t(blockIdx.x) * ROWS; n0 < N; n0 += int64_t(gridDim.x) * ROWS) {
    const int64_t n = n0 + threadIdx.x / W;
    const bool there = n < N;
    const float mu = there ? mean[n] : 0.0f, r = there ? rstd[n] : 0.0f;
    float xh[NI][V], g[NI][V], sg = 0.0f, sx = 0.0f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const bool in = there && V * (sub + i * W) < C;
      typename Vec<T, V>::type v = {}, d = {};
      if (in) {
        v = ldv<T, V>(x, n * C + V * (sub + i * W));
        d = ldv<T, V>(dy, n * C + V * (sub + i * W));
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        xh[i][j] = in ? (get<T, V>(v, j) - mu) * r : 0.0f;
        const float e = get<T, V>(d, j);
        aw[i][j] = fmaf(e, xh[i][j], aw[i][j]);
        ab[i][j] += e;
        g[i][j] = e * wr[i][j];
        sg += g[i][j];
        sx = fmaf(g[i][j], xh[i][j], sx);
      }
    }
    if (!dx) continue;
    const float mg = lane_sum<W>(sg) / float(C), mx = lane_sum<W>(sx) / float(C);
    if (!there) continue;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (V * (sub + i * W) < C) {
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = r * (g[i][j] - mg - xh[i][j] * mx);
        stv<T, V>(dx, n * C + V * (sub + i * W), o);
      }
  }
  if (!partial) return;
  // the groups' sums of one column, added in order
  float* const out = partial + int64_t(blockIdx.x) * 2 * C;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) red[(threadIdx.x / W) * (W * V) + V * sub + j] = k ? ab[i][j] : aw[i][j];
      __syncthreads();
      for (int q = threadIdx.x; q < W * V; q += kShortThreads) {
        const int c = V * W * i + q;
        if (c >= C) continue;
        float s = 0.0f;
        for (int u = 0; u < ROWS; ++u) s += red[u * W * V + q];
        out[k * C + c] = s;
      }
    }
}

// dw and db of rows too long for the registers: workgroup (step i, part of the
// rows), which walks down its rows in the A V places of that step.
template <typename T, int V, bool K1>
__global__ __launch_bounds__(1024) void k_norm_dw(const T* __restrict__ x, const T* __restrict__ dy,
                                                  const float* __restrict__ mean, const float* __restrict__ rstd,
                                                  int64_t N, int C, int L, int A, float* __restrict__ partial) {
  extern __shared__ float lds[];  // [A V], [A V / K]
  const int K = (L + 1) * (L + 1), t = threadIdx.x;
  const Places<V> pl(A, K, C, t);
  float* const red = lds;
  float* const sums = lds + A * V;
  lds_poison(lds, A * V + pl.cpc);
  const int R = C * K, at = int(blockIdx.x) * A * V + V * t;
  float aw[V], ab[V];
#pragma unroll
  for (int j = 0; j < V; ++j) aw[j] = ab[j] = 0.0f;
  if (pl.on && at < R)
#pragma unroll 4
    for (int64_t n = blockIdx.y; n < N; n += gridDim.y) {
      auto xi = step_load<T, V>(x + n * R, at, R), gi = step_load<T, V>(dy + n * R, at, R);
      const float mu = mean[n];
      step_fix<false, T, V>(xi, at, R);
      step_fix<false, T, V>(gi, at, R);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = get<T, V>(gi, j);
        const bool zero = K1 || j == pl.j0;
        aw[j] = fmaf(d, (get<T, V>(xi, j) - (zero ? mu : 0.0f)) * rstd[n * (L + 1) + (K1 ? 0 : pl.deg[j])], aw[j]);
        ab[j] += d;
      }
    }
  if (pl.on)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      red[V * t + j] = aw[j];
      if (K1)
        sums[V * t + j] = ab[j];
      else if (j == pl.j0)
        sums[pl.ch] = ab[j];
    }
  __syncthreads();
  float* const out = partial + int64_t(blockIdx.y) * (L + 2) * C;
  const int64_t c0 = int64_t(blockIdx.x) * pl.cpc;
  const int nc = int(C - c0 < pl.cpc ? C - c0 : pl.cpc);
  for (int q = t; q < (L + 2) * nc; q += int(blockDim.x)) {
    const int l = q / nc, c = q - l * nc;
    float s = 0.0f;
    if (l <= L)
      for (int m = 0; m < 2 * l + 1; ++m) s += red[c * K + l * l + m];
    else
      s = sums[c];
    out[int64_t(l) * C + c0 + c] = s;
  }
}

constexpr int64_t kMaxLds = 150 << 10;

// LDS bytes of a layout: the backward's sums by element (steps), the row's, the weights.
int64_t norm_lds(int L, int64_t C, int64_t A, int V, int steps) {
  const int64_t K = int64_t(L + 1) * (L + 1), AV = A * V;
  const int64_t all = (C * K + AV - 1) / AV;
  return (steps * (AV + AV / K) + (K == 1 ? 2 * A : AV + AV / K) + L + 2 + (L + 2) * (C | 1) +
          (steps > all ? steps : all + 8) * (AV / K)) * 4;
}

// The layout for rows of C channels: groups of 4 elements, of 8 in the bf16 forward
// where length and address make them 16 aligned bytes (`wide`), and the thread count
// that leaves the fewest lanes and steps of a row idle, at up to 32 elements a
// thread in registers.  back: the backward, whose sums by element take LDS.
bool layout(int L, int64_t C, bool bf16, bool wide, bool back, Lay* out) {
  const int64_t K = int64_t(L + 1) * (L + 1), R = C * K;
  if (R >= (int64_t(1) << 30) || R < 8) return false;
  // one coefficient of degree 0 in a group at most; and eight places' statistics beside
  // two rows leave the backward too few registers (degree 16, 64 channels: 618 us against 436)
  const int V = bf16 && wide && R % 8 == 0 && (K == 1 || (K >= 8 && !back)) ? 8 : 4;
  int64_t g = V;
  while (K % g) g /= 2;  // V is a power of two: the common divisor
  const int64_t unit = K / g;  // A is a multiple of it
  double best = 0.0;
  for (int64_t threads = 64; threads <= 1024; threads += 64) {
    const int64_t A = threads / unit * unit;
    if (A == 0 || norm_lds(L, C, A, V, 0) > kMaxLds) continue;
    const int64_t steps = (R + A * V - 1) / (A * V);
    static constexpr int kReg[] = {1, 2, 3, 4, 5, 6, 7, 8};
    int reg = 0;
    for (int r : kReg)
      if (r >= steps && (back ? (threads <= 512 || (V == 4 && r >= 4 && r <= 6)) && norm_lds(L, C, A, V, r) <= kMaxLds
                              : r * V <= 32)) {
        reg = r;
        break;
      }
    // the share of lanes and steps at work; more than 4 waves in step leave the barriers less to overlap
    const double use = double(R) / (double(threads) * V * (reg ? reg : steps)) *
                       (threads > 512 ? 0.7 : threads > 256 ? 0.85 : 1.0) * (reg ? 1.0 : 0.25);
    if (use > best * 1.02) {
      best = use;
      *out = Lay{int(A), int(threads), int(steps), V, reg};
    }
  }
  return best > 0.0;
}

// Rows of L = 0 that a wave or less takes: W lanes and NI steps for C channels.
struct Short {
  int V, NI, W;
};
bool short_rows(int L, int64_t C, bool bf16, bool wide, Short* out) {
  if (L != 0) return false;
  int V = wide ? (bf16 ? 8 : 4) : 1;
  if (C % V != 0) V = 1;
  for (int W : {8, 16, 32, 64})
    for (int NI : {1, 2, 4})
      if ((W == 64 || NI == 1) && int64_t(V) * W * NI >= C) return *out = Short{V, NI, W}, true;
  return false;
}

constexpr int kAnyThreads = 256;

// Sum of v over the workgroup's 256 threads, in a fixed order; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kAnyThreads / 64; ++i) s += red[i];
  return s;
}

// Any degree and channel count: one workgroup a row (a channel, in the weights' sums), a
// degree at a time.  y may be x (and dx below dy): an element is read for the last time by
// the thread that writes it.
constexpr int64_t kAnyGrid = 1 << 20;  // workgroups at most: a launch holds less than 2^32 threads
template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_any(const T* x, const float* __restrict__ w,
                                                          const float* __restrict__ b, float eps, int64_t N, int64_t C,
                                                          int L, T* y, float* __restrict__ mean,
                                                          float* __restrict__ rstd) {
  __shared__ float red[kAnyThreads / 64];
  lds_poison(red, kAnyThreads / 64);
  const int64_t K = int64_t(L + 1) * (L + 1);
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const int64_t base = n * C * K;
    for (int l = 0; l <= L; ++l) {
      const int64_t M = 2 * l + 1, cnt = C * M;
      float mu = 0.0f;
      if (l == 0) {
        float s = 0.0f;
        for (int64_t c = threadIdx.x; c < C; c += kAnyThreads) s += ld(x, base + c * K);
        mu = block_sum(s, red) / float(C);
        if (mean && threadIdx.x == 0) mean[n] = mu;
      }
      float s = 0.0f;
      for (int64_t q = threadIdx.x; q < cnt; q += kAnyThreads) {
        const int64_t c = q / M;
        const float v = ld(x, base + c * K + l * l + (q - c * M)) - mu;
        s = fmaf(v, v, s);
      }
      const float r = 1.0f / sqrtf(block_sum(s, red) / float(cnt) + eps);
      if (rstd && threadIdx.x == 0) rstd[n * (L + 1) + l] = r;
      for (int64_t q = threadIdx.x; q < cnt; q += kAnyThreads) {
        const int64_t c = q / M, i = base + c * K + l * l + (q - c * M);
        const float v = (ld(x, i) - mu) * r;
        const float wl = w ? w[l * C + c] : 1.0f;
        st(y, i, l == 0 && b ? fmaf(v, wl, b[c]) : v * wl);
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_dx_any(const T* __restrict__ x, const T* dy,
                                                             const float* __restrict__ w,
                                                             const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, int64_t N, int64_t C,
                                                             int L, T* dx) {
  __shared__ float red[kAnyThreads / 64];
  lds_poison(red, kAnyThreads / 64);
  const int64_t K = int64_t(L + 1) * (L + 1);
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const int64_t base = n * C * K;
    for (int l = 0; l <= L; ++l) {
      const int64_t M = 2 * l + 1, cnt = C * M;
      const float mu = l == 0 ? mean[n] : 0.0f, r = rstd[n * (L + 1) + l];
      float sg = 0.0f, sx = 0.0f;
      for (int64_t q = threadIdx.x; q < cnt; q += kAnyThreads) {
        const int64_t c = q / M, i = base + c * K + l * l + (q - c * M);
        const float g = ld(dy, i) * (w ? w[l * C + c] : 1.0f);
        sg += g;
        sx = fmaf(g, (ld(x, i) - mu) * r, sx);
      }
      sg = l == 0 ? block_sum(sg, red) / float(cnt) : 0.0f;
      sx = block_sum(sx, red) / float(cnt);
      for (int64_t q = threadIdx.x; q < cnt; q += kAnyThreads) {
        const int64_t c = q / M, i = base + c * K + l * l + (q - c * M);
        const float g = ld(dy, i) * (w ? w[l * C + c] : 1.0f);
        st(dx, i, r * (g - sg - (ld(x, i) - mu) * r * sx));
      }
    }
  }
}

// Partial sums of dw and db over a chunk of rows: workgroup (channels, chunk).
// partial[chunk][(L + 2) C]: L + 1 rows of dw, then db.
template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_dw_any(const T* __restrict__ x, const T* __restrict__ dy,
                                                             const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, int64_t N, int64_t C,
                                                             int L, int64_t chunk, float* __restrict__ partial) {
  __shared__ float red[kAnyThreads / 64];
  lds_poison(red, kAnyThreads / 64);
  const int64_t n0 = int64_t(blockIdx.y) * chunk;
  const int64_t rows = n0 + chunk < N ? chunk : N - n0;
  const int64_t K = int64_t(L + 1) * (L + 1);
  for (int64_t c = blockIdx.x; c < C; c += gridDim.x) {
    float* const out = partial + int64_t(blockIdx.y) * (L + 2) * C + c;
    for (int l = 0; l <= L; ++l) {
      const int64_t M = 2 * l + 1;
      float s = 0.0f, sb = 0.0f;
      for (int64_t q = threadIdx.x; q < rows * M; q += kAnyThreads) {
        const int64_t r = q / M, n = n0 + r, i = (n * C + c) * K + l * l + (q - r * M);
        const float d = ld(dy, i);
        s = fmaf(d, (ld(x, i) - (l == 0 ? mean[n] : 0.0f)) * rstd[n * (L + 1) + l], s);
        sb += d;
      }
      s = block_sum(s, red);
      if (threadIdx.x == 0) out[l * C] = s;
      if (l == 0) {
        sb = block_sum(sb, red);
        if (threadIdx.x == 0) out[(L + 1) * C] = sb;
      }
    }
  }
}

// The parts' sums, added in order: a workgroup takes 16 columns at a time, 64 groups of
// threads every 64th part each, then a tree over the groups.
constexpr int kSumThreads = 1024, kSumCols = 16;
__global__ __launch_bounds__(kSumThreads) void k_norm_sum(const float* __restrict__ partial, int parts, int64_t cols,
                                                          int64_t wcols, float* __restrict__ dw,
                                                          float* __restrict__ db) {
  __shared__ float red[kSumThreads];
  lds_poison(red, kSumThreads);
  const int c = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
  for (int64_t col0 = int64_t(blockIdx.x) * kSumCols; col0 < cols; col0 += int64_t(gridDim.x) * kSumCols) {
    const int64_t col = col0 + c;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 8
      for (int i = g; i < parts; i += kSumThreads / kSumCols) s += partial[i * cols + col];
    }
    __syncthreads();  // the columns before are read
    red[threadIdx.x] = s;
#pragma unroll
    for (int o = kSumThreads / 2; o >= kSumCols; o /= 2) {
      __syncthreads();
      if (int(threadIdx.x) < o) red[threadIdx.x] += red[threadIdx.x + o];
    }
    if (g == 0 && col < cols) {
      if (col < wcols) {
        if (dw) dw[col] = red[c];
      } else if (db) {
        db[col - wcols] = red[c];
      }
    }
  }
}

hipError_t sum_parts(const NormArgs& a, int64_t parts, hipStream_t s) {
  const int64_t cols = (a.L + 2) * a.C, n = std::min((cols + kSumCols - 1) / kSumCols, kAnyGrid);
  k_norm_sum<<<dim3{uint32_t(n)}, kSumThreads, 0, s>>>(a.partial, int(parts), cols, (a.L + 1) * a.C, a.dw, a.db);
  return hipGetLastError();
}

int64_t any_chunks(int64_t N) { return N < 64 ? 1 : (N < 64 * 64 ? N / 64 : 64); }

}  // namespace

namespace {

// Rows per launch: enough workgroups to fill the chip (16 waves a CU), the rest of
// the rows in turn, so that a workgroup loads its weights once.
int64_t grid_rows(int64_t N, int threads) {
  const int64_t n = 256 * 16 / (threads / 64);
  return N < n ? N : n;
}
// The backward: two rows at least, where they fill the chip at all, since every
// workgroup writes a part of the weights' gradient.
int64_t grid_rows_back(int64_t N, int threads) {
  const int64_t n = grid_rows(N, threads), half = (N + 1) / 2;
  return n <= half ? n : std::max<int64_t>(half, std::min<int64_t>(n, 256));
}

template <typename T, int V, int NI>
hipError_t run_norm(const NormArgs& a, const Lay& y, hipStream_t s) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1);
  const size_t lds = size_t(norm_lds(a.L, a.C, y.A, V, 0));
  const uint32_t grid = uint32_t(grid_rows(a.N, y.threads));
  const T* x = static_cast<const T*>(a.x);
  T* o = static_cast<T*>(a.y);
  const bool even = a.C * K % V == 0;
  auto k = a.L == 0 ? k_norm<T, V, NI, true, false> : k_norm<T, V, NI, false, false>;
  if constexpr (NI > 0)
    if (even) k = a.L == 0 ? k_norm<T, V, NI, true, true> : k_norm<T, V, NI, false, true>;
  k<<<grid, y.threads, lds, s>>>(x, a.w, a.b, a.eps, a.N, int(a.C), a.L, y.A, o, a.mean, a.rstd);
  return hipGetLastError();
}

template <typename T, int V, int NI>
hipError_t run_norm_backward(const NormArgs& a, const Lay& y, hipStream_t s) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1);
  const size_t lds = size_t(norm_lds(a.L, a.C, y.A, V, NI));
  const uint32_t grid = uint32_t(grid_rows_back(a.N, y.threads));
  const T *x = static_cast<const T*>(a.x), *g = static_cast<const T*>(a.dy);
  T* o = static_cast<T*>(a.y);
  float* const part = NI > 0 && (a.dw || a.db) ? a.partial : nullptr;
  // up to 512 threads may hold twice the registers
  constexpr int kMax = NI > 0 ? 512 : 1024;
  const bool even = a.C * K % V == 0;
  auto pick = [&](auto one) {
    constexpr bool K1 = decltype(one)::value;
    auto k = k_norm_backward<T, V, NI, K1, false, kMax>;
    if constexpr (NI > 0)
      if (even) k = k_norm_backward<T, V, NI, K1, true, kMax>;
    if constexpr (V == 4 && NI >= 4 && NI <= 6)
      if (y.threads > 512) k = even ? k_norm_backward<T, V, NI, K1, true, 1024> : k_norm_backward<T, V, NI, K1, false, 1024>;
    return k;
  };
  auto k = pick(std::true_type{});
  if constexpr (V == 4)  // eight places a thread: L = 0 alone
    if (a.L > 0) k = pick(std::false_type{});
  k<<<grid, y.threads, lds, s>>>(x, g, a.w, a.mean_in, a.rstd_in, a.N, int(a.C), a.L, y.A, o, part);
  return hipGetLastError();
}

// Workgroups of the kernels for short rows.
int64_t short_grid(int64_t N, const Short& h) {
  const int64_t rows = kShortThreads / h.W, n = (N + rows - 1) / rows;
  return n < 1024 ? n : 1024;
}

template <typename T, int V, int NI, int W>
hipError_t run_short(const NormArgs& a, bool back, uint32_t grid, hipStream_t s) {
  const T* x = static_cast<const T*>(a.x);
  T* o = static_cast<T*>(a.y);
  if (back)
    k_norm_short_backward<T, V, NI, W><<<grid, kShortThreads, 0, s>>>(
        x, static_cast<const T*>(a.dy), a.w, a.mean_in, a.rstd_in, a.N, int(a.C), o,
        a.dw || a.db ? a.partial : nullptr);
  else
    k_norm_short<T, V, NI, W><<<grid, kShortThreads, 0, s>>>(x, a.w, a.b, a.eps, a.N, int(a.C), o, a.mean, a.rstd);
  return hipGetLastError();
}
template <typename T, int V>
hipError_t with_short(const NormArgs& a, bool back, const Short& h, hipStream_t s) {
  const uint32_t g = uint32_t(short_grid(a.N, h));
  if (h.W == 8) return run_short<T, V, 1, 8>(a, back, g, s);
  if (h.W == 16) return run_short<T, V, 1, 16>(a, back, g, s);
  if (h.W == 32) return run_short<T, V, 1, 32>(a, back, g, s);
  if (h.NI == 1) return run_short<T, V, 1, 64>(a, back, g, s);
  if (h.NI == 2) return run_short<T, V, 2, 64>(a, back, g, s);
  return run_short<T, V, 4, 64>(a, back, g, s);
}
hipError_t launch_short(const NormArgs& a, bool back, const Short& h, hipStream_t s) {
  if (a.bf16) return h.V == 8 ? with_short<uint16_t, 8>(a, back, h, s) : with_short<uint16_t, 1>(a, back, h, s);
  return h.V == 4 ? with_short<float, 4>(a, back, h, s) : with_short<float, 1>(a, back, h, s);
}

// Parts of the rows for k_norm_dw.
int64_t dw_parts(int64_t N, const Lay& y) {
  const int64_t n = (256 * 16 / (y.threads / 64) + y.NI - 1) / y.NI;
  return n < 1 ? 1 : (N < n ? N : n);
}

template <typename T, int V>
hipError_t run_norm_dw(const NormArgs& a, const Lay& y, hipStream_t s) {
  const int K = (a.L + 1) * (a.L + 1);
  const size_t lds = (size_t(y.A) * V + size_t(y.A) * V / K) * 4;
  const dim3 grid{uint32_t(y.NI), uint32_t(dw_parts(a.N, y))};
  const T *x = static_cast<const T*>(a.x), *g = static_cast<const T*>(a.dy);
  auto k = k_norm_dw<T, V, true>;
  if constexpr (V == 4)
    if (K > 1) k = k_norm_dw<T, V, false>;
  k<<<grid, y.threads, lds, s>>>(x, g, a.mean_in, a.rstd_in, a.N, int(a.C), a.L, y.A, a.partial);
  return hipGetLastError();
}

// f<T, V, NI>() of a layout.
template <typename T, int V, typename F>
hipError_t with_steps(int reg, F f) {
  switch (reg) {
    case 1: return f.template operator()<T, V, 1>();
    case 2: return f.template operator()<T, V, 2>();
    case 3: return f.template operator()<T, V, 3>();
    case 4: return f.template operator()<T, V, 4>();
    case 5:
      if constexpr (V <= 4 || F::back) return f.template operator()<T, V, 5>();
      break;
    case 6:
      if constexpr (V <= 4 || F::back) return f.template operator()<T, V, 6>();
      break;
    case 7:
      if constexpr (V <= 4 || F::back) return f.template operator()<T, V, 7>();
      break;
    case 8:
      if constexpr (V <= 4 || F::back) return f.template operator()<T, V, 8>();
      break;
    case 0: return f.template operator()<T, V, 0>();
  }
  return hipErrorInvalidValue;
}
template <typename F>
hipError_t with_layout(bool bf16, const Lay& y, F f) {
  if (bf16) return y.V == 8 ? with_steps<uint16_t, 8>(y.steps_reg, f) : with_steps<uint16_t, 4>(y.steps_reg, f);
  return with_steps<float, 4>(y.steps_reg, f);
}

struct Forward {
  static constexpr bool back = false;
  const NormArgs& a;
  const Lay& y;
  hipStream_t s;
  template <typename T, int V, int NI>
  hipError_t operator()() const {
    return run_norm<T, V, NI>(a, y, s);
  }
};
struct Backward {
  static constexpr bool back = true;
  const NormArgs& a;
  const Lay& y;
  hipStream_t s;
  template <typename T, int V, int NI>
  hipError_t operator()() const {
    if constexpr (NI == 0) {  // dw and db before dx, which may be written over dy
      hipError_t e = a.dw || a.db ? run_norm_dw<T, V>(a, y, s) : hipSuccess;
      if (e == hipSuccess && a.y) e = run_norm_backward<T, V, 0>(a, y, s);
      return e;
    } else {
      return run_norm_backward<T, V, NI>(a, y, s);
    }
  }
};

bool wide16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Partial sums of the backward with layout y.
int64_t parts_of(int64_t N, const Lay& y) { return y.steps_reg ? grid_rows_back(N, y.threads) : dw_parts(N, y); }

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  const bool wide = wide16(a.x) && wide16(a.y);
  Short h;
  if (short_rows(a.L, a.C, a.bf16, wide, &h)) return launch_short(a, false, h, s);
  Lay y;
  if (layout(a.L, a.C, a.bf16, wide, false, &y)) return with_layout(a.bf16, y, Forward{a, y, s});
  const dim3 grid{uint32_t(std::min(a.N, kAnyGrid))};
  if (a.bf16)
    k_norm_any<<<grid, kAnyThreads, 0, s>>>(static_cast<const uint16_t*>(a.x), a.w, a.b, a.eps, a.N, a.C, a.L,
                                            static_cast<uint16_t*>(a.y), a.mean, a.rstd);
  else
    k_norm_any<<<grid, kAnyThreads, 0, s>>>(static_cast<const float*>(a.x), a.w, a.b, a.eps, a.N, a.C, a.L,
                                            static_cast<float*>(a.y), a.mean, a.rstd);
  return hipGetLastError();
}

int64_t norm_partial_floats(int L, int64_t N, int64_t C, bool bf16) {
  // whichever way the call's addresses will allow
  int64_t parts = any_chunks(N);
  for (bool wide : {false, true}) {
    Lay y;
    Short h;
    if (short_rows(L, C, bf16, wide, &h))
      parts = std::max(parts, short_grid(N, h));
    else if (layout(L, C, bf16, wide, true, &y))
      parts = std::max(parts, parts_of(N, y));
  }
  return parts * (L + 2) * C;
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
  const bool wide = wide16(a.x) && wide16(a.dy) && wide16(a.y);
  Short h;
  if (a.N > 0 && short_rows(a.L, a.C, a.bf16, wide, &h)) {
    const hipError_t e = launch_short(a, true, h, s);
    return e != hipSuccess || !(a.dw || a.db) ? e : sum_parts(a, short_grid(a.N, h), s);
  }
  Lay y;
  if (a.N > 0 && layout(a.L, a.C, a.bf16, wide, true, &y)) {
    const hipError_t e = with_layout(a.bf16, y, Backward{a, y, s});
    if (e != hipSuccess || !(a.dw || a.db)) return e;
    return sum_parts(a, parts_of(a.N, y), s);
  }
  const int64_t chunks = any_chunks(a.N), chunk = (a.N + chunks - 1) / chunks;
  const int64_t used = a.N ? (a.N + chunk - 1) / chunk : 0;
  const dim3 grid{uint32_t(std::min(a.N, kAnyGrid))}, gw{uint32_t(std::min(a.C, kAnyGrid)), uint32_t(used)};
  const bool weights = a.dw || a.db;
  // dw and db before dx, which may be written over dy
  if (a.bf16) {
    const auto *x = static_cast<const uint16_t*>(a.x), *dy = static_cast<const uint16_t*>(a.dy);
    if (weights && a.N)
      k_norm_dw_any<<<gw, kAnyThreads, 0, s>>>(x, dy, a.mean_in, a.rstd_in, a.N, a.C, a.L, chunk, a.partial);
    if (a.y && a.N)
      k_norm_dx_any<<<grid, kAnyThreads, 0, s>>>(x, dy, a.w, a.mean_in, a.rstd_in, a.N, a.C, a.L,
                                                 static_cast<uint16_t*>(a.y));
  } else {
    const auto *x = static_cast<const float*>(a.x), *dy = static_cast<const float*>(a.dy);
    if (weights && a.N)
      k_norm_dw_any<<<gw, kAnyThreads, 0, s>>>(x, dy, a.mean_in, a.rstd_in, a.N, a.C, a.L, chunk, a.partial);
    if (a.y && a.N)
      k_norm_dx_any<<<grid, kAnyThreads, 0, s>>>(x, dy, a.w, a.mean_in, a.rstd_in, a.N, a.C, a.L,
                                                 static_cast<float*>(a.y));
  }
  return weights ? sum_parts(a, used, s) : hipGetLastError();
}

}  // namespace gtp
