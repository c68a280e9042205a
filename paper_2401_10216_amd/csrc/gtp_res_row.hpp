// Rows of the residual step in registers (gtp_res_fwd.hip, gtp_res_bwd*.hip): how a row lies on
// the lanes that share it, and their sums by degree.
//
// A team of 16 or 64 lanes, or a workgroup, takes a row; its elements stay in registers between the
// sums and the results, so each tensor is read or written once.  A wave's teams add up a degree across
// their lanes (no LDS, no barrier: the waves of a CU run past each other's loads); longer rows take a
// workgroup, whose waves meet in LDS.
#pragma once

#include "gtp_norm_core.hpp"
#include "gtp_res.hpp"

namespace gtp {

// W: lanes of a team, 0 = the workgroup; V elements at a time on A threads, NI steps.
struct ResLay {
  int W, V, NI, A, threads;
  int teams() const { return W ? threads / W : 1; }
};
// The layout of rows in registers; false where a row does not fit them, or has fewer than 8 elements.
bool residual_layout(const ResArgs& a, bool wide, bool back, ResLay* out);

constexpr int kTeamThreads = 256;

// Tables in LDS, a degree's row of C in C | 1: P = scale w1 [L+1], Q = scale w1's shift [C] (zeros without post),
// W2 [L+1], B2 [C].
struct ResTables {
  float *P, *Q, *W2, *B2;
  __host__ __device__ static int64_t floats(int L, int64_t C) { return 2 * ((L + 1) * (C | 1) + C); }
  __device__ ResTables(float* lds, int L, int C) {
    P = lds;
    Q = P + (L + 1) * (C | 1);
    W2 = Q + C;
    B2 = W2 + (L + 1) * (C | 1);
  }
  __device__ void load(const ResWeights& w, int L) const {
    const int C = int(w.C);
    for (int l = 0; l <= L; ++l)
      for (int c = threadIdx.x; c < C; c += int(blockDim.x)) {
        P[l * (C | 1) + c] = w.s(l, c) * w.post_w(l, c);
        W2[l * (C | 1) + c] = w.pre_w(l, c);
      }
    for (int c = threadIdx.x; c < C; c += int(blockDim.x)) {
      Q[c] = w.s(0, c) * w.post_b(0, c);
      B2[c] = w.pre_b(0, c);
    }
  }
};

// What a team's lanes do together.  red: of a workgroup, [A V] (K1: [A]) by place, [slots] at degree 0, [L + 2] results.
template <int W, int V, bool K1>
struct Team {
  const Places<V>& pl;
  int A, K, C, L, t;
  float *red, *zero, *stat;
  __device__ int slots() const { return K1 ? A : pl.cpc; }
  __host__ __device__ static int64_t floats(int64_t A, int64_t K, int L) {
    return W ? 0 : (K1 ? 2 * A : A * V + A * V / K) + L + 2;
  }
  __device__ Team(const Places<V>& p, int A_, int K_, int C_, int L_, int t_, float* lds)
      : pl(p), A(A_), K(K_), C(C_), L(L_), t(t_), red(lds), zero(lds + (K1 ? A_ : A_ * V)), stat(zero + slots()) {}
  __device__ bool at_zero(int j) const { return K1 || j == pl.j0; }
  // What one lane wrote to LDS is there for the team's others.
  __device__ void meet() const {
    if constexpr (W == 0) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }

  // Means over a row: m[j] of q[.] over the degree of place j, m0 of s at degree 0 (q, s: the lane's sums,
  // zeros where it has no places).
  __device__ void means(const float (&q)[V], float s, float (&m)[V], float& m0) const {
    const float inv = 1.0f / float(C);
    if constexpr (W > 0) {
      m0 = lane_sum<W>(s) * inv;
      degrees(q, m, [&](int l, float v) { return v * (inv / float(2 * l + 1)); });
    } else {
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
      if (pl.on) {
        if constexpr (K1) {
          float u = 0.0f;
#pragma unroll
          for (int j = 0; j < V; ++j) u += q[j];
          red[t] = u;
          zero[t] = s;
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) red[V * t + j] = q[j];
          if (pl.j0 >= 0) zero[pl.ch] = s;
        }
      }
      __syncthreads();
      if (wave == 0) {
        float u = 0.0f, v = 0.0f;
        for (int c = lane; c < slots(); c += 64) {
          u += zero[c];
          if constexpr (K1) v += red[c];
        }
        u = wave_sum(u);
        if constexpr (K1) v = wave_sum(v);
        if (lane == 0) {
          stat[L + 1] = u * inv;
          if constexpr (K1) stat[0] = v * inv;
        }
      }
      if constexpr (!K1)
        by_degree(red, K, pl.cpc, L, 0, [&](int l, float v) {
          if (lane == 0) stat[l] = v * (inv / float(2 * l + 1));
        });
      __syncthreads();
      m0 = stat[L + 1];
#pragma unroll
      for (int j = 0; j < V; ++j) m[j] = stat[K1 ? 0 : pl.deg[j]];
    }
  }

  // f(l, sum over the degree) for each place's degree, across a wave's team.
  template <typename F>
  __device__ void degrees(const float (&q)[V], float (&m)[V], F f) const {
    if constexpr (K1) {
      float u = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) u += q[j];
      u = f(0, lane_sum<W>(u));
#pragma unroll
      for (int j = 0; j < V; ++j) m[j] = u;
    } else {
      for (int l = 0; l <= L; ++l) {
        float u = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) u += pl.deg[j] == l ? q[j] : 0.0f;
        u = f(l, lane_sum<W>(u));
#pragma unroll
        for (int j = 0; j < V; ++j) m[j] = pl.deg[j] == l ? u : m[j];
      }
    }
  }

  // Mean at degree 0 and 1 / size of each place's degree of the values val(i, j), there(i, j) in the row;
  // out(l, 1 / size) by one lane.  Squares at degree 0 are taken about the mean (a workgroup: about each thread's
  // own, joined with the threads' sums), so that a mean far from zero costs no digits.
  template <int NI, typename F, typename G, typename O>
  __device__ void statistics(F val, G there, float eps, float& mu, float (&r)[V], O out) const {
    float q[V], s = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = 0.0f;
    if (pl.on)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j)
          s += at_zero(j) ? val(i, j) : 0.0f;  // zero past the row's end
    auto squares = [&](float about) {
      if (pl.on)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float v = val(i, j);
            v = at_zero(j) ? (there(i, j) ? v - about : 0.0f) : v;
            q[j] = fmaf(v, v, q[j]);
          }
    };
    const float inv = 1.0f / float(C);
    if constexpr (W > 0) {
      mu = lane_sum<W>(s) * inv;
      squares(mu);
      degrees(q, r, [&](int l, float v) {
        const float one = 1.0f / sqrtf(v * (inv / float(2 * l + 1)) + eps);
        if (t == 0) out(l, one);
        return one;
      });
    } else {
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, R = C * K;
      const int mine = K1 ? elements_of(R, V, A * V, t) : (C - pl.ch + pl.cpc - 1) / pl.cpc;
      squares(mine > 0 ? s / float(mine) : 0.0f);
      if (pl.on) {
        if constexpr (K1) {
          float u = 0.0f;
#pragma unroll
          for (int j = 0; j < V; ++j) u += q[j];
          red[t] = u;
          zero[t] = s;
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) red[V * t + j] = q[j];
          if (pl.j0 >= 0) zero[pl.ch] = s;
        }
      }
      __syncthreads();
      if (wave == 0) {
        float u = 0.0f;
        for (int c = lane; c < slots(); c += 64) u += zero[c];
        const float m = wave_sum(u) * inv;
        float v = 0.0f;
        for (int c = lane; c < slots(); c += 64) {
          const int nc = K1 ? elements_of(R, V, A * V, c) : (C - c + pl.cpc - 1) / pl.cpc;  // 0 past the last
          if (nc > 0) {
            const float d = zero[c] / float(nc) - m;
            v += red[K1 ? c : c * K] + float(nc) * d * d;
          }
        }
        const float one = 1.0f / sqrtf(wave_sum(v) * inv + eps);
        if (lane == 0) {
          stat[0] = one;
          stat[L + 1] = m;
          out(0, one);
        }
      }
      if constexpr (!K1)
        by_degree(red, K, pl.cpc, L, 1, [&](int l, float v) {
          const float one = 1.0f / sqrtf(v * (inv / float(2 * l + 1)) + eps);
          if (lane == 0) {
            stat[l] = one;
            out(l, one);
          }
        });
      __syncthreads();
      mu = stat[L + 1];
#pragma unroll
      for (int j = 0; j < V; ++j) r[j] = stat[K1 ? 0 : pl.deg[j]];
    }
  }
};

// A row's NI steps of V elements in registers.  Only the last step may pass the row's end.
template <typename T, int V, int NI>
struct RowRegs {
  typename Vec<T, V>::type v[NI];
  __device__ __forceinline__ void load(const T* row, int t, int AV, int R) {
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = step_load<T, V>(row, i * AV + V * t, R);
  }
  __device__ __forceinline__ void fix(int t, int AV, int R) {  // zeros past the end
    step_fix<false, T, V>(v[NI - 1], (NI - 1) * AV + V * t, R);
  }
  __device__ __forceinline__ float operator()(int i, int j) const { return get<T, V>(v[i], j); }
  __device__ __forceinline__ void renewed() {
#pragma unroll
    for (int i = 0; i < NI; ++i) renew(v[i]);
  }
};

// f.template operator()<T, V, NI, W, K1>() of a layout.
template <typename T, int V, int W, bool K1, int MOST, int NI, typename F>
hipError_t res_with_steps(const ResLay& y, F f) {
  if constexpr (NI > MOST) {
    return hipErrorInvalidValue;
  } else {
    if (y.NI == NI) return f.template operator()<T, V, NI, W, K1>();
    return res_with_steps<T, V, W, K1, MOST, NI + 1>(y, f);
  }
}
template <typename T, int V, bool K1, typename F>
hipError_t res_with_team(const ResLay& y, F f) {
  if (y.W == 16) return res_with_steps<T, V, 16, K1, 2, 1>(y, f);
  if (y.W == 64) return res_with_steps<T, V, 64, K1, 32 / V, 1>(y, f);
  return res_with_steps<T, V, 0, K1, 32 / V, 1>(y, f);
}

}  // namespace gtp
