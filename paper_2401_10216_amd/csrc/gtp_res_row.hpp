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

int64_t res_lds(const ResLay& y, int64_t K, int L, bool back);  // LDS bytes; back: of the gradient

constexpr int kTeamThreads = 256;

// What a thread's places hold: place j of step i is element V t + i A V + j of the row, always of one
// coefficient (one degree); a step moves it on by A V / K channels.
template <int V, bool K1>
struct Spots {
  int deg[V];
  uint32_t next;      // bit j: place j's channel is the one behind place 0's (V <= K: at most two)
  int ch0, j0, ch;    // channel of place 0 at step 0; the place of a degree-0 coefficient (-1: none) and its channel
  int cpc;            // channels a step moves on by
  bool on;
  __device__ __forceinline__ Spots(int A, int K, int t) {
    on = t < A;
    cpc = A * V / K;
    j0 = -1;
    next = 0;
    const int first = on ? V * t : 0;
    ch0 = ch = first / K;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (first + j) / K, k = first + j - c * K;
      deg[j] = K1 ? 0 : degree_of(k);
      if (!K1 && c != ch0) next |= 1u << j;
      if (!K1 && k == 0) j0 = j, ch = c;
    }
  }
  // v at the places of degree 0, else 0
  __device__ __forceinline__ float zero(int j, float v) const { return K1 || j == j0 ? v : 0.0f; }
  // the sum of v at the places of degree 0
  __device__ __forceinline__ float sum_zero(const float (&v)[V]) const {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) s = K1 ? s + v[j] : j == j0 ? v[j] : s;
    return s;
  }
};

// Tables in LDS: P = scale w1 and W2 for each element of the row, so that a thread reads those of
// its V elements at once (from a table by degree and channel, an address and a word each, they took
// half of the kernels' instructions), then Q = scale's times the first norm's shift and B2 by channel.
struct ResTables {
  float *P, *W2, *Q, *B2;
  __host__ __device__ static int64_t floats(int64_t elements, int64_t channels) { return 2 * (elements + channels); }
  // elements: NI A V, channels: NI A V / K, of all steps: the row's and what the last step has past them
  __device__ ResTables(float* lds, int elements, int channels) {
    P = lds;
    W2 = P + elements;
    Q = W2 + elements;
    B2 = Q + channels;
  }
  // The teams deal the steps.  A table's loads all together, none under a condition of its own: one after the other
  // they took 26 us for rows of 5184 elements.
  template <int V, int NI, int TEAMS, bool K1>
  __device__ void load(const ResWeights& w, const Spots<V, K1>& at, int A, int t, int team) const {
    constexpr int S = (NI + TEAMS - 1) / TEAMS, Z = K1 ? V : 1;
    const int C = int(w.C);
    auto channel = [&](int s, int j) { return (K1 ? V * t + j : at.ch0 + int((at.next >> j) & 1u)) + (s * TEAMS + team) * at.cpc; };
    auto times = [&](const float* from, float (&v)[S][V]) {
      if (!from) return;
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int c = channel(s, j);
          v[s][j] *= from[at.deg[j] * C + (c < C ? c : C - 1)];
        }
    };
    auto elements = [&](float* to, const float* one, const float* other) {
      float v[S][V];
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < V; ++j) v[s][j] = 1.0f;
      times(one, v);
      times(other, v);
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at.on && s * TEAMS + team < NI)
            to[(s * TEAMS + team) * A * V + V * t + j] = channel(s, j) < C ? v[s][j] : 0.0f;
    };
    // by channel: shift times row 0 of `one`
    auto channels = [&](float* to, const float* shift, const float* one) {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < Z; ++j) {
          const int c = K1 ? channel(s, j) : at.ch + (s * TEAMS + team) * at.cpc, in = c < C ? c : C - 1;
          float v = 0.0f;
          if (shift) v = shift[in] * (one ? one[in] : 1.0f);
          if (at.on && (K1 || at.j0 >= 0) && s * TEAMS + team < NI) to[c] = c < C ? v : 0.0f;
        }
    };
    elements(P, w.scale, w.w1);
    elements(W2, w.w2, nullptr);
    channels(Q, w.b1, w.scale);
    channels(B2, w.b2, nullptr);
  }
};

template <int V>
__device__ __forceinline__ void read_table(const float* p, float (&o)[V]) {
#pragma unroll
  for (int j = 0; j < V; j += 4) {
    typedef float f4 __attribute__((ext_vector_type(4)));
    const f4 v = *reinterpret_cast<const f4*>(p + j);
    o[j] = v[0], o[j + 1] = v[1], o[j + 2] = v[2], o[j + 3] = v[3];
  }
}

// What a team's lanes do together.  red: of a workgroup, [A V] (K1: [A]) by place, [slots] at degree 0, [L + 2] results.
template <int W, int V, bool K1>
struct Team {
  const Spots<V, K1>& pl;
  int A, K, C, L, t;
  float *red, *zero, *stat;
  __device__ int slots() const { return K1 ? A : pl.cpc; }
  __host__ __device__ static int64_t floats(int64_t A, int64_t K, int L) {
    return W ? 0 : (K1 ? 2 * A : A * V + A * V / K) + L + 2;
  }
  __device__ Team(const Spots<V, K1>& p, int A_, int K_, int C_, int L_, int t_, float* lds)
      : pl(p), A(A_), K(K_), C(C_), L(L_), t(t_), red(lds), zero(lds + (K1 ? A_ : A_ * V)), stat(zero + slots()) {}
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
    float q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = 0.0f;
    if (pl.on)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) q[j] += val(i, j);  // zero past the row's end
    const float s = pl.sum_zero(q);
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = 0.0f;
    auto squares = [&](float about) {
      float off[V];
#pragma unroll
      for (int j = 0; j < V; ++j) off[j] = pl.zero(j, about);
      if (pl.on)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float v = there(i, j) ? val(i, j) - off[j] : 0.0f;
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
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = typename Vec<T, V>::type{};
  }
  __device__ __forceinline__ float operator()(int i, int j) const { return get<T, V>(v[i], j); }
  // fp32 rows only: something made of the element in its place
  __device__ __forceinline__ void set(int i, int j, float f) {
    if constexpr (sizeof(T) == 4) v[i][j] = f;
  }
  __device__ __forceinline__ void renewed() {
#pragma unroll
    for (int i = 0; i < NI; ++i) renew(v[i]);
  }
};

// A row's gate: with one coefficient a channel as the row's elements; else C numbers dealt to the team's lanes (NI a
// lane at most, since K >= V), which put their sigmoids in LDS.
template <typename T, int V, int NI, bool K1>
struct RowGate {
  RowRegs<T, V, NI> row;
  float own[NI];
  __device__ __forceinline__ void load(const T* gate, int t, int AV, int C, int lanes) {
    if constexpr (K1) {
      row.load(gate, t, AV, C);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) own[i] = ld(gate, t + i * lanes < C ? t + i * lanes : C - 1);
    }
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
