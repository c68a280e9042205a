// The residual step's gradient, rows in registers (formulas in gtp_res.hpp, rows and teams in
// gtp_res_row.hpp).  HBM bounds it: r, a, dh, dr and the gate read once, dx, da and dgate written once.
//
// A row's tensors stay in registers between the sums over it: of g2 xh2, then (from D) of g1 xh1.  The
// weights' four sums stay in registers too, one for each place and step, over all rows that a team takes; at the
// end the teams' are added in order and each workgroup leaves a part.  The gate's gradient sums a channel's
// coefficients, which lie on neighbouring places, through LDS.
#pragma once

#include <algorithm>

#include "gtp_res_row.hpp"

namespace gtp {
namespace {

template <typename T, int V, int NI, int W, bool K1>
__global__ __launch_bounds__(W ? kTeamThreads : 512) void k_res_backward(const ResArgs a, const ResWeights w, int A,
                                                                         float* __restrict__ partial) {
  // ResTables, then for each team its gate [NI A V / K] and its elements [NI A V], then a workgroup's Team
  extern __shared__ __align__(16) float lds[];
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V;
  const int t = W ? threadIdx.x % (W ? W : 1) : threadIdx.x, team = W ? threadIdx.x / (W ? W : 1) : 0;
  const int TEAMS = W ? kTeamThreads / (W ? W : 1) : 1;
  const Places<V> pl(A, K, C, t);
  const ResTables tab(lds, L, C);
  const int room = NI * pl.cpc;
  float* const gates = lds + ResTables::floats(L, C) + team * room;
  float* const all = lds + ResTables::floats(L, C) + TEAMS * room;
  float* const el = all + team * NI * AV;
  const Team<W, V, K1> us(pl, A, K, C, L, t, all + TEAMS * NI * AV);
  lds_poison(lds, int(ResTables::floats(L, C) + TEAMS * (room + NI * AV) + Team<W, V, K1>::floats(A, K, L)));
  tab.load(w, L);
  __syncthreads();
  int chan[V];
#pragma unroll
  for (int j = 0; j < V; ++j) chan[j] = pl.at[j] - pl.deg[j] * (C | 1);
  const T* const gate = static_cast<const T*>(a.gate);
  auto there = [&](int i, int j) { return i < NI - 1 || i * AV + V * t + j < R; };
  constexpr int Z = K1 ? V : 1;  // places of degree 0
  float e1[NI][V], e2[NI][V], f0[NI][Z], g0[NI][Z];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) e1[i][j] = e2[i][j] = 0.0f;
#pragma unroll
    for (int j = 0; j < Z; ++j) f0[i][j] = g0[i][j] = 0.0f;
  }
  for (int64_t n0 = int64_t(blockIdx.x) * TEAMS; n0 < a.N; n0 += int64_t(gridDim.x) * TEAMS) {
    const bool mine = n0 + team < a.N;
    const int64_t n = mine ? n0 + team : a.N - 1;
    RowRegs<T, V, NI> rv, dv, qv, av, gv;
    float mu2 = 0.0f, r2[V], mu1 = 0.0f, r1[V];
    if (pl.on) {
      rv.load(static_cast<const T*>(a.x) + n * R, t, AV, R);
      dv.load(static_cast<const T*>(a.dh) + n * R, t, AV, R);
      if (a.dr) qv.load(static_cast<const T*>(a.dr) + n * R, t, AV, R);
      av.load(static_cast<const T*>(a.a) + n * R, t, AV, R);
      if (K1 && gate) gv.load(gate + n * R, t, AV, R);
      mu2 = a.mean2[n];
      if (w.post) mu1 = a.mean1[n];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        r2[j] = a.rstd2[n * (L + 1) + (K1 ? 0 : pl.deg[j])];
        r1[j] = w.post ? a.rstd1[n * (L + 1) + (K1 ? 0 : pl.deg[j])] : 1.0f;
      }
      rv.fix(t, AV, R);
      dv.fix(t, AV, R);
      if (a.dr) qv.fix(t, AV, R);
      av.fix(t, AV, R);
      if (K1 && gate) gv.fix(t, AV, R);
    }
    const float one = mine ? 1.0f : 0.0f;  // a team without a row of its own adds nothing to the weights' sums
    float q[V], s = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = 0.0f;
    auto xh2 = [&](int i, int j) { return (us.at_zero(j) ? rv(i, j) - mu2 : rv(i, j)) * r2[j]; };
    auto xh1 = [&](int i, int j) { return (us.at_zero(j) ? av(i, j) - mu1 : av(i, j)) * r1[j]; };
    if (pl.on) {
      const int cpc = renewed(pl.cpc);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = dv(i, j), x = xh2(i, j);  // d is zero past the row's end
          const float g = there(i, j) ? d * tab.W2[pl.at[j] + i * cpc] : 0.0f;
          q[j] = fmaf(g, x, q[j]);
          e2[i][j] = fmaf(mine ? d : 0.0f, x, e2[i][j]);
          if (us.at_zero(j)) {
            s += g;
            g0[i][K1 ? j : 0] = fmaf(d, one, g0[i][K1 ? j : 0]);
          }
        }
    }
    float m2[V], mg2, m1[V], mg1;
    us.means(q, s, m2, mg2);
    if (!K1 && gate) {
      for (int c = t; c < C; c += W ? W : int(blockDim.x)) gates[c] = sigmoid(ld(gate, n * C + c));
      us.meet();
    }
    s = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = 0.0f;
    float g1[NI][V];
    if (pl.on) {
      const int cpc = renewed(pl.cpc);
      rv.renewed();
      dv.renewed();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float o[V], u[V], v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int c = chan[j] + i * cpc;
          const bool zero = us.at_zero(j);
          const float g = dv(i, j) * tab.W2[pl.at[j] + i * cpc];
          const float d = (a.dr ? qv(i, j) : 0.0f) + r2[j] * (g - xh2(i, j) * m2[j] - (zero ? mg2 : 0.0f));
          o[j] = d;
          const float p = tab.P[pl.at[j] + i * cpc], y = xh1(i, j);
          float open = 1.0f, x = 1.0f;
          if (gate) {
            if constexpr (K1) {
              x = gv(i, j);
              open = sigmoid(x);
            } else {
              open = gates[c];
            }
          }
          const bool in = there(i, j);
          const float uo = in && mine ? d * open : 0.0f;
          e1[i][j] = fmaf(uo, y, e1[i][j]);
          const float full = d * p;
          v[j] = fmaf(full, y, zero ? d * tab.Q[c] : 0.0f);  // D s t
          if constexpr (K1) v[j] *= open * sigmoid(-x);
          u[j] = in ? full * open : 0.0f;
          g1[i][j] = u[j];
          q[j] = fmaf(u[j], y, q[j]);
          if (zero) {
            s += u[j];
            f0[i][K1 ? j : 0] += uo;
          }
        }
        if (mine && a.dx) step_store<false, T, V>(static_cast<T*>(a.dx) + n * R, i * AV + V * t, R, o);
        if (a.dgate) {
          if constexpr (K1) {
            if (mine) step_store<false, T, V>(static_cast<T*>(a.dgate) + n * R, i * AV + V * t, R, v);
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) el[i * AV + V * t + j] = v[j];
          }
        }
        if (!w.post && mine && a.da) step_store<false, T, V>(static_cast<T*>(a.da) + n * R, i * AV + V * t, R, u);
      }
    }
    const bool norm1 = w.post && a.da;
    if (norm1) us.means(q, s, m1, mg1);  // a workgroup's first barrier: the elements are there
    if (!K1 && a.dgate) {
      if (W || !norm1) us.meet();
      for (int c = t; c < C; c += W ? W : int(blockDim.x)) {
        float v = 0.0f;
        for (int k = 0, m = c % K; k < K; ++k, m = m + 1 < K ? m + 1 : 0) v += el[c * K + m];  // turned: spread over the banks
        const float x = ld(gate, n * C + c);
        if (mine) st(static_cast<T*>(a.dgate), n * C + c, sigmoid(x) * sigmoid(-x) * v);
      }
    }
    if (norm1 && pl.on && mine) {
      av.renewed();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j)
          o[j] = r1[j] * (g1[i][j] - xh1(i, j) * m1[j] - (us.at_zero(j) ? mg1 : 0.0f));
        step_store<false, T, V>(static_cast<T*>(a.da) + n * R, i * AV + V * t, R, o);
      }
    }
  }
  if (!partial) return;
  float* const out = partial + int64_t(blockIdx.x) * res_columns(L, C);
  // E1 and E2, then F and G, each through the teams' elements
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    if (pl.on)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) el[i * AV + V * t + j] = which ? e2[i][j] : e1[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < (L + 1) * C; c += int(blockDim.x)) {
      const int l = c / C, ch = c - l * C;
      float v = 0.0f;
      for (int k = 0; k < TEAMS; ++k)
        for (int m = 0; m < 2 * l + 1; ++m) v += all[k * NI * AV + ch * K + l * l + m];
      out[which * (L + 1) * C + c] = v;
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    if (pl.on)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (us.at_zero(j)) el[K1 ? i * AV + V * t + j : i * pl.cpc + pl.ch] = which ? g0[i][K1 ? j : 0] : f0[i][K1 ? j : 0];
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += int(blockDim.x)) {
      float v = 0.0f;
      for (int k = 0; k < TEAMS; ++k) v += all[k * NI * AV + c];
      out[(2 * (L + 1) + which) * C + c] = v;
    }
  }
}

// Workgroups: two rows a team at least, where they fill the chip at all, since every workgroup leaves a part of the
// weights' gradients.
inline int64_t res_grid(int64_t N, const ResLay& y) {
  const int64_t rows = (N + y.teams() - 1) / y.teams(), n = std::min<int64_t>(rows, 256 * 8 / (y.threads / 64));
  const int64_t half = (rows + 1) / 2;
  return n <= half ? n : std::max<int64_t>(half, std::min<int64_t>(n, 256));
}

struct Backward {
  const ResArgs& a;
  const ResLay& y;
  hipStream_t s;
  template <typename T, int V, int NI, int W, bool K1>
  hipError_t operator()() const {
    const int64_t K = int64_t(a.L + 1) * (a.L + 1), teams = y.teams(), AV = int64_t(y.A) * V;
    const size_t lds = size_t(ResTables::floats(a.L, a.C) + teams * NI * (AV / K + AV) + Team<W, V, K1>::floats(y.A, K, a.L)) * 4;
    k_res_backward<T, V, NI, W, K1><<<uint32_t(res_grid(a.N, y)), y.threads, lds, s>>>(
        a, ResWeights(a), y.A, a.weights() ? a.work : nullptr);
    return hipGetLastError();
  }
};

}  // namespace

// Of one type each, a file of its own.
hipError_t launch_res_backward_f32(const ResArgs& a, const ResLay& y, hipStream_t s);
hipError_t launch_res_backward_bf16(const ResArgs& a, const ResLay& y, hipStream_t s);

}  // namespace gtp
