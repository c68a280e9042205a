// The residual step, forward, rows in registers (formulas in gtp_res.hpp, rows and teams in
// gtp_res_row.hpp).  HBM bounds it: x, a and the gate read once, r and h written once.
#include <algorithm>

#include "gtp_res_row.hpp"

namespace gtp {
namespace {

constexpr int64_t kMaxLds = 150 << 10;

template <typename T, int V, int NI, int W, bool K1>
__global__ __launch_bounds__(W ? kTeamThreads : 512) void k_res(const ResArgs a, const ResWeights w, int A) {
  // ResTables, then for each team its gate [NI A V / K], then a workgroup's Team
  extern __shared__ __align__(16) float lds[];
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V;
  const int t = W ? threadIdx.x % (W ? W : 1) : threadIdx.x, team = W ? threadIdx.x / (W ? W : 1) : 0;
  const int TEAMS = W ? kTeamThreads / (W ? W : 1) : 1;
  const Places<V> pl(A, K, C, t);
  const ResTables tab(lds, L, C);
  const int room = NI * pl.cpc;  // channels of all steps: C and what the last step has past them
  float* const gates = lds + ResTables::floats(L, C) + team * room;
  const Team<W, V, K1> us(pl, A, K, C, L, t, lds + ResTables::floats(L, C) + TEAMS * room);
  lds_poison(lds, int(ResTables::floats(L, C) + TEAMS * room + Team<W, V, K1>::floats(A, K, L)));
  tab.load(w, L);
  __syncthreads();
  int chan[V];
#pragma unroll
  for (int j = 0; j < V; ++j) chan[j] = pl.at[j] - pl.deg[j] * (C | 1);
  const T* const gate = static_cast<const T*>(a.gate);
  auto there = [&](int i, int j) { return i < NI - 1 || i * AV + V * t + j < R; };
  for (int64_t n0 = int64_t(blockIdx.x) * TEAMS; n0 < a.N; n0 += int64_t(gridDim.x) * TEAMS) {
    const bool mine = n0 + team < a.N;
    const int64_t n = mine ? n0 + team : a.N - 1;
    RowRegs<T, V, NI> av, xv, gv;
    if (pl.on) {
      av.load(static_cast<const T*>(a.a) + n * R, t, AV, R);
      xv.load(static_cast<const T*>(a.x) + n * R, t, AV, R);
      if (K1 && gate) gv.load(gate + n * R, t, AV, R);
      av.fix(t, AV, R);
      xv.fix(t, AV, R);
      if (K1 && gate) gv.fix(t, AV, R);
    }
    if (!K1 && gate)  // a workgroup's barriers since the row before's use of them stand in its second statistics
      for (int c = t; c < C; c += W ? W : int(blockDim.x)) gates[c] = sigmoid(ld(gate, n * C + c));
    float mu1 = 0.0f, r1[V];
#pragma unroll
    for (int j = 0; j < V; ++j) r1[j] = 1.0f;
    if (w.post) {
      us.template statistics<NI>([&](int i, int j) { return av(i, j); }, there, a.eps, mu1, r1, [&](int l, float v) {
        if (a.rstd1 && mine) a.rstd1[n * (L + 1) + l] = v;
      });
      if (a.mean1 && mine && t == 0) a.mean1[n] = mu1;
    }
    if (!K1 && gate && (W || !w.post)) us.meet();  // a workgroup's first statistics have met
    const int cpc = renewed(pl.cpc);
    float rv[NI][V];
    if (pl.on) {
      av.renewed();
      xv.renewed();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int c = chan[j] + i * cpc;
          const bool zero = us.at_zero(j);
          const float p = tab.P[pl.at[j] + i * cpc], f = zero ? av(i, j) - mu1 : av(i, j);
          const float s = fmaf(f * r1[j], p, zero ? tab.Q[c] : 0.0f);
          float g = 1.0f;
          if (gate) g = K1 ? sigmoid(gv(i, j)) : gates[c];
          o[j] = rv[i][j] = there(i, j) ? fmaf(g, s, xv(i, j)) : 0.0f;
        }
        if (mine) {
          T* const row = static_cast<T*>(a.r) + n * R;
          step_store<false, T, V>(row, i * AV + V * t, R, o);
        }
      }
    }
    float mu2, r2[V];
    us.template statistics<NI>([&](int i, int j) { return rv[i][j]; }, there, a.eps, mu2, r2, [&](int l, float v) {
      if (a.rstd2 && mine) a.rstd2[n * (L + 1) + l] = v;
    });
    if (!mine) continue;  // the last turn
    if (a.mean2 && t == 0) a.mean2[n] = mu2;
    if (!pl.on) continue;
    const int cpc2 = renewed(pl.cpc);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const bool zero = us.at_zero(j);
        o[j] = fmaf((zero ? rv[i][j] - mu2 : rv[i][j]) * r2[j], tab.W2[pl.at[j] + i * cpc2],
                    zero ? tab.B2[chan[j] + i * cpc2] : 0.0f);
      }
      step_store<false, T, V>(static_cast<T*>(a.h) + n * R, i * AV + V * t, R, o);
    }
  }
}

struct Forward {
  const ResArgs& a;
  const ResLay& y;
  hipStream_t s;
  template <typename T, int V, int NI, int W, bool K1>
  hipError_t operator()() const {
    const int64_t K = int64_t(a.L + 1) * (a.L + 1), teams = y.teams(), rows = (a.N + teams - 1) / teams;
    const size_t lds = size_t(ResTables::floats(a.L, a.C) + teams * NI * (y.A * V / K) + Team<W, V, K1>::floats(y.A, K, a.L)) * 4;
    const int64_t fill = 256 * 16 / (y.threads / 64);
    k_res<T, V, NI, W, K1><<<uint32_t(std::min(rows, fill)), y.threads, lds, s>>>(a, ResWeights(a), y.A);
    return hipGetLastError();
  }
};

bool wide16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

bool residual_layout(const ResArgs& a, bool wide, bool back, ResLay* out) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1), R = a.C * K;
  if (R >= (int64_t(1) << 30) || R < 8) return false;
  // one coefficient of degree 0 in a group at most
  const int V = !back && a.bf16 && wide && R % 8 == 0 && (K == 1 || K >= 8) ? 8 : 4;
  int64_t g = V;
  while (K % g) g /= 2;
  const int64_t unit = K / g;  // A is a multiple of it
  const int64_t tables = ResTables::floats(a.L, a.C) * 4;
  auto fits = [&](int64_t A, int64_t threads, int64_t teams, int64_t steps) {
    const int64_t AV = A * V;
    const int64_t team = (back ? steps * AV : 0) + steps * AV / K;
    const int64_t block = teams == 1 && threads != kTeamThreads / 64 ? AV + AV / K + A + a.L + 2 : 0;
    return tables + (teams * team + block) * 4 <= kMaxLds;
  };
  for (int W : {16, 64}) {
    const int64_t A = W / unit * unit, steps = A ? (R + A * V - 1) / (A * V) : 0;
    if (A == 0 || steps > (W == 16 ? 2 : 32 / V) || !fits(A, kTeamThreads, kTeamThreads / W, steps)) continue;
    *out = ResLay{W, V, int(steps), int(A), kTeamThreads};
    return true;
  }
  double best = 0.0;
  for (int64_t threads = 64; threads <= 512; threads += 64) {
    const int64_t A = threads / unit * unit, steps = A ? (R + A * V - 1) / (A * V) : 0;
    if (A == 0 || steps > 32 / V || !fits(A, threads, 1, steps)) continue;
    // the share of lanes and steps at work; more than 4 waves in step leave the barriers less to overlap
    const double use = double(R) / (double(threads) * V * double(steps)) * (threads > 256 ? 0.85 : 1.0);
    if (use > best * 1.02) best = use, *out = ResLay{0, V, int(steps), int(A), int(threads)};
  }
  return best > 0.0;
}

hipError_t launch_residual(const ResArgs& a, hipStream_t s) {
  ResLay y;
  if (!residual_layout(a, wide16(a.x) && wide16(a.a) && wide16(a.r) && wide16(a.h), false, &y))
    return launch_residual_any(a, s);
  const Forward f{a, y, s};
  if (!a.bf16) return a.L == 0 ? res_with_team<float, 4, true>(y, f) : res_with_team<float, 4, false>(y, f);
  if (y.V == 8) return a.L == 0 ? res_with_team<uint16_t, 8, true>(y, f) : res_with_team<uint16_t, 8, false>(y, f);
  return a.L == 0 ? res_with_team<uint16_t, 4, true>(y, f) : res_with_team<uint16_t, 4, false>(y, f);
}

}  // namespace gtp
