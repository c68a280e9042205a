// The residual step, forward, rows in registers (formulas in gtp_res.hpp, rows and teams in
// gtp_res_row.hpp).  HBM bounds it: x, a and the gate read once, r and h written once.
//
// Measured (copies on this chip: 5.5 TB/s): fp32 rows of 128 channels, 16384 of degree 1 28.8 us (4.95 TB/s), of degree
// 3 117 us (4.7), of degree 6 377 us (4.4); 64 channels of degree 8 277 us (4.9); 65536 rows of 256 scalars 69 us (4.9);
// bf16, 32768 x 128 of degree 6, no norm behind the part: 419 us (3.9: twice as many elements a byte, some 20 vector
// instructions each, and every second workgroup of the CU in a barrier).  1728 x 256 of degree 2: 25 us (2.6), seven rows a
// CU, a load, two sums and a store one after the other; 27 rows: 9.7 us, of which a launch is 3 and the tables 2.
#include <algorithm>

#include "gtp_res_row.hpp"

namespace gtp {
namespace {

template <typename T, int V, int NI, int W, bool K1>
__global__ __launch_bounds__(W ? kTeamThreads : 512) void k_res(const ResArgs a, const ResWeights w, int A) {
  // ResTables, then for each team its gate [NI A V / K + 1], then a workgroup's Team
  extern __shared__ __align__(16) float lds[];
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V;
  const int t = W ? threadIdx.x % (W ? W : 1) : threadIdx.x, team = W ? threadIdx.x / (W ? W : 1) : 0;
  constexpr int TEAMS = W ? kTeamThreads / (W ? W : 1) : 1;
  const Spots<V, K1> pl(A, K, t);
  const int channels = NI * pl.cpc, tables = int(ResTables::floats(NI * AV, channels));
  const ResTables tab(lds, NI * AV, channels);
  float* const gates = lds + tables + team * (channels + 1);
  const Team<W, V, K1> us(pl, A, K, C, L, t, lds + tables + TEAMS * (channels + 1));
  lds_poison(lds, int(tables + TEAMS * (channels + 1) + Team<W, V, K1>::floats(A, K, L)));
  const T* const gate = static_cast<const T*>(a.gate);
  const int lanes = W ? W : int(blockDim.x);
  auto there = [&](int i, int j) { return i < NI - 1 || i * AV + V * t + j < R; };
  const int64_t stride = int64_t(gridDim.x) * TEAMS;
  RowRegs<T, V, NI> av, xv;
  RowGate<T, V, NI, K1> gv;
  auto load = [&](int64_t n) {
    n = n < a.N ? n : a.N - 1;  // always: a load under a condition would be waited for
    av.load(static_cast<const T*>(a.a) + n * R, t, AV, R);
    xv.load(static_cast<const T*>(a.x) + n * R, t, AV, R);
    if (gate) gv.load(gate + n * C, t, AV, C, lanes);
  };
  // the first row in flight while the tables are made, where the registers hold both
  constexpr bool FIRST = W > 0 || NI * V < 16;
  if (FIRST) load(int64_t(blockIdx.x) * TEAMS + team);
  tab.template load<V, NI, TEAMS, K1>(w, pl, A, t, team);
  __syncthreads();
  for (int64_t n0 = int64_t(blockIdx.x) * TEAMS; n0 < a.N; n0 += stride) {
    const bool mine = n0 + team < a.N;
    const int64_t n = n0 + team;
    if (!FIRST) load(n);
    av.fix(t, AV, pl.on ? R : 0);
    xv.fix(t, AV, pl.on ? R : 0);
    if (K1 && gate) gv.row.fix(t, AV, pl.on ? R : 0);
    if (!K1 && gate)  // a workgroup's barriers since the row before's use of them stand in its second statistics
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (t + i * lanes < C) gates[t + i * lanes] = sigmoid(gv.own[i]);
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
    float rv[NI][V], off[V];
#pragma unroll
    for (int j = 0; j < V; ++j) off[j] = pl.zero(j, mu1);
    if (pl.on) {
      av.renewed();
      xv.renewed();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float o[V], p[V], q[V], g[V];
        read_table<V>(tab.P + i * AV + V * t, p);
        if constexpr (K1) {
          read_table<V>(tab.Q + i * AV + V * t, q);
        } else {
          const float q0 = tab.Q[pl.ch + i * pl.cpc];
#pragma unroll
          for (int j = 0; j < V; ++j) q[j] = pl.zero(j, q0);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = 1.0f;
        if (gate) {
          if constexpr (K1) {
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = sigmoid(gv.row(i, j));
          } else {
            const float lo = gates[pl.ch0 + i * pl.cpc], up = gates[pl.ch0 + i * pl.cpc + 1];
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = (pl.next >> j) & 1u ? up : lo;
          }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float s = fmaf((av(i, j) - off[j]) * r1[j], p[j], q[j]);
          o[j] = rv[i][j] = there(i, j) ? fmaf(g[j], s, xv(i, j)) : 0.0f;
        }
        if (mine) step_store<false, T, V>(static_cast<T*>(a.r) + n * R, i * AV + V * t, R, o);
      }
    }
    if (FIRST) load(n + stride);  // the next row's, in flight meanwhile
    float mu2, r2[V];
    us.template statistics<NI>([&](int i, int j) { return rv[i][j]; }, there, a.eps, mu2, r2, [&](int l, float v) {
      if (a.rstd2 && mine) a.rstd2[n * (L + 1) + l] = v;
    });
    if (!mine) continue;  // the last turn
    if (a.mean2 && t == 0) a.mean2[n] = mu2;
    if (!pl.on) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) off[j] = pl.zero(j, mu2);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float o[V], p[V], q[V];
      read_table<V>(tab.W2 + i * AV + V * t, p);
      if constexpr (K1) {
        read_table<V>(tab.B2 + i * AV + V * t, q);
      } else {
        const float b0 = tab.B2[pl.ch + i * pl.cpc];
#pragma unroll
        for (int j = 0; j < V; ++j) q[j] = pl.zero(j, b0);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = fmaf((rv[i][j] - off[j]) * r2[j], p[j], q[j]);
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
    const size_t lds = size_t(res_lds(y, K, a.L, false));
    // workgroups that the CUs hold at once, by the registers that a row's elements take: each makes the tables (12927 x 21
    // of degree 8, fp32: four 99 us, six 115)
    const int64_t held = std::clamp<int64_t>(12 / std::max(1, NI * V * int(sizeof(T)) / 16), 1, 4);
    const int64_t fill = 256 * std::max<int64_t>(1, held * kTeamThreads / y.threads);
    k_res<T, V, NI, W, K1><<<uint32_t(std::min(rows, fill)), y.threads, lds, s>>>(a, ResWeights(a), y.A);
    return hipGetLastError();
  }
};

bool wide16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

constexpr int64_t kMaxLds = 150 << 10;

// LDS bytes of a layout; back: the gradient's, which has the teams' elements besides.  The gates' room is counted for every
// row, also for scalars, whose gates lie in registers: that, not the registers, ends their layouts at 7168 scalars, gradient
// 4096.
int64_t res_lds(const ResLay& y, int64_t K, int L, bool back) {
  const int64_t AV = int64_t(y.A) * y.V, elements = y.NI * AV, channels = elements / K;
  const int64_t block = y.W ? 0 : (K == 1 ? 2 * int64_t(y.A) : AV + AV / K) + L + 2;
  return (ResTables::floats(elements, channels) + y.teams() * ((back ? 4 : 1) * (channels + 1) + (back ? elements : 0)) + 4 + block) * 4;
}

bool residual_layout(const ResArgs& a, bool wide, bool back, ResLay* out) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1), R = a.C * K;
  if (R >= (int64_t(1) << 30) || R < 8) return false;
  // one coefficient of degree 0 in a group at most
  const int V = !back && a.bf16 && wide && R % 8 == 0 && (K == 1 || K >= 8) ? 8 : 4;
  int64_t g = V;
  while (K % g) g /= 2;
  const int64_t unit = K / g;  // A is a multiple of it
  auto fits = [&](const ResLay& y) { return res_lds(y, K, a.L, back) <= kMaxLds; };
  // a wave's team, forward up to 6 steps: 16384 x 128 channels of degree 3 took 123 us in 8 steps of a wave, 117 in 2 of a
  // workgroup (backward 191 and 203)
  for (int W : {16, 64}) {
    const int64_t A = W / unit * unit, steps = A ? (R + A * V - 1) / (A * V) : 0;
    if (A == 0 || steps > (W == 16 ? 2 : back || V == 8 ? 32 / V : 6)) continue;
    const ResLay y{W, V, int(steps), int(A), kTeamThreads};
    if (fits(y)) return *out = y, true;
  }
  double best = 0.0;
  for (int64_t threads : {256, 512}) {
    const int64_t A = threads / unit * unit, steps = A ? (R + A * V - 1) / (A * V) : 0;
    if (A == 0 || steps > 32 / V) continue;
    const ResLay y{0, V, int(steps), int(A), int(threads)};
    // the share of lanes and steps at work, less where a workgroup's registers leave the CU no second one (of 256
    // threads; of 512, no second wave on a SIMD): 6272 elements, fp32, backward: 355 us on 512 threads in 4 steps, 450 on 256
    // in 7; bf16, forward: 383 on 512 in 2 steps of 8, 473 on 256 in 4.  Even 512 threads in 5 to 8 steps, which spill, are ahead
    // of a row that is read for each pass: 4000 x 9720 elements, fp32, backward 384 us in 5 (1193), 10368 in 6 513 (1450), bf16
    // 269 and 391 (1022 and 1304)
    const int64_t few = back ? (threads > kTeamThreads ? 4 : 3) : (threads > kTeamThreads ? 16 : 20) / V;
    const double use = double(R) / (double(threads) * V * double(steps)) *
                       (threads > kTeamThreads ? 0.95 : 1.0) * (steps <= few ? 1.0 : back && threads > kTeamThreads ? 0.5 : 0.75);
    if (use > best * 1.02 && fits(y)) best = use, *out = y;
  }
  return best > 0.0;
}

hipError_t launch_residual(const ResArgs& a, hipStream_t s) {
  ResLay y;
  if (!residual_layout(a, wide16(a.x) && wide16(a.a) && wide16(a.r) && wide16(a.h), false, &y))
    return residual_is_long(a) ? launch_residual_long(a, s) : launch_residual_any(a, s);
  const Forward f{a, y, s};
  if (!a.bf16) return a.L == 0 ? res_with_team<float, 4, true>(y, f) : res_with_team<float, 4, false>(y, f);
  if (y.V == 8) return a.L == 0 ? res_with_team<uint16_t, 8, true>(y, f) : res_with_team<uint16_t, 8, false>(y, f);
  return a.L == 0 ? res_with_team<uint16_t, 4, true>(y, f) : res_with_team<uint16_t, 4, false>(y, f);
}

}  // namespace gtp
