// The residual step's gradient, rows in registers (formulas in gtp_res.hpp, rows and teams in
// gtp_res_row.hpp).  HBM bounds it: r, a, dh, dr and the gate read once, dx, da and dgate written once.
//
// A row's tensors stay in registers between the sums over it: of g2 xh2, then (from D) of g1 xh1.  The
// weights' four sums stay in registers too, one for each place and step, over all rows that a team takes; at the
// end the teams' are added in order and each workgroup leaves a part.  The gate's gradient sums a channel's
// coefficients, which lie on neighbouring places, through LDS.
//
// Measured with the sum of the parts: fp32, 8192 x 128 channels of degree 6 325 us (3.8 TB/s; 326 the kernel), 16384 of
// degree 3 191 us (4.3), of degree 1 54 us (4.1), 65536 x 256 scalars 118 us (4.5); 1728 x 256 of degree 2 44 us (37 and 5).
// What bounds it is the registers: an element takes seven of 32 bits (four tensors, two sums, g1), so a SIMD holds one
// or two waves, whose barriers, LDS reads and loads nothing else hides; vector unit 40 % busy.  In bf16 an element takes
// as many instructions for half the bytes: 16384 x 128 of degree 3 184 us (2.2 TB/s), 50001 x 500 scalars 86 us (3.5).
#pragma once

#include <algorithm>

#include "gtp_res_row.hpp"

namespace gtp {
namespace {

typedef float f32v4 __attribute__((ext_vector_type(4)));

template <typename T, int V, int NI, int W, bool K1, int MAXT>
__global__ __launch_bounds__(MAXT) void k_res_backward(const ResArgs a, const ResWeights w, int A,
                                                                         float* __restrict__ partial) {
  // ResTables, then for each team the sigmoids of its gate and of minus it, of two rows in turn [4 (NI A V / K + 1)], then
  // (16-byte aligned) its elements [NI A V], then a workgroup's Team
  extern __shared__ __align__(16) float lds[];
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V;
  const int t = W ? threadIdx.x % (W ? W : 1) : threadIdx.x, team = W ? threadIdx.x / (W ? W : 1) : 0;
  constexpr int TEAMS = W ? kTeamThreads / (W ? W : 1) : 1;
  const Spots<V, K1> pl(A, K, t);
  const int channels = NI * pl.cpc, tables = int(ResTables::floats(NI * AV, channels)), room = 4 * (channels + 1);
  const ResTables tab(lds, NI * AV, channels);
  float* gates = lds + tables + team * room;
  int turn = 2 * (channels + 1);
  float* const all = lds + (tables + TEAMS * room + 3) / 4 * 4;
  float* const el = all + team * NI * AV;
  const Team<W, V, K1> us(pl, A, K, C, L, t, all + TEAMS * NI * AV);
  lds_poison(lds, int((tables + TEAMS * room + 3) / 4 * 4 + TEAMS * NI * AV + Team<W, V, K1>::floats(A, K, L)));
  const T* const gate = static_cast<const T*>(a.gate);
  const int lanes = W ? W : int(blockDim.x);
  auto there = [&](int i, int j) { return i < NI - 1 || i * AV + V * t + j < R; };
  const int64_t stride = int64_t(gridDim.x) * TEAMS;
  RowRegs<T, V, NI> rv, dv, qv, av;
  RowGate<T, V, NI, K1> gv;
  float mu2, mu1 = 0.0f, r2[V], r1[V];
#pragma unroll
  for (int j = 0; j < V; ++j) r1[j] = 1.0f;
  // Loads always (under a condition they would be waited for): a row's, as soon as the one before is done with the registers.
  auto clamped = [&](int64_t n) { return n < a.N ? n : a.N - 1; };
  auto load = [&](int64_t n) {
    n = clamped(n);
    rv.load(static_cast<const T*>(a.x) + n * R, t, AV, R);
    dv.load(static_cast<const T*>(a.dh) + n * R, t, AV, R);
    if (a.dr) qv.load(static_cast<const T*>(a.dr) + n * R, t, AV, R);
    if (gate) gv.load(gate + n * C, t, AV, C, lanes);
    mu2 = a.mean2[n];
#pragma unroll
    for (int j = 0; j < V; ++j) r2[j] = a.rstd2[n * (L + 1) + pl.deg[j]];
  };
  auto load_a = [&](int64_t n) {
    n = clamped(n);
    av.load(static_cast<const T*>(a.a) + n * R, t, AV, R);
    if (w.post) {
      mu1 = a.mean1[n];
#pragma unroll
      for (int j = 0; j < V; ++j) r1[j] = a.rstd1[n * (L + 1) + pl.deg[j]];
    }
  };
  load(int64_t(blockIdx.x) * TEAMS + team);
  load_a(int64_t(blockIdx.x) * TEAMS + team);
  tab.template load<V, NI, TEAMS, K1>(w, pl, A, t, team);
  __syncthreads();
  constexpr int Z = K1 ? V : 1;  // places of degree 0
  float e1[NI][V], e2[NI][V], f0[NI][Z], g0[NI][Z];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) e1[i][j] = e2[i][j] = 0.0f;
#pragma unroll
    for (int j = 0; j < Z; ++j) f0[i][j] = g0[i][j] = 0.0f;
  }
  const bool norm1 = w.post && a.da;
  constexpr bool KEEP = sizeof(T) == 4;  // what is made of an element takes its register; of bf16 ones it is made again
  for (int64_t n0 = int64_t(blockIdx.x) * TEAMS; n0 < a.N; n0 += stride) {
    const bool mine = n0 + team < a.N;
    const int64_t n = n0 + team;
    const int end = pl.on ? R : 0;
    if (W && !mine) {  // zeros instead of the last row, loaded again: it adds nothing to the weights' sums, infinite or not
      rv.clear(), dv.clear(), qv.clear(), av.clear();
      mu2 = mu1 = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j) r2[j] = r1[j] = 0.0f;
    }
    rv.fix(t, AV, end);
    dv.fix(t, AV, end);
    float off2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) off2[j] = pl.zero(j, mu2);
    if (!K1 && gate) {
      // the row before's may still be read by others of a workgroup; the ones of the row before that, behind
      // barriers, not
      gates += turn;
      turn = -turn;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (t + i * lanes < C) {
          gates[t + i * lanes] = sigmoid(gv.own[i]);
          gates[channels + 1 + t + i * lanes] = sigmoid(-gv.own[i]);
        }
      if (W) us.meet();  // a workgroup's first means meet
    }
    float q[V], q0[V];
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = q0[j] = 0.0f;
    if (pl.on) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float p[V], d[V];
        read_table<V>(tab.W2 + i * AV + V * t, p);
#pragma unroll
        for (int j = 0; j < V; ++j) {  // dh, and the tables, are zero past the row's end
          d[j] = dv(i, j);
          const float x = (rv(i, j) - off2[j]) * r2[j], g = d[j] * p[j];
          q[j] = fmaf(g, x, q[j]);
          q0[j] += g;
          e2[i][j] = fmaf(d[j], x, e2[i][j]);
          rv.set(i, j, x);
          dv.set(i, j, g);
          if constexpr (K1) g0[i][j] += d[j];
        }
        if constexpr (!K1) g0[i][0] += pl.sum_zero(d);
      }
    }
    float m2[V], mg2, m1[V], mg1;
    us.means(q, pl.sum_zero(q0), m2, mg2);
    if (a.dr) qv.fix(t, AV, end);
    av.fix(t, AV, end);
    if (K1 && gate) gv.row.fix(t, AV, end);
    float mz[V], off1[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      q[j] = q0[j] = 0.0f;
      mz[j] = pl.zero(j, mg2);
      off1[j] = pl.zero(j, mu1);
    }
    float g1[NI][V];
    if (pl.on) {
      rv.renewed();
      dv.renewed();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float o[V], u[V], v[V], p[V], p2[V], b[V], open[V], shut[V];
        if constexpr (!KEEP) read_table<V>(tab.W2 + i * AV + V * t, p2);
        read_table<V>(tab.P + i * AV + V * t, p);
        if constexpr (K1) {
          read_table<V>(tab.Q + i * AV + V * t, b);
        } else {
          const float shift = tab.Q[pl.ch + i * pl.cpc];
#pragma unroll
          for (int j = 0; j < V; ++j) b[j] = pl.zero(j, shift);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) open[j] = shut[j] = 1.0f;
        if (gate) {
          if constexpr (K1) {
#pragma unroll
            for (int j = 0; j < V; ++j) open[j] = sigmoid(gv.row(i, j)), shut[j] = sigmoid(-gv.row(i, j));
          } else {
            const float lo = gates[pl.ch0 + i * pl.cpc], up = gates[pl.ch0 + i * pl.cpc + 1];
#pragma unroll
            for (int j = 0; j < V; ++j) open[j] = (pl.next >> j) & 1u ? up : lo;
          }
        }
        float uo[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float x = KEEP ? rv(i, j) : (rv(i, j) - off2[j]) * r2[j], g = KEEP ? dv(i, j) : dv(i, j) * p2[j];
          const float y = (av(i, j) - off1[j]) * r1[j];
          o[j] = fmaf(r2[j], g - fmaf(x, m2[j], mz[j]), a.dr ? qv(i, j) : 0.0f);
          const float d = there(i, j) ? o[j] : 0.0f;
          uo[j] = there(i, j) ? d * open[j] : 0.0f;
          u[j] = uo[j] * p[j];
          e1[i][j] = fmaf(uo[j], y, e1[i][j]);
          v[j] = d * fmaf(p[j], y, b[j]);  // D s t
          if constexpr (K1) {
            v[j] *= open[j] * shut[j];
            f0[i][j] += uo[j];
          }
          g1[i][j] = u[j];
          av.set(i, j, y);
          q[j] = fmaf(u[j], y, q[j]);
          q0[j] += u[j];
        }
        if constexpr (!K1) f0[i][0] += pl.sum_zero(uo);
        if (mine && a.dx) step_store<false, T, V>(static_cast<T*>(a.dx) + n * R, i * AV + V * t, R, o);
        if (a.dgate) {
          if constexpr (K1) {
            if (mine) step_store<false, T, V>(static_cast<T*>(a.dgate) + n * R, i * AV + V * t, R, v);
          } else {
#pragma unroll
            for (int j = 0; j < V; j += 4)
              *reinterpret_cast<f32v4*>(el + i * AV + V * t + j) = f32v4{v[j], v[j + 1], v[j + 2], v[j + 3]};
          }
        }
        if (!w.post && mine && a.da) step_store<false, T, V>(static_cast<T*>(a.da) + n * R, i * AV + V * t, R, u);
      }
    }
    load(n + stride);  // the next row's, in flight meanwhile
    if (norm1) us.means(q, pl.sum_zero(q0), m1, mg1);  // a workgroup's first barrier: the elements are there
    if (!K1 && a.dgate) {
      if (W || !norm1) us.meet();
      for (int c = t; c < C; c += W ? W : int(blockDim.x)) {
        float v = 0.0f;
        int m = c & ((K & -K) - 1);  // an even K's turned against each other: spread over the banks
#pragma unroll 4
        for (int k = 0; k < K; ++k, m = m + 1 < K ? m + 1 : 0) v += el[c * K + m];
        if (mine) st(static_cast<T*>(a.dgate), n * C + c, gates[c] * gates[channels + 1 + c] * v);
      }
    }
    if (norm1 && pl.on && mine) {
      av.renewed();
#pragma unroll
      for (int j = 0; j < V; ++j) mz[j] = pl.zero(j, mg1);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float y = KEEP ? av(i, j) : (av(i, j) - off1[j]) * r1[j];
          o[j] = r1[j] * (g1[i][j] - fmaf(y, m1[j], mz[j]));
        }
        step_store<false, T, V>(static_cast<T*>(a.da) + n * R, i * AV + V * t, R, o);
      }
    }
    load_a(n + stride);
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
          if (K1 || j == pl.j0) el[K1 ? i * AV + V * t + j : i * pl.cpc + pl.ch] = which ? g0[i][K1 ? j : 0] : f0[i][K1 ? j : 0];
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += int(blockDim.x)) {
      float v = 0.0f;
      for (int k = 0; k < TEAMS; ++k) v += all[k * NI * AV + c];
      out[(2 * (L + 1) + which) * C + c] = v;
    }
  }
}

// Workgroups: as many as the CUs hold at once (each makes the tables and leaves a part of the weights' gradients), and
// two rows a team at least, where that fills the chip.  50001 rows of 500 scalars, bf16, 2 steps of a wave: 512 workgroups
// 100 us, 768 86, 1024 110 (three fit a CU: 146 registers a lane, and 49 KB of LDS each with the room for gates that scalars leave unused).
inline int64_t res_grid(int64_t N, const ResLay& y) {
  const int64_t rows = (N + y.teams() - 1) / y.teams();
  const int64_t n = std::min<int64_t>(rows, y.threads > kTeamThreads || y.NI > 4 ? 256 : y.NI > 2 ? 512 : 768),
                half = (rows + 1) / 2;
  return n <= half ? n : std::max<int64_t>(half, std::min<int64_t>(n, 256));
}

struct Backward {
  const ResArgs& a;
  const ResLay& y;
  hipStream_t s;
  template <typename T, int V, int NI, int W, bool K1>
  hipError_t operator()() const {
    const size_t lds = size_t(res_lds(y, int64_t(a.L + 1) * (a.L + 1), a.L, true));
    auto k = k_res_backward<T, V, NI, W, K1, kTeamThreads>;
    if constexpr (W == 0)
      if (y.threads > kTeamThreads) k = k_res_backward<T, V, NI, W, K1, 512>;
    k<<<uint32_t(res_grid(a.N, y)), y.threads, lds, s>>>(a, ResWeights(a), y.A, a.weights() ? a.work : nullptr);
    return hipGetLastError();
  }
};

}  // namespace

// Of one type each, a file of its own.
hipError_t launch_res_backward_f32(const ResArgs& a, const ResLay& y, hipStream_t s);
hipError_t launch_res_backward_bf16(const ResArgs& a, const ResLay& y, hipStream_t s);

}  // namespace gtp
