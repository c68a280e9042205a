// The residual step for rows that do not fit the registers of a workgroup (formulas in gtp_res.hpp): rows of
// degree 8 with some 150 channels and more.
//
// The same places as in gtp_res_row.hpp, so that every access is coalesced and a degree's sum lies in a thread's
// registers, but a row is read again for each pass, from the caches where they hold it.  Forward: the squares of a (its
// mean from its degree 0 alone), those of r, the results.  Backward: the means of g2 xh2, then of g1 xh1 with the gate's
// gradient; the weights' sums, by workgroups that walk down the rows in the places of one step; the rows'
// gradients: five reads of a tensor forward where rows in registers take two, fourteen backward for four, and weights
// gathered by channel.  1200 x 512 channels of degree 8, fp32: 593 us forward and 1330 backward (1.3 and 0.9 TB/s of what has
// to move; a degree at a time, gtp_res_any.hip: 1146 and 2922); bf16: 580 and 1205 (1008 and 2689), so that it is not the
// bytes that bound it but the gathers, four addresses a thread and table in every pass.
#include <algorithm>

#include "gtp_res_row.hpp"

namespace gtp {
namespace {

constexpr int V = 4, kThreads = 1024, kSteps = 2;  // steps whose loads are in flight together: with four, 128 registers a lane spill
typedef Spots<V, false> Place;
typedef Team<0, V, false> Block;

template <typename T>
using Row4 = typename Vec<T, V>::type;

// Weights of the thread's elements at step i: P = scale w1 and W2, gathered (the tables of (L + 1) C stay in the caches).
struct Gather {
  const ResWeights& w;
  const Place& at;
  __device__ int channel(int i, int j) const { return at.ch0 + int((at.next >> j) & 1u) + i * at.cpc; }
  __device__ int clamped(int i, int j) const {
    const int c = channel(i, j);
    return c < w.C ? c : int(w.C) - 1;
  }
  __device__ void read(const float* from, int i, float (&o)[V]) const {
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = from ? from[at.deg[j] * w.C + clamped(i, j)] : 1.0f;
  }
  __device__ void part(int i, float (&p)[V]) const {
    float q[V];
    read(w.scale, i, p);
    read(w.w1, i, q);
#pragma unroll
    for (int j = 0; j < V; ++j) p[j] *= q[j];
  }
  // shift [l = 0] times row 0 of `one`
  __device__ void shift(const float* b, const float* one, int i, float (&o)[V]) const {
    const int c = at.ch + i * at.cpc, in = c < w.C ? c : int(w.C) - 1;
    const float v = b ? b[in] * (one ? one[in] : 1.0f) : 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = at.zero(j, v);
  }
  template <typename T>
  __device__ void open(const T* gate, int i, float (&o)[V]) const {  // gate: the row's, or null
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = 1.0f;
    if (!gate) return;
    const float lo = sigmoid(ld(gate, clamped(i, 0))), up = sigmoid(ld(gate, clamped(i, V - 1)));
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = (at.next >> j) & 1u ? up : lo;
  }
};

// f(i, first element) for the thread's steps, kSteps of which load() issues the loads of at once.
template <typename F, typename G>
__device__ __forceinline__ void over_steps(int R, int AV, F load, G f) {
  const int steps = (R + AV - 1) / AV;
  for (int i0 = 0; i0 < steps; i0 += kSteps) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) load(i, i0 + i);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (i0 + i < steps) f(i, i0 + i);
  }
}

// A row's elements at kSteps steps.
template <typename T>
struct Steps {
  Row4<T> v[kSteps];
  __device__ void load(const T* row, int i, int step, int t, int AV, int R) { v[i] = step_load<T, V>(row, step * AV + V * t, R); }
  __device__ void get4(int i, int step, int t, int AV, int R, float (&o)[V]) {  // zeros past the row's end
    Row4<T> u = v[i];
    step_fix<false, T, V>(u, step * AV + V * t, R);
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = get<T, V>(u, j);
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_long(const ResArgs a, const ResWeights w, int A) {
  extern __shared__ float lds[];
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V, t = threadIdx.x;
  const Place pl(A, K, t);
  const Block us(pl, A, K, C, L, t, lds);
  lds_poison(lds, int(Block::floats(A, K, L)));
  const Gather g{w, pl};
  const int end = pl.on ? R : 0;
  for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
    const T* const ar = static_cast<const T*>(a.a) + n * R;
    const T* const xr = static_cast<const T*>(a.x) + n * R;
    const T* const gate = a.gate ? static_cast<const T*>(a.gate) + n * C : nullptr;
    float none[V], r1[V], r2[V], off[V], q[V], mu1 = 0.0f, mu2, unused;
#pragma unroll
    for (int j = 0; j < V; ++j) none[j] = off[j] = 0.0f, r1[j] = 1.0f;
    Steps<T> as, xs;
    auto size = [&](float* mean, float* rstd, float mu, float (&r)[V]) {  // 1 / size from the means of the squares
#pragma unroll
      for (int j = 0; j < V; ++j) r[j] = 1.0f / sqrtf(r[j] + a.eps);
      if (mean && t == 0) mean[n] = mu;
      if (rstd && t <= L) rstd[n * (L + 1) + t] = 1.0f / sqrtf(us.stat[t] + a.eps);
    };
    if (w.post) {
      float s = 0.0f;
      for (int c = t; c < C; c += kThreads) s += ld(ar, int64_t(c) * K);
      // the sum of every thread: thread t < A alone has a place in means()
      s = wave_sum(s);
      __syncthreads();
      if ((t & 63) == 0) lds[t >> 6] = s;
      __syncthreads();
      mu1 = 0.0f;
      for (int i = 0; i < kThreads / 64; ++i) mu1 += lds[i];
      mu1 /= float(C);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) off[j] = pl.zero(j, mu1), q[j] = 0.0f;
      over_steps(R, AV, [&](int i, int step) { as.load(ar, i, step, t, AV, R); },
                 [&](int i, int step) {
                   float v[V];
                   as.get4(i, step, t, AV, end, v);
#pragma unroll
                   for (int j = 0; j < V; ++j) {
                     const float d = step * AV + V * t + j < end ? v[j] - off[j] : 0.0f;
                     q[j] = fmaf(d, d, q[j]);
                   }
                 });
      us.means(q, 0.0f, r1, unused);
      size(a.mean1, a.rstd1, mu1, r1);
    }
    // r before its rounding
    auto load = [&](int i, int step) {
      as.load(ar, i, step, t, AV, R);
      xs.load(xr, i, step, t, AV, R);
    };
    auto sum = [&](int i, int step, float (&o)[V]) {
      float v[V], x[V], p[V], b[V], open[V];
      as.get4(i, step, t, AV, end, v);
      xs.get4(i, step, t, AV, end, x);
      g.part(step, p);
      g.shift(w.b1, w.scale, step, b);
      g.open(gate, step, open);
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = fmaf(open[j], fmaf((v[j] - off[j]) * r1[j], p[j], b[j]), x[j]);
    };
    float s = 0.0f;
    for (int c = t; c < C; c += kThreads) {
      const float v = (ld(ar, int64_t(c) * K) - mu1) * (w.post ? 1.0f / sqrtf(us.stat[0] + a.eps) : 1.0f);
      s += fmaf(gate ? sigmoid(ld(gate, c)) : 1.0f, fmaf(v, w.s(0, c) * w.post_w(0, c), w.s(0, c) * w.post_b(0, c)),
                ld(xr, int64_t(c) * K));
    }
    s = wave_sum(s);
    __syncthreads();
    if ((t & 63) == 0) lds[t >> 6] = s;
    __syncthreads();
    mu2 = 0.0f;
    for (int i = 0; i < kThreads / 64; ++i) mu2 += lds[i];
    mu2 /= float(C);
    __syncthreads();
    float off2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) off2[j] = pl.zero(j, mu2), q[j] = 0.0f;
    over_steps(R, AV, load, [&](int i, int step) {
      float o[V];
      sum(i, step, o);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = step * AV + V * t + j < end ? o[j] - off2[j] : 0.0f;
        q[j] = fmaf(d, d, q[j]);
      }
    });
    us.means(q, 0.0f, r2, unused);
    size(a.mean2, a.rstd2, mu2, r2);
    over_steps(R, AV, load, [&](int i, int step) {
      float o[V], p[V], b[V];
      sum(i, step, o);
      g.read(w.w2, step, p);
      g.shift(w.b2, nullptr, step, b);
      if (pl.on) step_store<false, T, V>(static_cast<T*>(a.r) + n * R, step * AV + V * t, R, o);
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = fmaf((o[j] - off2[j]) * r2[j], p[j], b[j]);
      if (pl.on) step_store<false, T, V>(static_cast<T*>(a.h) + n * R, step * AV + V * t, R, o);
    });
    __syncthreads();  // stat is read
  }
}

// What the backward's kernels read of a row, and D with what comes of it.
template <typename T>
struct LongBack {
  const ResArgs& a;
  const ResWeights& w;
  const Place& pl;
  Gather g;
  int t, AV, R, end;
  float off1[V], off2[V], r1[V], r2[V];
  Steps<T> rs, hs, ds, as;
  __device__ LongBack(const ResArgs& a_, const ResWeights& w_, const Place& p, int t_, int AV_, int R_)
      : a(a_), w(w_), pl(p), g{w_, p}, t(t_), AV(AV_), R(R_), end(p.on ? R_ : 0) {}
  __device__ void row(int64_t n) {
    const float mu2 = a.mean2[n], mu1 = w.post ? a.mean1[n] : 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      off2[j] = pl.zero(j, mu2);
      off1[j] = pl.zero(j, mu1);
      r2[j] = a.rstd2[n * (a.L + 1) + pl.deg[j]];
      r1[j] = w.post ? a.rstd1[n * (a.L + 1) + pl.deg[j]] : 1.0f;
    }
  }
  __device__ void load(int64_t n, int i, int step, bool first) {  // first: r and dh alone
    rs.load(static_cast<const T*>(a.x) + n * R, i, step, t, AV, R);
    hs.load(static_cast<const T*>(a.dh) + n * R, i, step, t, AV, R);
    if (first) return;
    if (a.dr) ds.load(static_cast<const T*>(a.dr) + n * R, i, step, t, AV, R);
    as.load(static_cast<const T*>(a.a) + n * R, i, step, t, AV, R);
  }
  // xh2 and g2 = dh w2 (and dh)
  __device__ void first(int i, int step, float (&x)[V], float (&gg)[V], float (&d)[V]) {
    float p[V];
    rs.get4(i, step, t, AV, end, x);
    hs.get4(i, step, t, AV, end, d);
    g.read(w.w2, step, p);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      x[j] = (x[j] - off2[j]) * r2[j];
      gg[j] = step * AV + V * t + j < end ? d[j] * p[j] : 0.0f;
    }
  }
  // D, xh1, the gate's sigmoid, P and the shift; D and the sigmoid zero past the row's end
  __device__ void second(int64_t n, int i, int step, const float (&x)[V], const float (&gg)[V], const float (&m2)[V],
                         float mg2, float (&d)[V], float (&y)[V], float (&open)[V], float (&p)[V], float (&b)[V]) {
    float q[V];
    as.get4(i, step, t, AV, end, y);
    if (a.dr) ds.get4(i, step, t, AV, end, q);
    g.part(step, p);
    g.shift(w.b1, w.scale, step, b);
    g.open(a.gate ? static_cast<const T*>(a.gate) + n * w.C : nullptr, step, open);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool in = step * AV + V * t + j < end;
      d[j] = fmaf(r2[j], gg[j] - fmaf(x[j], m2[j], pl.zero(j, mg2)), a.dr ? q[j] : 0.0f);
      d[j] = in ? d[j] : 0.0f;
      open[j] = in ? open[j] : 0.0f;
      y[j] = (y[j] - off1[j]) * r1[j];
    }
  }
};

// means[n]: [L + 2] of g2 xh2 by degree and g2 at degree 0, then as many of g1 xh1 and g1; and the gate's gradient.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_long_means(const ResArgs a, const ResWeights w, int A,
                                                             float* __restrict__ means) {
  extern __shared__ __align__(16) float lds[];  // kSteps steps' elements, then Block's
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V, t = threadIdx.x;
  const Place pl(A, K, t);
  const Block us(pl, A, K, C, L, t, lds + kSteps * AV);
  lds_poison(lds, kSteps * AV + int(Block::floats(A, K, L)));
  LongBack<T> b(a, w, pl, t, AV, R);
  for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
    b.row(n);
    float q[V], q0[V], m2[V], mg2, m1[V], mg1;
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = q0[j] = 0.0f;
    over_steps(R, AV, [&](int i, int step) { b.load(n, i, step, true); },
               [&](int i, int step) {
                 float x[V], g[V], d[V];
                 b.first(i, step, x, g, d);
#pragma unroll
                 for (int j = 0; j < V; ++j) q[j] = fmaf(g[j], x[j], q[j]), q0[j] += g[j];
               });
    us.means(q, pl.sum_zero(q0), m2, mg2);
    float* const out = means + n * 2 * (L + 2);
    if (t < L + 2) out[t] = us.stat[t];
    if (!w.post && !a.dgate) {
      __syncthreads();
      continue;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = q0[j] = 0.0f;
    const int steps = (R + AV - 1) / AV;
    for (int i0 = 0; i0 < steps; i0 += kSteps) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) b.load(n, i, i0 + i, false);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        float x[V], g[V], d[V], y[V], open[V], p[V], sh[V];
        b.first(i, i0 + i, x, g, d);
        b.second(n, i, i0 + i, x, g, m2, mg2, d, y, open, p, sh);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float u = d[j] * open[j] * p[j];
          q[j] = fmaf(u, y[j], q[j]);
          q0[j] += u;
          if (a.dgate && pl.on) lds[i * AV + V * t + j] = d[j] * fmaf(p[j], y[j], sh[j]);
        }
      }
      if (!a.dgate) continue;
      __syncthreads();
      // four lanes a channel
      const int first = i0 * pl.cpc, count = kSteps * pl.cpc < C - first ? kSteps * pl.cpc : C - first;
      for (int c0 = 0; c0 < count; c0 += kThreads / 4) {
        const int c = c0 + t / 4;
        float v = 0.0f;
        if (c < count)
          for (int k = t & 3; k < K; k += 4) v += lds[c * K + k];
        v = lane_sum<4>(v);
        if (c < count && (t & 3) == 0) {
          const int64_t at = n * C + first + c;
          const float z = ld(static_cast<const T*>(a.gate), at);
          st(static_cast<T*>(a.dgate), at, sigmoid(z) * sigmoid(-z) * v);
        }
      }
      __syncthreads();
    }
    us.means(q, pl.sum_zero(q0), m1, mg1);
    if (t < L + 2) out[L + 2 + t] = us.stat[t];
    __syncthreads();  // stat is read
  }
}

// The weights' sums: workgroup (step, part of the rows), which walks down its rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_long_weights(const ResArgs a, const ResWeights w, int A,
                                                               const float* __restrict__ means,
                                                               float* __restrict__ partial) {
  extern __shared__ float lds[];  // [A V]
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V, t = threadIdx.x, step = blockIdx.x;
  const Place pl(A, K, t);
  lds_poison(lds, AV);
  LongBack<T> b(a, w, pl, t, AV, R);
  float e1[V], e2[V], f[V], g0[V];
#pragma unroll
  for (int j = 0; j < V; ++j) e1[j] = e2[j] = f[j] = g0[j] = 0.0f;
#pragma unroll 2
  for (int64_t n = blockIdx.y; n < a.N; n += gridDim.y) {
    b.load(n, 0, step, false);
    b.row(n);
    const float* const m = means + n * 2 * (L + 2);
    float m2[V], x[V], g[V], h[V], d[V], y[V], open[V], p[V], sh[V];
#pragma unroll
    for (int j = 0; j < V; ++j) m2[j] = m[pl.deg[j]];
    b.first(0, step, x, g, h);
    b.second(n, 0, step, x, g, m2, m[L + 1], d, y, open, p, sh);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float u = d[j] * open[j];
      e1[j] = fmaf(u, y[j], e1[j]);
      e2[j] = fmaf(h[j], x[j], e2[j]);
      f[j] += u;
      g0[j] += h[j];
    }
  }
  float* const out = partial + int64_t(blockIdx.y) * res_columns(L, C);
  const int c0 = step * pl.cpc, nc = C - c0 < pl.cpc ? C - c0 : pl.cpc;
#pragma unroll
  for (int which = 0; which < 4; ++which) {
    __syncthreads();
    if (pl.on)
#pragma unroll
      for (int j = 0; j < V; ++j) lds[V * t + j] = which == 0 ? e1[j] : which == 1 ? e2[j] : which == 2 ? f[j] : g0[j];
    __syncthreads();
    const int rows = which < 2 ? L + 1 : 1;
    for (int q = t; q < rows * nc; q += kThreads) {
      const int l = q / nc, c = q - l * nc;
      float s = 0.0f;
      for (int m = 0; m < 2 * l + 1; ++m) s += lds[c * K + l * l + m];
      out[(which < 2 ? which * (L + 1) + l : 2 * (L + 1) + which - 2) * int64_t(C) + c0 + c] = s;
    }
  }
}

// dx and da: workgroup (row, chunk of kSteps steps).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_long_gradients(const ResArgs a, const ResWeights w, int A,
                                                                 const float* __restrict__ means) {
  const int L = a.L, K = (L + 1) * (L + 1), C = int(a.C), R = C * K, AV = A * V, t = threadIdx.x;
  const Place pl(A, K, t);
  LongBack<T> b(a, w, pl, t, AV, R);
  const int chunks = ((R + AV - 1) / AV + kSteps - 1) / kSteps;
  for (int64_t id = blockIdx.x; id < a.N * chunks; id += gridDim.x) {
    const int64_t n = id / chunks;
    const int i0 = int(id - n * chunks) * kSteps;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) b.load(n, i, i0 + i, false);
    b.row(n);
    const float* const m = means + n * 2 * (L + 2);
    const float mg2 = m[L + 1], mg1 = w.post ? m[2 * L + 3] : 0.0f;
    float m2[V], m1[V];
#pragma unroll
    for (int j = 0; j < V; ++j) m2[j] = m[pl.deg[j]], m1[j] = w.post ? m[L + 2 + pl.deg[j]] : 0.0f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int at = (i0 + i) * AV + V * t;
      float x[V], g[V], d[V], y[V], open[V], p[V], sh[V];
      b.first(i, i0 + i, x, g, d);
      b.second(n, i, i0 + i, x, g, m2, mg2, d, y, open, p, sh);
      if (!pl.on) continue;
      if (a.dx) step_store<false, T, V>(static_cast<T*>(a.dx) + n * R, at, R, d);
      if (!a.da) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float u = d[j] * open[j] * p[j];
        d[j] = w.post ? b.r1[j] * (u - fmaf(y[j], m1[j], pl.zero(j, mg1))) : u;
      }
      step_store<false, T, V>(static_cast<T*>(a.da) + n * R, at, R, d);
    }
  }
}

constexpr int64_t kMaxLds = 150 << 10, kGrid = 1 << 20;

// Threads with places; 0: not a case for these kernels.
int long_lanes(const ResArgs& a) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1), R = a.C * K;
  if (a.L == 0 || R < 4 * V || R >= (int64_t(1) << 30)) return 0;
  const int64_t unit = K % 4 == 0 ? K / 4 : K % 2 == 0 ? K / 2 : K, A = kThreads / unit * unit;
  if (A == 0 || a.L + 2 > kThreads) return 0;
  return (kSteps * A * V + Block::floats(A, K, a.L)) * 4 <= kMaxLds ? int(A) : 0;
}

// Parts of the rows for the weights' sums.
int64_t weight_parts(const ResArgs& a, int A) {
  const int64_t R = a.C * (a.L + 1) * (a.L + 1), steps = (R + A * V - 1) / (A * V);
  return std::max<int64_t>(1, std::min<int64_t>(a.N, 512 / std::max<int64_t>(1, steps)));
}

template <typename T>
hipError_t run_long(const ResArgs& a, int A, hipStream_t s) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1);
  k_res_long<T><<<uint32_t(std::min<int64_t>(a.N, 512)), kThreads, size_t(Block::floats(A, K, a.L)) * 4, s>>>(
      a, ResWeights(a), A);
  return hipGetLastError();
}

template <typename T>
hipError_t run_long_backward(const ResArgs& a, int A, hipStream_t s) {
  const int64_t K = int64_t(a.L + 1) * (a.L + 1), AV = int64_t(A) * V, steps = (a.C * K + AV - 1) / AV;
  const int64_t means = a.N * 2 * (a.L + 2), parts = weight_parts(a, A);
  const ResWeights w(a);
  k_res_long_means<T><<<uint32_t(std::min<int64_t>(a.N, 512)), kThreads,
                        size_t(kSteps * AV + Block::floats(A, K, a.L)) * 4, s>>>(a, w, A, a.work);
  if (a.weights())  // before dx, which may be written over dr
    k_res_long_weights<T><<<dim3{uint32_t(steps), uint32_t(parts)}, kThreads, size_t(AV) * 4, s>>>(a, w, A, a.work,
                                                                                                  a.work + means);
  if (a.dx || a.da)
    k_res_long_gradients<T><<<uint32_t(std::min(a.N * ((steps + kSteps - 1) / kSteps), kGrid)), kThreads, 0, s>>>(
        a, w, A, a.work);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && a.weights() ? launch_residual_sum(a, a.work + means, parts, s) : e;
}

}  // namespace

bool residual_is_long(const ResArgs& a) { return long_lanes(a) > 0; }

hipError_t launch_residual_long(const ResArgs& a, hipStream_t s) {
  return a.bf16 ? run_long<uint16_t>(a, long_lanes(a), s) : run_long<float>(a, long_lanes(a), s);
}

int64_t residual_long_floats(const ResArgs& a) {
  return a.N * 2 * (a.L + 2) + weight_parts(a, long_lanes(a)) * res_columns(a.L, a.C);
}

hipError_t launch_residual_long_backward(const ResArgs& a, hipStream_t s) {
  return a.bf16 ? run_long_backward<uint16_t>(a, long_lanes(a), s) : run_long_backward<float>(a, long_lanes(a), s);
}

}  // namespace gtp
