// The residual step for rows of any degree and channel count (formulas in gtp_res.hpp), and
// the sum of the parts of its weights' gradients.
//
// One workgroup a row, a degree at a time, every pass from memory (a row's second and later
// reads come from the caches).  r may be x, and dx may be dr: an element is read for the last
// time by the thread that writes it.  The backward takes the means that its gradients need to
// the work first, so that the weights' sums and the rows' gradients are passes of their own.
#include <algorithm>

#include "gtp_norm_core.hpp"
#include "gtp_res.hpp"

namespace gtp {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kGrid = 1 << 20;  // workgroups at most: a launch holds less than 2^32 threads

// Sum of v over the workgroup's threads, in a fixed order; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) s += red[i];
  return s;
}

// q / d for 0 <= q < 2^31 without a division.
struct Divide {
  uint32_t d, inv;
  __device__ __forceinline__ explicit Divide(uint32_t d_) : d(d_), inv(d_ > 1 ? 0xffffffffu / d_ : 0) {}
  __device__ __forceinline__ uint32_t operator()(uint32_t q) const {
    if (d == 1) return q;
    uint32_t n = __umulhi(q, inv);  // at most two too few
    uint32_t r = q - n * d;
    if (r >= d) ++n, r -= d;
    return r >= d ? n + 1 : n;
  }
};

// f(channel, element) over a degree's elements of the row at `base`, dealt to the threads.
template <typename F>
__device__ __forceinline__ void over_degree(int64_t base, int64_t C, int64_t K, int l, F f) {
  const int64_t M = 2 * l + 1, at = base + l * l;
  const Divide by{uint32_t(M)};
  if (C * M < (int64_t(1) << 31) - kThreads) {  // 64-bit divisions took longer than all else
    const int n = int(C * M);
#pragma unroll 4
    for (int q = threadIdx.x; q < n; q += kThreads) {
      const uint32_t c = by(uint32_t(q));
      f(int64_t(c), at + int64_t(c) * K + (q - int(c * uint32_t(M))));
    }
  } else {
    for (int64_t q = threadIdx.x; q < C * M; q += kThreads) {
      const int64_t c = q / M;
      f(c, at + c * K + (q - c * M));
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_any(const T* x, const T* __restrict__ a, const T* __restrict__ gate,
                                                      ResWeights w, float eps, int64_t N, int L, T* r,
                                                      T* __restrict__ h, float* __restrict__ mean1,
                                                      float* __restrict__ rstd1, float* __restrict__ mean2,
                                                      float* __restrict__ rstd2) {
  __shared__ float red[kThreads / 64];
  lds_poison(red, kThreads / 64);
  const int64_t C = w.C, K = int64_t(L + 1) * (L + 1);
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    const int64_t base = n * C * K;
    for (int l = 0; l <= L; ++l) {
      const float cnt = float(C) * float(2 * l + 1);
      float mu1 = 0.0f, r1 = 1.0f, mu2 = 0.0f;
      if (w.post) {
        float s = 0.0f;
        if (l == 0) {
          over_degree(base, C, K, l, [&](int64_t, int64_t i) { s += ld(a, i); });
          mu1 = block_sum(s, red) / cnt;
          s = 0.0f;
        }
        over_degree(base, C, K, l, [&](int64_t, int64_t i) {
          const float v = ld(a, i) - mu1;
          s = fmaf(v, v, s);
        });
        r1 = 1.0f / sqrtf(block_sum(s, red) / cnt + eps);
      }
      auto sum = [&](int64_t c, int64_t i) {  // r before its rounding
        const float t = w.post ? fmaf((ld(a, i) - mu1) * r1, w.post_w(l, c), w.post_b(l, c)) : ld(a, i);
        return fmaf(w.s(l, c) * (gate ? sigmoid(ld(gate, n * C + c)) : 1.0f), t, ld(x, i));
      };
      float s = 0.0f;
      if (l == 0) {
        over_degree(base, C, K, l, [&](int64_t c, int64_t i) { s += sum(c, i); });
        mu2 = block_sum(s, red) / cnt;
        s = 0.0f;
      }
      over_degree(base, C, K, l, [&](int64_t c, int64_t i) {
        const float v = sum(c, i) - mu2;
        s = fmaf(v, v, s);
      });
      const float r2 = 1.0f / sqrtf(block_sum(s, red) / cnt + eps);
      over_degree(base, C, K, l, [&](int64_t c, int64_t i) {
        const float v = sum(c, i);
        st(r, i, v);
        st(h, i, fmaf((v - mu2) * r2, w.pre_w(l, c), w.pre_b(l, c)));
      });
      if (threadIdx.x == 0) {
        if (l == 0 && mean1) mean1[n] = mu1;
        if (rstd1) rstd1[n * (L + 1) + l] = r1;
        if (l == 0 && mean2) mean2[n] = mu2;
        if (rstd2) rstd2[n * (L + 1) + l] = r2;
      }
    }
  }
}

// The backward's elements.  means: for each row [L + 2] of g2 xh2 by degree and of g2 at degree
// 0, then as many of g1 xh1 and g1.
template <typename T>
struct Back {
  const T *r, *a, *gate, *dh, *dr;
  ResWeights w;
  const float *mean1, *rstd1, *mean2, *rstd2;
  float* means;
  int64_t N;
  int L;
  __device__ float open(int64_t n, int64_t c) const { return gate ? sigmoid(ld(gate, n * w.C + c)) : 1.0f; }
  __device__ float xh2(int64_t n, int l, int64_t i) const {
    return (ld(r, i) - (l == 0 ? mean2[n] : 0.0f)) * rstd2[n * (L + 1) + l];
  }
  // xh1, or a without the norm behind the part
  __device__ float xh1(int64_t n, int l, int64_t i) const {
    return w.post ? (ld(a, i) - (l == 0 ? mean1[n] : 0.0f)) * rstd1[n * (L + 1) + l] : ld(a, i);
  }
  // D for the means m = means + n * 2 (L + 2)
  __device__ float d(int64_t n, int l, int64_t c, int64_t i, float along, float mean_g) const {
    const float g = ld(dh, i) * w.pre_w(l, c);
    return (dr ? ld(dr, i) : 0.0f) + rstd2[n * (L + 1) + l] * (g - xh2(n, l, i) * along - mean_g);
  }
  __device__ float d(int64_t n, int l, int64_t c, int64_t i) const {
    const float* m = means + n * 2 * (L + 2);
    return d(n, l, c, i, m[l], l == 0 ? m[L + 1] : 0.0f);
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_means(const Back<T> b) {
  __shared__ float red[kThreads / 64];
  lds_poison(red, kThreads / 64);
  const int L = b.L;
  const int64_t C = b.w.C, K = int64_t(L + 1) * (L + 1);
  for (int64_t n = blockIdx.x; n < b.N; n += gridDim.x) {
    const int64_t base = n * C * K;
    float* const m = b.means + n * 2 * (L + 2);
    for (int l = 0; l <= L; ++l) {
      const float cnt = float(C) * float(2 * l + 1);
      float s = 0.0f, u = 0.0f;
      over_degree(base, C, K, l, [&](int64_t c, int64_t i) {
        const float g = ld(b.dh, i) * b.w.pre_w(l, c);
        s = fmaf(g, b.xh2(n, l, i), s);
        u += g;
      });
      const float along = block_sum(s, red) / cnt, mg = l == 0 ? block_sum(u, red) / cnt : 0.0f;
      if (threadIdx.x == 0) {
        m[l] = along;
        if (l == 0) m[L + 1] = mg;
      }
      if (!b.w.post) continue;
      s = u = 0.0f;
      over_degree(base, C, K, l, [&](int64_t c, int64_t i) {
        const float g = b.d(n, l, c, i, along, mg) * b.open(n, c) * b.w.s(l, c) * b.w.post_w(l, c);
        s = fmaf(g, b.xh1(n, l, i), s);
        u += g;
      });
      const float along1 = block_sum(s, red) / cnt, mg1 = l == 0 ? block_sum(u, red) / cnt : 0.0f;
      if (threadIdx.x == 0) {
        m[L + 2 + l] = along1;
        if (l == 0) m[2 * L + 3] = mg1;
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_gradients(const Back<T> b, T* dx, T* __restrict__ da,
                                                            T* __restrict__ dgate) {
  const int L = b.L;
  const int64_t C = b.w.C, K = int64_t(L + 1) * (L + 1);
  for (int64_t n = blockIdx.x; n < b.N; n += gridDim.x) {
    const int64_t base = n * C * K;
    const float* const m = b.means + n * 2 * (L + 2) + L + 2;
    if (dgate) {
      // a channel to a thread, or, of degree 3 and more, to a wave
      const int lanes = K < 16 ? 1 : 64, lane = threadIdx.x & (lanes - 1);
      for (int64_t c = threadIdx.x / lanes; c < C; c += kThreads / lanes) {
        float s = 0.0f;
        for (int k = lane; k < int(K); k += lanes) {
          const int l = degree_of(k);
          const int64_t i = base + c * K + k;
          const float t = b.w.post ? fmaf(b.xh1(n, l, i), b.w.post_w(l, c), b.w.post_b(l, c)) : ld(b.a, i);
          s = fmaf(b.d(n, l, c, i) * b.w.s(l, c), t, s);
        }
        if (lanes == 64) s = wave_sum(s);
        if (lane != 0) continue;
        const float v = ld(b.gate, n * C + c);
        st(dgate, n * C + c, sigmoid(v) * sigmoid(-v) * s);
      }
      __syncthreads();  // dx may be written over dr
    }
    for (int l = 0; l <= L; ++l)
      over_degree(base, C, K, l, [&](int64_t c, int64_t i) {
        const float d = b.d(n, l, c, i);
        if (da) {
          float g = d * b.open(n, c) * b.w.s(l, c);
          if (b.w.post)
            g = b.rstd1[n * (L + 1) + l] *
                (g * b.w.post_w(l, c) - b.xh1(n, l, i) * m[l] - (l == 0 ? m[L + 1] : 0.0f));
          st(da, i, g);
        }
        if (dx) st(dx, i, d);
      });
    __syncthreads();
  }
}

// The weights' sums over a chunk of rows: workgroup (degree and channel, chunk).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_weights(const Back<T> b, int64_t chunk, float* __restrict__ partial) {
  __shared__ float red[kThreads / 64];
  lds_poison(red, kThreads / 64);
  const int L = b.L;
  const int64_t C = b.w.C, K = int64_t(L + 1) * (L + 1), n0 = int64_t(blockIdx.y) * chunk;
  const int64_t rows = n0 + chunk < b.N ? chunk : b.N - n0;
  float* const out = partial + int64_t(blockIdx.y) * res_columns(L, C);
  for (int64_t id = blockIdx.x; id < C * (L + 1); id += gridDim.x) {
    const int l = int(id / C);
    const int64_t c = id - l * C, M = 2 * l + 1;
    float e1 = 0.0f, e2 = 0.0f, f = 0.0f, g = 0.0f;
    const Divide by{uint32_t(M)};
    for (int64_t q = threadIdx.x; q < rows * M; q += kThreads) {
      const int64_t k = q < (int64_t(1) << 31) ? by(uint32_t(q)) : q / M;
      const int64_t n = n0 + k, i = (n * C + c) * K + l * l + (q - k * M);
      const float u = b.d(n, l, c, i) * b.open(n, c), d = ld(b.dh, i);
      e1 = fmaf(u, b.xh1(n, l, i), e1);
      e2 = fmaf(d, b.xh2(n, l, i), e2);
      f += u;
      g += d;
    }
    e1 = block_sum(e1, red);
    e2 = block_sum(e2, red);
    if (l == 0) {
      f = block_sum(f, red);
      g = block_sum(g, red);
    }
    if (threadIdx.x == 0) {
      out[l * C + c] = e1;
      out[(L + 1 + l) * C + c] = e2;
      if (l == 0) out[2 * (L + 1) * C + c] = f, out[(2 * L + 3) * C + c] = g;
    }
  }
}

// The same of scalars (K = 1), a thread a channel: the other way, neighbours read a row apart.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_res_weights_scalars(const Back<T> b, int64_t chunk,
                                                                  float* __restrict__ partial) {
  const int64_t C = b.w.C, n0 = int64_t(blockIdx.y) * chunk, n1 = n0 + chunk < b.N ? n0 + chunk : b.N;
  float* const out = partial + int64_t(blockIdx.y) * res_columns(0, C);
  for (int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x; c < C; c += int64_t(gridDim.x) * kThreads) {
    float e1 = 0.0f, e2 = 0.0f, f = 0.0f, g = 0.0f;
#pragma unroll 4
    for (int64_t n = n0; n < n1; ++n) {
      const int64_t i = n * C + c;
      const float u = b.d(n, 0, c, i) * b.open(n, c), d = ld(b.dh, i);
      e1 = fmaf(u, b.xh1(n, 0, i), e1);
      e2 = fmaf(d, b.xh2(n, 0, i), e2);
      f += u;
      g += d;
    }
    out[c] = e1;
    out[C + c] = e2;
    out[2 * C + c] = f;
    out[3 * C + c] = g;
  }
}

// The parts' sums, added in order: a workgroup takes 8 columns (l, c) of E1 and E2 at a time
// (and of F and G, at degree 0), 128 groups of threads every 128th part each, then a tree over
// the groups.
constexpr int kSumThreads = 1024, kSumCols = 8;
__global__ __launch_bounds__(kSumThreads) void k_res_sum(const float* __restrict__ partial, int64_t parts, int L,
                                                         ResWeights w, float* __restrict__ dscale,
                                                         float* __restrict__ dw1, float* __restrict__ db1,
                                                         float* __restrict__ dw2, float* __restrict__ db2) {
  __shared__ float red[4][kSumThreads];
  lds_poison(&red[0][0], 4 * kSumThreads);
  const int64_t C = w.C, cols = (L + 1) * C, all = res_columns(L, C);
  const int j = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
  for (int64_t col0 = int64_t(blockIdx.x) * kSumCols; col0 < cols; col0 += int64_t(gridDim.x) * kSumCols) {
    const int64_t col = col0 + j;
    const bool in = col < cols, zero = col < C;
    const float* const p = partial + (in ? col : 0);
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (in) {
#pragma unroll 8
      for (int64_t i = g; i < parts; i += kSumThreads / kSumCols) {
        s[0] += p[i * all];
        s[1] += p[i * all + cols];
        if (zero) {
          s[2] += p[i * all + 2 * cols];
          s[3] += p[i * all + 2 * cols + C];
        }
      }
    }
    __syncthreads();  // the columns before are read
#pragma unroll
    for (int k = 0; k < 4; ++k) red[k][threadIdx.x] = s[k];
#pragma unroll
    for (int o = kSumThreads / 2; o >= kSumCols; o /= 2) {
      __syncthreads();
      if (int(threadIdx.x) < o)
#pragma unroll
        for (int k = 0; k < 4; ++k) red[k][threadIdx.x] += red[k][threadIdx.x + o];
    }
    if (g != 0 || !in) continue;
    const int l = int(col / C);
    const int64_t c = col - l * C;
    const float e1 = red[0][j], f = red[2][j];
    if (dw1) dw1[col] = w.s(l, c) * e1;
    if (dscale) dscale[col] = fmaf(w.post_w(l, c), e1, w.post_b(l, c) * f);
    if (dw2) dw2[col] = red[1][j];
    if (l == 0) {
      if (db1) db1[c] = w.s(0, c) * f;
      if (db2) db2[c] = red[3][j];
    }
  }
}

int64_t chunks_of(int64_t N) { return N < 64 ? 1 : (N < 64 * 64 ? N / 64 : 64); }

template <typename T>
hipError_t run_any(const ResArgs& a, hipStream_t s) {
  const uint32_t grid = uint32_t(std::min(a.N, kGrid));
  k_res_any<T><<<grid, kThreads, 0, s>>>(static_cast<const T*>(a.x), static_cast<const T*>(a.a),
                                         static_cast<const T*>(a.gate), ResWeights(a), a.eps, a.N, a.L,
                                         static_cast<T*>(a.r), static_cast<T*>(a.h), a.mean1, a.rstd1, a.mean2, a.rstd2);
  return hipGetLastError();
}

template <typename T>
hipError_t run_any_backward(const ResArgs& a, hipStream_t s) {
  const int64_t means = a.N * 2 * (a.L + 2), chunks = chunks_of(a.N), chunk = (a.N + chunks - 1) / chunks;
  const int64_t used = (a.N + chunk - 1) / chunk;
  const Back<T> b{static_cast<const T*>(a.x), static_cast<const T*>(a.a), static_cast<const T*>(a.gate),
                  static_cast<const T*>(a.dh), static_cast<const T*>(a.dr), ResWeights(a), a.mean1, a.rstd1, a.mean2,
                  a.rstd2, a.work, a.N, a.L};
  const uint32_t grid = uint32_t(std::min(a.N, kGrid));
  k_res_means<T><<<grid, kThreads, 0, s>>>(b);
  // the weights before dx, which may be written over dr
  if (a.weights() && a.L == 0 && a.C >= kThreads)
    k_res_weights_scalars<T><<<dim3{uint32_t(std::min((a.C + kThreads - 1) / kThreads, kGrid / used)), uint32_t(used)},
                               kThreads, 0, s>>>(b, chunk, a.work + means);
  else if (a.weights())
    k_res_weights<T><<<dim3{uint32_t(std::min(a.C * (a.L + 1), kGrid / used)), uint32_t(used)}, kThreads, 0, s>>>(
        b, chunk, a.work + means);
  if (a.dx || a.da || a.dgate)
    k_res_gradients<T><<<grid, kThreads, 0, s>>>(b, static_cast<T*>(a.dx), static_cast<T*>(a.da),
                                                 static_cast<T*>(a.dgate));
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && a.weights() ? launch_residual_sum(a, a.work + means, used, s) : e;
}

}  // namespace

hipError_t launch_residual_sum(const ResArgs& a, const float* partial, int64_t parts, hipStream_t s) {
  const int64_t n = std::min(((a.L + 1) * a.C + kSumCols - 1) / kSumCols, kGrid);
  k_res_sum<<<uint32_t(n), kSumThreads, 0, s>>>(partial, parts, a.L, ResWeights(a), a.dscale, a.dw1, a.db1, a.dw2,
                                                a.db2);
  return hipGetLastError();
}

hipError_t launch_residual_any(const ResArgs& a, hipStream_t s) {
  return a.bf16 ? run_any<uint16_t>(a, s) : run_any<float>(a, s);
}

int64_t residual_any_floats(const ResArgs& a) {
  return a.N * 2 * (a.L + 2) + chunks_of(a.N) * res_columns(a.L, a.C);
}

hipError_t launch_residual_any_backward(const ResArgs& a, hipStream_t s) {
  return a.bf16 ? run_any_backward<uint16_t>(a, s) : run_any_backward<float>(a, s);
}

}  // namespace gtp
