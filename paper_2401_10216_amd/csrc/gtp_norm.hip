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

// Any degree and channel count: one workgroup a row, a degree at a time.
template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_any(const T* __restrict__ x, const float* __restrict__ w,
                                                          const float* __restrict__ b, float eps, int64_t C, int L,
                                                          T* __restrict__ y, float* __restrict__ mean,
                                                          float* __restrict__ rstd) {
  __shared__ float red[kAnyThreads / 64];
  lds_poison(red, kAnyThreads / 64);
  const int64_t n = blockIdx.x;
  const int64_t K = int64_t(L + 1) * (L + 1), base = n * C * K;
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

template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_dx_any(const T* __restrict__ x, const T* __restrict__ dy,
                                                             const float* __restrict__ w,
                                                             const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, int64_t C, int L,
                                                             T* __restrict__ dx) {
  __shared__ float red[kAnyThreads / 64];
  lds_poison(red, kAnyThreads / 64);
  const int64_t n = blockIdx.x;
  const int64_t K = int64_t(L + 1) * (L + 1), base = n * C * K;
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

// Partial sums of dw and db over a chunk of rows: workgroup (c, chunk).
// partial[chunk][(L + 2) C]: L + 1 rows of dw, then db.
template <typename T>
__global__ __launch_bounds__(kAnyThreads) void k_norm_dw_any(const T* __restrict__ x, const T* __restrict__ dy,
                                                             const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, int64_t N, int64_t C,
                                                             int L, int64_t chunk, float* __restrict__ partial) {
  __shared__ float red[kAnyThreads / 64];
  lds_poison(red, kAnyThreads / 64);
  const int64_t c = blockIdx.x, n0 = int64_t(blockIdx.y) * chunk;
  const int64_t rows = n0 + chunk < N ? chunk : N - n0;
  const int64_t K = int64_t(L + 1) * (L + 1);
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

// The chunks' partial sums, added in order: a workgroup takes 64 columns, its 16
// waves every 16th chunk each.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void k_norm_sum(const float* __restrict__ partial, int64_t chunks,
                                                          int64_t cols, int64_t wcols, float* __restrict__ dw,
                                                          float* __restrict__ db) {
  __shared__ float red[kSumThreads];
  lds_poison(red, kSumThreads);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = int64_t(blockIdx.x) * 64 + lane;
  float s = 0.0f;
  if (col < cols)
    for (int64_t i = wave; i < chunks; i += kSumThreads / 64) s += partial[i * cols + col];
  red[threadIdx.x] = s;
  __syncthreads();
  if (wave == 0 && col < cols) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < kSumThreads / 64; ++i) t += red[i * 64 + lane];
    if (col < wcols) {
      if (dw) dw[col] = t;
    } else if (db) {
      db[col - wcols] = t;
    }
  }
}

int64_t any_chunks(int64_t N) { return N < 64 ? 1 : (N < 64 * 64 ? N / 64 : 64); }

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  const dim3 grid{uint32_t(a.N)};
  if (a.bf16)
    k_norm_any<<<grid, kAnyThreads, 0, s>>>(static_cast<const uint16_t*>(a.x), a.w, a.b, a.eps, a.C, a.L,
                                            static_cast<uint16_t*>(a.y), a.mean, a.rstd);
  else
    k_norm_any<<<grid, kAnyThreads, 0, s>>>(static_cast<const float*>(a.x), a.w, a.b, a.eps, a.C, a.L,
                                            static_cast<float*>(a.y), a.mean, a.rstd);
  return hipGetLastError();
}

int64_t norm_partial_floats(int L, int64_t N, int64_t C, bool bf16) {
  (void)bf16;
  return any_chunks(N) * (L + 2) * C;
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
  const int64_t chunks = any_chunks(a.N), chunk = (a.N + chunks - 1) / chunks;
  const int64_t used = a.N ? (a.N + chunk - 1) / chunk : 0;
  const dim3 grid{uint32_t(a.N)}, gw{uint32_t(a.C), uint32_t(used)};
  const bool weights = a.dw || a.db;
  if (a.bf16) {
    const auto *x = static_cast<const uint16_t*>(a.x), *dy = static_cast<const uint16_t*>(a.dy);
    if (a.y && a.N)
      k_norm_dx_any<<<grid, kAnyThreads, 0, s>>>(x, dy, a.w, a.mean_in, a.rstd_in, a.C, a.L,
                                                 static_cast<uint16_t*>(a.y));
    if (weights && a.N)
      k_norm_dw_any<<<gw, kAnyThreads, 0, s>>>(x, dy, a.mean_in, a.rstd_in, a.N, a.C, a.L, chunk, a.partial);
  } else {
    const auto *x = static_cast<const float*>(a.x), *dy = static_cast<const float*>(a.dy);
    if (a.y && a.N)
      k_norm_dx_any<<<grid, kAnyThreads, 0, s>>>(x, dy, a.w, a.mean_in, a.rstd_in, a.C, a.L, static_cast<float*>(a.y));
    if (weights && a.N)
      k_norm_dw_any<<<gw, kAnyThreads, 0, s>>>(x, dy, a.mean_in, a.rstd_in, a.N, a.C, a.L, chunk, a.partial);
  }
  if (weights) {
    const int64_t cols = (a.L + 2) * a.C;
    k_norm_sum<<<dim3{uint32_t((cols + 63) / 64)}, kSumThreads, 0, s>>>(a.partial, used, cols, (a.L + 1) * a.C, a.dw,
                                                                       a.db);
  }
  return hipGetLastError();
}

}  // namespace gtp
