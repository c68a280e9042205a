// The gradient of the queries with a bias by distance, and the bias's gradient.
#include "gtp_attn_dq.hpp"

namespace gtp {
namespace {

// Sums of `n` entries of `cols` floats, one behind the other, in order, in chunks of up to kChunk entries:
// workgroup (key head and chunk, 64 columns), its four waves a quarter of the chunk each.
constexpr int kChunk = 256;
__global__ __launch_bounds__(256) void k_bias_sum(const float* __restrict__ in, int64_t n, int64_t chunks, int cols,
                                                  float* __restrict__ out) {
  __shared__ float red[4][64];
  lds_poison(&red[0][0], 256);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = int(blockIdx.y) * 64 + lane;
  const int64_t hk = blockIdx.x / chunks, e0 = (blockIdx.x % chunks) * kChunk + wave * (kChunk / 4);
  const int64_t e1 = e0 + kChunk / 4 < n ? e0 + kChunk / 4 : n;
  float v = 0.0f;
  if (c < cols) {
    const float* const p = in + hk * n * cols + c;
#pragma unroll 8
    for (int64_t e = e0; e < e1; ++e) v += p[e * cols];
  }
  red[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && c < cols)
    out[int64_t(blockIdx.x) * cols + c] = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}

int64_t chunks(int64_t n) { return n <= kChunk ? 1 : (n + kChunk - 1) / kChunk; }

}  // namespace

void launch_attn_dq_bias(const AttnArgs& a, hipStream_t s) { launch_dq_kernel<kBias>(a, s); }

int64_t attn_bias_parts(const AttnArgs& a) {
  const int64_t BM = dq_rows_a_tile(a);
  return (a.max_q * a.G + BM - 1) / BM * a.splits * a.B;
}

// The workgroups' sums, and those of chunks of them twice over.
int64_t bias_part_floats(const AttnArgs& a) {
  const int64_t n = attn_bias_parts(a);
  return (n + chunks(n)) * a.Hk * a.G * a.buckets;
}

hipError_t launch_attn_bias_sum(const AttnArgs& a, hipStream_t s) {
  const int cols = a.G * a.buckets;
  int64_t n = attn_bias_parts(a);
  float *in = a.bias_part, *spare = in + n * a.Hk * cols;
  for (;;) {
    const int64_t m = chunks(n);
    float* const out = m == 1 ? a.dbias : spare;
    k_bias_sum<<<dim3(uint32_t(a.Hk * m), uint32_t((cols + 63) / 64)), 256, 0, s>>>(in, n, m, cols, out);
    if (m == 1) return hipGetLastError();
    spare = in;  // done with: longer than what comes
    in = out;
    n = m;
  }
}

}  // namespace gtp
