// The buckets of a bias by distance, made ahead for all heads.
//
// A score's bucket takes nine vector instructions beside some ten of the attention itself, and is the same for
// every head.  Made once, a byte a pair (read by each head from the caches, 16 bytes a lane and tile of 32 x 32),
// a score takes one instruction for it instead.  8192^2 pairs: 14-20 us.
#include "gtp_attn_core.hpp"

namespace gtp {
namespace {

constexpr int kTiles = 16;  // tiles that a workgroup takes, a wave four

// Workgroup: 32 columns (rows of `a`, a segment's `at`) and 16 tiles of 32 of the other side, whose positions it stages.
__global__ __launch_bounds__(256) void k_bias_bytes(const AttnArgs a, const float* __restrict__ pos,
                                                    const int64_t* off, int64_t most, int64_t total,
                                                    const float* __restrict__ pos2, const int64_t* off2, int64_t most2,
                                                    int64_t total2, uint8_t* __restrict__ out) {
  __shared__ float x[32 * kTiles], y[32 * kTiles], z[32 * kTiles];
  lds_poison(x, 32 * kTiles);
  lds_poison(y, 32 * kTiles);
  lds_poison(z, 32 * kTiles);
  const int64_t blocks = bytes_tiles(most), tiles = bytes_tiles(most2), chunks = (tiles + kTiles - 1) / kTiles;
  const int64_t chunk = blockIdx.x % chunks, block = blockIdx.x / chunks % blocks, b = blockIdx.x / chunks / blocks;
  int64_t s, n, s2, n2;
  segment(off, b, most, total, s, n);
  segment(off2, b, most2, total2, s2, n2);
  if (block * 32 >= n || chunk * kTiles * 32 >= n2) return;  // pairs that no kernel looks at
  for (int i = threadIdx.x; i < 32 * kTiles; i += 256) {
    const int64_t j = chunk * kTiles * 32 + i, at = 3 * (s2 + (j < n2 ? j : n2 - 1));
    x[i] = pos2[at], y[i] = pos2[at + 1], z[i] = pos2[at + 2];
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hi = lane >> 5;
  const int64_t i = block * 32 + (lane & 31), at = 3 * (s + (i < n ? i : n - 1));
  const float px = pos[at], py = pos[at + 1], pz = pos[at + 2];
  const Buckets bucket(a);
  for (int k = wave; k < kTiles; k += 4) {
    const int64_t tile = chunk * kTiles + k;
    if (tile >= tiles) break;
    u32x4 v;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = 32 * k + 8 * g + 4 * hi + j;
        w |= bucket(px - x[e], py - y[e], pz - z[e]) << (8 * j + 2);
      }
      v[g] = w;
    }
    reinterpret_cast<u32x4*>(out)[((b * blocks + block) * tiles + tile) * 64 + lane] = v;
  }
}

}  // namespace

// Made ahead where four heads at least share them, for segments longer than the kernels' short forms take, where their
// making is small beside the heads' work, where segments are not so uneven that most pairs would be of none, and up to
// 1 GiB, a fraction of a percent of the card's memory: what they save does not fall off with the size, but what they
// take grows with its square, and beyond a call runs without.  8 heads of 128, bf16, forward and gradients: 32768 rows (1 GiB)
// 7.2 and 30.2 ms (each made at its score 8.6 and 41.3), 16384 rows 1.8 and 7.6 (2.2 and 10.2); of 64, fp32, 32768 rows 14.3 and
// 48.8 (15.6 and 62); what the limit costs: 50000 rows of 128, bf16, 20.2 and 99.8 ms instead of 17.5 and 72.8.
constexpr int64_t kMostBytes = int64_t(1) << 30;
int64_t bias_bytes(const AttnArgs& a) {
  if (!a.bias || a.H < 4 || a.max_q <= 256 || a.max_k <= 256 || dq_rows_a_tile(a) == 64) return 0;
  const int64_t n = a.B * bytes_tiles(a.max_q) * bytes_tiles(a.max_k);  // KB
  const double pairs = double(a.Tq) * double(a.max_k);
  return n <= kMostBytes / 1024 && double(n) * 1024.0 <= 2.0 * pairs + 65536.0 ? n * 1024 : 0;
}

bool bias_bytes_for_keys(const AttnArgs& a) { return a.G == 1; }

hipError_t launch_bias_bytes(const AttnArgs& a, bool keys, hipStream_t s) {
  const int64_t most = keys ? a.max_k : a.max_q, most2 = keys ? a.max_q : a.max_k;
  const uint32_t n = uint32_t(a.B * bytes_tiles(most) * ((bytes_tiles(most2) + kTiles - 1) / kTiles));
  if (keys)
    k_bias_bytes<<<n, 256, 0, s>>>(a, a.k_pos, a.k_off, a.max_k, a.Tk, a.q_pos, a.q_off, a.max_q, a.Tq, a.bytes_k);
  else
    k_bias_bytes<<<n, 256, 0, s>>>(a, a.q_pos, a.q_off, a.max_q, a.Tq, a.k_pos, a.k_off, a.max_k, a.Tk, a.bytes);
  return hipGetLastError();
}

}  // namespace gtp
