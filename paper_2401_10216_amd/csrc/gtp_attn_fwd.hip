// The forward without a bias (gtp_attn_fwd.hpp), the join of its parts, the sum of the
// gradients' parts, and how many parts there are.
#include <cmath>

#include "gtp_attn_fwd.hpp"

namespace gtp {
namespace {

constexpr int kParts = 128;     // at most, of a split call

template <typename T>
__device__ __forceinline__ void store_one(T* p, float v) {
  if constexpr (sizeof(T) == 4) {
    *p = v;
  } else {
    const __bf16 one = static_cast<__bf16>(v);
    *p = __builtin_bit_cast(uint16_t, one);
  }
}

// Joins the parts of a split forward: o = sum_s e^(lse_s - lse) o_s.  WAVES waves take a
// row: their lanes first the parts, two each (at most kParts), then the elements, each wave its parts of
// them in order; the waves' sums are added in order.  What it costs is the wait for loads
// one after the other, so many parts are dealt to more waves.
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs a) {
  static_assert(kParts <= 128, "two parts a lane");
  constexpr int ROWS = 4 / WAVES;
  __shared__ float sums[WAVES > 1 ? WAVES * 256 : 1];
  lds_poison(sums, int(sizeof(sums) / 4));
  const int64_t per = (a.max_q * a.H + ROWS - 1) / ROWS, b = blockIdx.x / per;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = wave % WAVES;
  const int64_t i = (blockIdx.x % per) * ROWS + wave / WAVES;
  int64_t qs, nq;
  segment(a.q_off, b, a.max_q, a.Tq, qs, nq);
  if (i >= nq * a.H) return;  // a whole workgroup, where waves share a row
  const int64_t t = qs + i / a.H, h = i % a.H, all = a.Tq * a.H, row = t * a.H + h;
  const float* const lses = a.part + a.splits * all * a.d;
  float own[2], e[2], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = lane + 64 * k;
    const float got = lses[int64_t(s < a.splits ? s : 0) * all + row];
    own[k] = s < a.splits ? got : -INFINITY;
    top = fmaxf(top, own[k]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    e[k] = own[k] == -INFINITY ? 0.0f : expf(own[k] - top);  // NaN where a part's row is
    sum += e[k];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
#pragma unroll
  for (int k = 0; k < 2; ++k) e[k] = sum == 0.0f ? 0.0f : e[k] / sum;
  if (lane == 0 && first == 0) a.lse[row] = sum == 0.0f ? -INFINITY : top + logf(sum);
  T* const out = static_cast<T*>(const_cast<void*>(a.out.p)) + t * a.out.row + h * a.out.head;
  for (int c0 = 0; c0 < a.d; c0 += 64) {
    const int c = c0 + lane;
    const float* const in = a.part + row * a.d + (c < a.d ? c : 0);
    float v = 0.0f;
    for (int s0 = first; s0 < a.splits; s0 += 8 * WAVES) {  // eight parts' loads at a time
      float p[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int s = s0 + k * WAVES;
        p[k] = in[int64_t(s < a.splits ? s : 0) * all * a.d];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int s = s0 + k * WAVES;
        const float low = __shfl(e[0], s & 63), high = __shfl(e[1], s & 63), ws = s < 64 ? low : high;
        v = s >= a.splits || ws == 0.0f ? v : fmaf(ws, p[k], v);
      }
    }
    if constexpr (WAVES > 1) {
      sums[wave * 256 + c] = v;  // c < 256: heads are at most 256 long
      continue;
    }
    if (c < a.d) store_one<T>(out + c, v);
  }
  if constexpr (WAVES > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += 256) {
      float v = sums[c];
#pragma unroll
      for (int k = 1; k < WAVES; ++k) v += sums[k * 256 + c];
      store_one<T>(out + c, v);
    }
  }
}

// Sums the parts of a split gradient, in order, a wave a row.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sum(const float* __restrict__ part, int splits, const int64_t* off,
                                                  int64_t most, int64_t total, int heads, int d, AttnRows out) {
  const int64_t per = (most * heads + 3) / 4, b = blockIdx.x / per;
  const int64_t i = (blockIdx.x % per) * 4 + (threadIdx.x >> 6);
  int64_t start, n;
  segment(off, b, most, total, start, n);
  if (i >= n * heads) return;
  const int64_t t = start + i / heads, h = i % heads, all = total * heads, row = t * heads + h;
  T* const o = static_cast<T*>(const_cast<void*>(out.p)) + t * out.row + h * out.head;
  for (int c = threadIdx.x & 63; c < d; c += 64) {
    float v = 0.0f;
#pragma unroll 8
    for (int s = 0; s < splits; ++s) v += part[(int64_t(s) * all + row) * d + c];
    store_one<T>(o + c, v);
  }
}

// Parts for n workgroups whose loops take `length` rows in tiles of `step`, at `per_cu`
// of them a CU at a time: where the time is least, counted in tiles of the longest part,
// times rounds of workgroups (a last one of fewer a CU is a little faster), with the
// writing and reading of a part's results, which take what some 256 rows' products of 16
// bits do or 64 of fp32.  A part has 128 rows at least and saves a twentieth at least.
// Two segments of 5000-6500 rows, 16 heads of 64 over 4, bf16: whole 626 us, in parts that
// fill all rounds 680 us; 4096 rows, 8 heads of 128, fp32: whole 632, in two parts 471.
int parts_for(int64_t n, int64_t length, int step, int per_cu, bool bf16) {
  const int64_t slots = 256 * per_cu, tiles = (length + step - 1) / step, join = (bf16 ? 256 : 64) / step;
  if (n <= 0 || n >= 8 * slots) return 1;
  int64_t best = 1;
  double least = INFINITY;
  for (int64_t s = 1; s <= kParts && (s == 1 || s <= length / 128); ++s) {
    const int64_t left = (n * s) % slots, longest = (tiles + s - 1) / s + (s > 1 ? join : 0);
    const double last = left ? 0.5 * (1.0 + double((left + 255) / 256) / per_cu) : 0.0;
    const double time = (double((n * s) / slots) + last) * double(longest);
    if (time < 0.95 * least) least = time, best = s;
  }
  return int(best);
}

}  // namespace

int attn_padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }

int dq_rows_a_tile(const AttnArgs& a) {
  const int DP = attn_padded(a.d), parts = a.bf16 ? 1 : 3;
  const int64_t rows = a.max_q * a.G;
  if (!a.bias) return rows_a_tile(rows);
  if (!a.bf16 && DP > 192) return 64;
  // LDS: two tiles of 32 rows, positions, the bias, a column of sums a lane
  auto lds = [&](int64_t lanes) {
    return 2 * 32 * parts * (2 * DP + 16) + 384 + (a.G * bias_stride(a.buckets) + lanes * a.buckets) * 4;
  };
  const int64_t all = 160 << 10;
  return rows >= 512 && DP * (a.bf16 ? 2 : 4) <= 256 && lds(256) > all / 2 && lds(512) <= all ? 256 : rows_a_tile(rows);
}

// Workgroups that a CU holds: by the waves a SIMD that the kernels' registers are cut for.
int attn_row_splits(const AttnArgs& a, bool backward) {
  const int BM = backward ? dq_rows_a_tile(a) : rows_a_tile(a.max_q * a.G), DP = attn_padded(a.d);
  const int waves = DP * (a.bf16 ? 2 : 4) <= 256 || (!backward && DP <= 128) ? 2 : 1;
  return parts_for((a.max_q * a.G + BM - 1) / BM * a.Hk * a.B, a.max_k, backward ? 32 : 32 * key_tiles(DP, a.bf16),
                   waves * 128 / BM, a.bf16);
}
int attn_key_splits(const AttnArgs& a) {
  const int BK = rows_a_tile(a.max_k), DP = attn_padded(a.d), bytes = DP * (a.bf16 ? 2 : 4);
  return parts_for((a.max_k + BK - 1) / BK * (DP > 128 ? 2 : 1) * a.Hk * a.B, a.max_q * a.G, bytes <= 128 ? 64 : 32,
                   (bytes <= (a.bf16 ? a.bias ? 192 : 256 : 128) ? 2 : 1) * 128 / BK, a.bf16);
}

hipError_t launch_attn_sum(const AttnArgs& a, const float* part, int splits, bool keys, const AttnRows& out,
                           hipStream_t s) {
  const int64_t* off = keys ? a.k_off : a.q_off;
  const int64_t most = keys ? a.max_k : a.max_q, total = keys ? a.Tk : a.Tq;
  const int heads = keys ? a.Hk : a.H;
  const uint32_t n = uint32_t((most * heads + 3) / 4 * a.B);
  if (n == 0) return hipSuccess;
  if (a.bf16)
    k_attn_sum<uint16_t><<<n, 256, 0, s>>>(part, splits, off, most, total, heads, a.d, out);
  else
    k_attn_sum<float><<<n, 256, 0, s>>>(part, splits, off, most, total, heads, a.d, out);
  return hipGetLastError();
}

template <typename T>
void join(const AttnArgs& a, hipStream_t s) {
  // four waves a row for many parts, whose loads one wave waits for eight at a time (32 rows
  // of 64: 64 parts by one wave 6.1 us, 125 by four 4.6); few parts of many rows want
  // fewer workgroups
  if (a.splits > 16)
    k_attn_join<T, 4><<<uint32_t(a.max_q * a.H * a.B), 256, 0, s>>>(a);
  else
    k_attn_join<T, 1><<<uint32_t((a.max_q * a.H + 3) / 4 * a.B), 256, 0, s>>>(a);
}

hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t s) {
  if (a.bytes)
    launch_attn_fwd_bytes(a, s);
  else if (a.bias)
    launch_attn_fwd_bias(a, s);
  else
    launch_fwd_kernel<kNoBias>(a, s);
  if (a.splits > 1) a.bf16 ? join<uint16_t>(a, s) : join<float>(a, s);
  return hipGetLastError();
}

}  // namespace gtp
