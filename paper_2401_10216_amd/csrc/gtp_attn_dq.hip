// Softmax attention, gradient of the queries: the probabilities are made again
// from the scores and the rows' lse,
//   P = exp(scale q k^T - lse),  dP = (dout v^T) m,  dS = P (dP - delta),
//   dq = scale dS k,  delta = rows' sums of dout o,
// m the factors 0 or 1 / (1 - p) of dropped probabilities (made again from the
// generator, not stored).  dS is rounded to the operands' type for the last product
// (fp32: in three parts).
//
// The rows lie as in the forward: a wave's 32 rows are the columns of its products,
// their q and dout in registers, keys and values staged for all waves.  dq and dk, dv
// each make S and dP for themselves: one kernel for all three would add to one of them
// with atomics, whose order changes the result.  The long cases (6 d flops a row and key)
// wait for matrix and vector unit by turns: fp32 heads longer than 64 leave room for one
// wave a SIMD.  4001 rows, 8 heads of 100, fp32: 622-664 us, 116-123 TFLOP/s, matrix unit
// busy 39 % of the cycles, vector unit 32 %; 8192 rows, 8 heads of 128, bf16: 440-472 us,
// 873-937 TFLOP/s, 39 % and 35 %.  Where probabilities are dropped, the draws add vector work
// of more than half of that (two segments of 5000-6500 rows, 16 heads of 64 over 4, bf16:
// 1028-1108 us with, 634-688 without).  fp32 heads above 128 keep 344 bytes a lane in scratch
// memory (193-256: 712; on two-wave workgroups 908 and 1120) although their rows stay
// unsplit: 4001 rows, 4 heads of 200, both gradients 2883 us (bf16: 690).
#include "gtp_attn_core.hpp"

namespace gtp {
namespace {

// delta[t, h] = sum_i dout[t, h, i] o[t, h, i]: 16 lanes a row.  In a
// pass of its own, once for both gradients: dout and o read once, HBM's time for the long
// cases and a launch's (4 us) for the short.
constexpr uint32_t kDeltaGrid = 1u << 20;  // workgroups at most: a launch holds less than 2^32 threads
template <typename T>
__global__ __launch_bounds__(256) void k_attn_delta(const AttnArgs a) {
  const int64_t n = a.Tq * a.H;
  const int i0 = threadIdx.x & 15;
  for (int64_t id = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); id < n; id += int64_t(gridDim.x) * 16) {
    const int64_t t = id / a.H, h = id % a.H;
    const T* o = static_cast<const T*>(a.o.p) + t * a.o.row + h * a.o.head;
    const T* g = static_cast<const T*>(a.dout.p) + t * a.dout.row + h * a.dout.head;
    float s = 0.0f;
    for (int i = i0; i < a.d; i += 16) s = fmaf(to_f32<T>(o[i]), to_f32<T>(g[i]), s);
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) s += __shfl_xor(s, x);  // a row's lanes are in the loop together
    if (i0 == 0) a.delta[id] = s;
  }
}

// Workgroup: 32 NW rows of one key head (a wave 32), keys in tiles of 32.
template <typename T, int DP, bool DROP, int NW>
__global__ __launch_bounds__(64 * NW, (waves_per_simd<T, DP>())) void k_attn_dq(const AttnArgs a, int64_t n_wg, int tiles) {
  constexpr int NT = 64 * NW, BM = 32 * NW, BN = 32, NC = DP / 16, NDT = DP / 32;
  __shared__ __align__(16) char tk[tile_bytes<T, DP, BN>()];
  __shared__ __align__(16) char tv[tile_bytes<T, DP, BN>()];
  lds_poison(reinterpret_cast<float*>(tk), int(sizeof(tk) / 4));
  lds_poison(reinterpret_cast<float*>(tv), int(sizeof(tv) / 4));
  const Work w(blockIdx.x, n_wg, tiles, a.splits, a.Hk);
  int64_t qs, nq, ks, nk;
  segment(a.q_off, w.b, a.max_q, a.Tq, qs, nq);
  segment(a.k_off, w.b, a.max_k, a.Tk, ks, nk);
  const int64_t rows = nq * a.G;
  if (int64_t(w.tile) * BM >= rows) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l31 = lane & 31, hi = lane >> 5;
  const int64_t R0 = int64_t(w.tile) * BM + wave * 32, R = R0 + l31;
  const bool there = R < rows;
  const int64_t Rc = there ? R : rows - 1;  // a row past the end reads the last one and counts nothing
  int g;
  const int64_t qi = qs + Group(a.G).row(Rc, &g);
  const int h = w.hk * a.G + g;
  RowOperands<T, DP, long_rows<T, DP>()> qf, gf;
  qf.load(static_cast<const T*>(a.q.p) + qi * a.q.row + h * a.q.head, there, hi, a.d, a.vec);
  gf.load(static_cast<const T*>(a.dout.p) + qi * a.dout.row + h * a.dout.head, there, hi, a.d, a.vec);
  // rows without a key, and rows past the end: every exponential is zero
  const float lse = there ? a.lse[qi * a.H + h] : -INFINITY;
  const float ref = lse == -INFINITY ? INFINITY : lse * kLog2e;
  const float delta = there ? a.delta[qi * a.H + h] : 0.0f;
  f32x16 acc[NDT];
#pragma unroll
  for (int i = 0; i < NDT; ++i) acc[i] = zero16();
  Drop drop;
  if constexpr (DROP) drop.init(a, w.b, w.hk);

  const T* const kb = static_cast<const T*>(a.k.p) + ks * a.k.row + w.hk * a.k.head;
  const T* const vb = static_cast<const T*>(a.v.p) + ks * a.v.row + w.hk * a.v.head;
  const uint8_t* const mask = a.mask ? a.mask + ks : nullptr;
  const int64_t ntile = (nk + BN - 1) / BN, per = (ntile + a.splits - 1) / a.splits;
  const int64_t j_end = (w.split + 1) * per * BN < nk ? (w.split + 1) * per * BN : nk;
  Stage<T, DP, BN, NT> sk, sv;
  Present<BN> here;
  auto fetch = [&](int64_t j0) {
    here.fetch(mask, kb, j0, nk, lane);
    sk.fetch([&](int r) { return kb + (j0 + r < nk ? j0 + r : j0) * a.k.row; }, a.d, a.vec);
    sv.fetch([&](int r) { return vb + (j0 + r < nk ? j0 + r : j0) * a.v.row; }, a.d, a.vec);
  };
  int64_t j0 = w.split * per * BN;
  constexpr bool AHEAD = !long_rows<T, DP>();
  if (AHEAD && j0 < j_end) fetch(j0);
  for (; j0 < j_end; j0 += BN) {
    if (!AHEAD) fetch(j0);
    __syncthreads();
    const bool whole = !mask && j0 + BN <= nk;
    const uint64_t keys = here.rows(mask, j0, nk, lane);  // zeros stand for absent keys' rows
    sk.commit(tk, a.d, a.vec, whole, keys);
    sv.commit(tv, a.d, a.vec, whole, keys);
    __syncthreads();
    if (AHEAD && j0 + BN < j_end) fetch(j0 + BN);  // in flight while this tile is worked on
    f32x16 s = zero16(), dp = zero16();
#pragma unroll
    for (int c = 0; c < NC; ++c)
      mma2<T>(tile_operand<T, DP, BN>(tk, l31, c, hi), qf(c), s, tile_operand<T, DP, BN>(tv, l31, c, hi), gf(c), dp);
    uint32_t keep = 0xffffu;
    if constexpr (DROP) keep = drop.keys_of_row(R0, j0, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = pow2(fmaf(s[r], a.scale2, -ref));
      const float g = DROP ? Drop::kept(dp[r] * a.keep, keep, r) : dp[r];
      s[r] = p * (g - delta);
    }
    if (!whole) {
      const uint32_t ok = uint32_t(keys) >> (4 * hi);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (ok >> tile_row(r, 0)) & 1u ? s[r] : 0.0f;
    }
    const Columns<T> ds(s);
    mma_turned<T, DP, BN>(tk, 0, 0, ds, lane, acc);
  }
  if (!there) return;
  if (lse == -INFINITY)  // an empty row: zeros, whatever k holds (a zero times an infinity would be NaN)
#pragma unroll
    for (int i = 0; i < NDT; ++i) acc[i] = zero16();
  if (a.splits > 1) {
    store_columns<float>(part_row(a.part, w.split, a.Tq * a.H, qi * a.H + h, a.d), acc, a.scale, 0, a.d, hi,
                         a.d % 4 == 0);
    return;
  }
  store_columns<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + qi * a.out.row + h * a.out.head, acc, a.scale, 0, a.d,
                   hi, a.vec);
}

template <typename T, int DP, bool DROP>
void launch_tiles(const AttnArgs& a, hipStream_t s) {
  const int64_t BM = rows_a_tile(a.max_q * a.G), tiles = (a.max_q * a.G + BM - 1) / BM, n = tiles * a.splits * a.Hk * a.B;
  if (BM == 64)
    k_attn_dq<T, DP, DROP, 2><<<uint32_t(n), 128, 0, s>>>(a, n, int(tiles));
  else
    k_attn_dq<T, DP, DROP, 4><<<uint32_t(n), 256, 0, s>>>(a, n, int(tiles));
}

template <typename T, int DP>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
  if (a.threshold)
    launch_tiles<T, DP, true>(a, s);
  else
    launch_tiles<T, DP, false>(a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_delta(const AttnArgs& a, hipStream_t s) {
  const int64_t all = (a.Tq * a.H + 15) / 16;
  const uint32_t n = all < kDeltaGrid ? uint32_t(all) : kDeltaGrid;
  if (a.bf16)
    k_attn_delta<uint16_t><<<n, 256, 0, s>>>(a);
  else
    k_attn_delta<float><<<n, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_attn_dq(const AttnArgs& a, hipStream_t s) {
  switch (attn_padded(a.d)) {
    case 32: return a.bf16 ? launch<uint16_t, 32>(a, s) : launch<float, 32>(a, s);
    case 64: return a.bf16 ? launch<uint16_t, 64>(a, s) : launch<float, 64>(a, s);
    case 96: return a.bf16 ? launch<uint16_t, 96>(a, s) : launch<float, 96>(a, s);
    case 128: return a.bf16 ? launch<uint16_t, 128>(a, s) : launch<float, 128>(a, s);
    case 192: return a.bf16 ? launch<uint16_t, 192>(a, s) : launch<float, 192>(a, s);
    default: return a.bf16 ? launch<uint16_t, 256>(a, s) : launch<float, 256>(a, s);
  }
}

}  // namespace gtp
