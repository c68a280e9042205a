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
#pragma once

#include "gtp_attn_core.hpp"
#include "gtp_norm_core.hpp"

namespace gtp {
namespace {

// Workgroup: 32 NW rows of one key head (a wave 32), keys in tiles of 32.
//
// BIAS: dbias[h, b] is the sum of dS over the pairs of bucket b.  Each lane adds its scores' dS to
// its own column of [buckets] sums in LDS (64 lanes on 64 banks; one lane alone adds to a word,
// so the order of its additions, and with it the result, is always the same); at the end the
// columns of a query head are added, and what the workgroups leave by launch_attn_bias_sum.
// The LDS's own fp32 addition took 260 cycles a wave: dq and dbias of two clusters of 3500-4300
// rows, 16 heads of 64 over 4, 64 buckets, bf16: 4051 us, by reading and writing 870, with the
// buckets made ahead and the heads' tables on different banks 720 (two waves a SIMD: vector unit
// 56 % busy, matrix unit 16 %, LDS 16 %).  fp32, two of 1777-2001, 8 heads of 64: 169 us.
template <typename T, int DP, bool DROP, int BIAS, int NW>
__global__ __launch_bounds__(64 * NW, (waves_per_simd<T, DP>())) void k_attn_dq(const AttnArgs a, int64_t n_wg, int tiles) {
  constexpr int NT = 64 * NW, BM = 32 * NW, BN = 32, NC = DP / 16, NDT = DP / 32;
  __shared__ __align__(16) char tk[tile_bytes<T, DP, BN>()];
  __shared__ __align__(16) char tv[tile_bytes<T, DP, BN>()];
  lds_poison(reinterpret_cast<float*>(tk), int(sizeof(tk) / 4));
  lds_poison(reinterpret_cast<float*>(tv), int(sizeof(tv) / 4));
  // kBias: positions of the tile's keys [3][BN]; a bias: it [G][bias_stride], the lanes' sums [buckets][NT]
  extern __shared__ __align__(16) float more[];
  const Work w(blockIdx.x, n_wg, tiles, a.splits, a.Hk);
  int64_t qs, nq, ks, nk;
  segment(a.q_off, w.b, a.max_q, a.Tq, qs, nq);
  segment(a.k_off, w.b, a.max_k, a.Tk, ks, nk);
  const int64_t rows = nq * a.G;
  constexpr int POS = BIAS == kBias ? 3 * BN : 0;
  float* const table = more + POS;
  float* const sums = table + a.G * bias_stride(a.buckets);
  float* const left = BIAS && a.dbias ? a.bias_part + (((w.hk * a.B + w.b) * a.splits + w.split) * tiles + w.tile) *
                                                          (int64_t(a.G) * a.buckets)
                                      : nullptr;
  if (int64_t(w.tile) * BM >= rows) {
    if (left)
      for (int i = threadIdx.x; i < a.G * a.buckets; i += NT) left[i] = 0.0f;
    return;
  }
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
  // The matrix unit's sums are cut downwards, some 2^-27 of a value's size on average, which a
  // bucket's sum of many dS of both signs would show: every other wave, and every other part of
  // the keys, has dout with its sign turned.
  const float turn = BIAS && ((wave ^ w.tile ^ w.split ^ int(w.b)) & 1) ? -1.0f : 1.0f;
  if (BIAS && turn < 0.0f) gf.negate();
  // rows without a key, and rows past the end: every exponential is zero
  const float lse = there ? a.lse[qi * a.H + h] : -INFINITY;
  const float ref = lse == -INFINITY ? INFINITY : lse * kLog2e;
  const float delta = there ? a.delta[qi * a.H + h] : 0.0f;
  f32x16 acc[NDT];
#pragma unroll
  for (int i = 0; i < NDT; ++i) acc[i] = zero16();
  Drop drop;
  if constexpr (DROP) drop.init(a, w.b, w.hk);

  float px = 0.0f, py = 0.0f, pz = 0.0f;
  const u32x4* bytes = nullptr;
  u32x4 ahead;
  if constexpr (BIAS != kNoBias) {
    lds_poison(more, POS + a.G * bias_stride(a.buckets) + (left ? a.buckets * NT : 0));
    if (left)
      for (int i = 0; i < a.buckets; ++i) sums[i * NT + threadIdx.x] = 0.0f;
    if constexpr (BIAS == kBias)
      px = a.q_pos[3 * qi], py = a.q_pos[3 * qi + 1], pz = a.q_pos[3 * qi + 2];
    else
      bytes = bucket_bytes(a.bytes, w.b, bytes_tiles(a.max_q), bytes_tiles(a.max_k), qi - qs, hi);
  }
  const float* const own = table + g * bias_stride(a.buckets);
  const Buckets bucket(a);

  const T* const kb = static_cast<const T*>(a.k.p) + ks * a.k.row + w.hk * a.k.head;
  const T* const vb = static_cast<const T*>(a.v.p) + ks * a.v.row + w.hk * a.v.head;
  const uint8_t* const mask = a.mask ? a.mask + ks : nullptr;
  const int64_t ntile = (nk + BN - 1) / BN, per = (ntile + a.splits - 1) / a.splits;
  const int64_t j_end = (w.split + 1) * per * BN < nk ? (w.split + 1) * per * BN : nk;
  Stage<T, DP, BN, NT> sk, sv;
  Present<BN> here;
  StagedPos<BN> sp;
  auto fetch = [&](int64_t j0) {
    here.fetch(mask, kb, j0, nk, lane);
    if constexpr (BIAS == kBias) {
      const int64_t j = j0 + (threadIdx.x & (BN - 1));
      sp.fetch(a.k_pos, ks + (j < nk ? j : j0));
    }
    if constexpr (BIAS == kBiasBytes) ahead = bytes[(j0 >> 5) * 64];
    sk.fetch([&](int r) { return kb + (j0 + r < nk ? j0 + r : j0) * a.k.row; }, a.d, a.vec);
    sv.fetch([&](int r) { return vb + (j0 + r < nk ? j0 + r : j0) * a.v.row; }, a.d, a.vec);
  };
  int64_t j0 = w.split * per * BN;
  constexpr bool AHEAD = !long_rows<T, DP>();
  if (AHEAD && j0 < j_end) fetch(j0);
  if constexpr (BIAS != kNoBias) load_bias(a, w.hk, table);  // behind the first tile's loads; the loop's barriers stand before its use
  for (; j0 < j_end; j0 += BN) {
    if (!AHEAD) fetch(j0);
    __syncthreads();
    const bool whole = !mask && j0 + BN <= nk;
    const uint64_t keys = here.rows(mask, j0, nk, lane);  // zeros stand for absent keys' rows
    sk.commit(tk, a.d, a.vec, whole, keys);
    sv.commit(tv, a.d, a.vec, whole, keys);
    if constexpr (BIAS == kBias) sp.commit(more);
    __syncthreads();
    u32x4 pairs;
    if constexpr (BIAS == kBiasBytes) pairs = ahead;
    if (AHEAD && j0 + BN < j_end) fetch(j0 + BN);  // in flight while this tile is worked on
    f32x16 s = zero16(), dp = zero16();
#pragma unroll
    for (int c = 0; c < NC; ++c)
      mma2<T>(tile_operand<T, DP, BN>(tk, l31, c, hi), qf(c), s, tile_operand<T, DP, BN>(tv, l31, c, hi), gf(c), dp);
    uint32_t keep = 0xffffu;
    if constexpr (DROP) keep = drop.keys_of_row(R0, j0, lane);
    uint32_t in[BIAS == kBias ? 16 : 1];  // the scores' buckets
    // where score r's bias, and its lane's sum, are
    auto bias_at = [&](int r) { return BIAS == kBias ? own[in[r]] : word_at(own, bucket_byte(pairs, r)); };
    auto sum_at = [&](int r) {
      return reinterpret_cast<float*>(reinterpret_cast<char*>(sums + threadIdx.x) +
                                      (BIAS == kBias ? 4 * in[r] : bucket_byte(pairs, r)) * NT);
    };
    auto one_bucket = [&](int r, int k) {
      return BIAS == kBias ? in[r] == in[k] : bucket_byte(pairs, r) == bucket_byte(pairs, k);
    };
    if constexpr (BIAS == kBiasBytes)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, bias_at(r));
    if constexpr (BIAS == kBias) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* const at = more + 8 * i + 4 * hi;
        const f32x4 x = *reinterpret_cast<const f32x4*>(at), y = *reinterpret_cast<const f32x4*>(at + BN),
                    z = *reinterpret_cast<const f32x4*>(at + 2 * BN);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 4 * i + j;
          in[r] = bucket(px - x[j], py - y[j], pz - z[j]);
          s[r] = fmaf(s[r], a.scale2, bias_at(r));
        }
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = pow2(BIAS ? s[r] - ref : fmaf(s[r], a.scale2, -ref));
      if constexpr (BIAS != kNoBias) {
        s[r] = p * (DROP ? Drop::kept(dp[r] * (a.keep * turn), keep, r) - delta : fmaf(dp[r], turn, -delta));
      } else {
        const float g = DROP ? Drop::kept(dp[r] * a.keep, keep, r) : dp[r];
        s[r] = p * (g - delta);
      }
    }
    if (!whole) {
      const uint32_t ok = uint32_t(keys) >> (4 * hi);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (ok >> tile_row(r, 0)) & 1u ? s[r] : 0.0f;
    }
    if constexpr (BIAS != kNoBias) {
      if (left) {
        // four at a time: their words are read together, and where two of them are one word, the
        // last one's writer adds them all (first together: a word is larger than what comes to it, and
        // one rounding at its size instead of four halves their error)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float *at[4], v[4], u[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) at[j] = sum_at(4 * i + j);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = *at[j];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float before = 0.0f;
#pragma unroll
            for (int k = 0; k < j; ++k) before = one_bucket(4 * i + k, 4 * i + j) ? u[k] : before;
            u[j] = before + s[4 * i + j];
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += u[j];
#pragma unroll
          for (int j = 0; j < 4; ++j) *at[j] = v[j];
        }
      }
    }
    const Columns<T> ds(s);
    mma_turned<T, DP, BN>(tk, 0, 0, ds, lane, acc);
  }
  if constexpr (BIAS != kNoBias) {
    if (left) {
      // which columns count for query head h: rows past the end and empty rows (of which 0 times an infinity may
      // be NaN) count for none
      int* const of = reinterpret_cast<int*>(tk);
      __syncthreads();
      of[threadIdx.x] = there && lse != -INFINITY ? g : -1;
      __syncthreads();
      for (int b = wave; b < a.buckets; b += NW)
        for (int h0 = 0; h0 < a.G; ++h0) {
          float v = 0.0f;
#pragma unroll
          for (int i = 0; i < NW; ++i) v += of[64 * i + lane] == h0 ? sums[b * NT + 64 * i + lane] : 0.0f;
          v = wave_sum(v);
          if (lane == 0) left[h0 * a.buckets + b] = v;
        }
    }
  }
  if (!there || !a.out.p) return;
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

template <typename T, int DP, bool DROP, int BIAS>
void launch_tiles(const AttnArgs& a, hipStream_t s) {
  const int64_t BM = dq_rows_a_tile(a), tiles = (a.max_q * a.G + BM - 1) / BM, n = tiles * a.splits * a.Hk * a.B;
  const size_t lds = BIAS ? ((BIAS == kBias ? 3 * 32 : 0) + size_t(a.G) * bias_stride(a.buckets) + (a.dbias ? size_t(a.buckets) * 2 * BM : 0)) * 4 : 0;
  if constexpr (BIAS != kNoBias && waves_per_simd<T, DP>() == 2)
    if (BM == 256) {
      k_attn_dq<T, DP, DROP, BIAS, 8><<<uint32_t(n), 512, lds, s>>>(a, n, int(tiles));
      return;
    }
  if constexpr (BIAS == kBiasBytes)  // made for long segments only
    k_attn_dq<T, DP, DROP, BIAS, 4><<<uint32_t(n), 256, lds, s>>>(a, n, int(tiles));
  else if (BM == 64)
    k_attn_dq<T, DP, DROP, BIAS, 2><<<uint32_t(n), 128, lds, s>>>(a, n, int(tiles));
  else
    k_attn_dq<T, DP, DROP, BIAS, 4><<<uint32_t(n), 256, lds, s>>>(a, n, int(tiles));
}

template <typename T, int DP, int BIAS>
void launch_dq_tiles(const AttnArgs& a, hipStream_t s) {
  if (a.threshold)
    launch_tiles<T, DP, true, BIAS>(a, s);
  else
    launch_tiles<T, DP, false, BIAS>(a, s);
}

template <int BIAS>
void launch_dq_kernel(const AttnArgs& a, hipStream_t s) {
  switch (attn_padded(a.d)) {
    case 32: return a.bf16 ? launch_dq_tiles<uint16_t, 32, BIAS>(a, s) : launch_dq_tiles<float, 32, BIAS>(a, s);
    case 64: return a.bf16 ? launch_dq_tiles<uint16_t, 64, BIAS>(a, s) : launch_dq_tiles<float, 64, BIAS>(a, s);
    case 96: return a.bf16 ? launch_dq_tiles<uint16_t, 96, BIAS>(a, s) : launch_dq_tiles<float, 96, BIAS>(a, s);
    case 128: return a.bf16 ? launch_dq_tiles<uint16_t, 128, BIAS>(a, s) : launch_dq_tiles<float, 128, BIAS>(a, s);
    case 192: return a.bf16 ? launch_dq_tiles<uint16_t, 192, BIAS>(a, s) : launch_dq_tiles<float, 192, BIAS>(a, s);
    default: return a.bf16 ? launch_dq_tiles<uint16_t, 256, BIAS>(a, s) : launch_dq_tiles<float, 256, BIAS>(a, s);
  }
}

}  // namespace
}  // namespace gtp
