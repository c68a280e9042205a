// Softmax attention, forward: o = softmax(scale q k^T) v over the keys of a
// row's segment, in one pass over the keys with the running maximum and sum of
// each row, and lse = log of the row's sum (the backward pass makes the
// probabilities again from it).
//
//   m' = max(m, scores of the tile),  l' = l 2^(m - m') + sum 2^(s - m'),
//   o' = o 2^(m - m') + 2^(s - m') v,  o = o' / l'  (scores in units of log 2).
// Probabilities are rounded to the operands' type (bf16: up to 2^-8 of each, as the inputs
// themselves are; fp32: in three parts, below an fp32 rounding), their sum l is of the
// unrounded ones in fp32.
//
// Long segments: a workgroup's four waves share the staged keys and values, each for 32
// rows, so a staged tile is used 128 times; two waves a SIMD, one with vector
// instructions (exponentials, rounding, the row's statistics) while the other's products
// run.  In bf16 the vector unit is the busier: 8192 rows, 8 heads of 128: 328-372 us,
// 740-838 TFLOP/s (library products of that type here: 1200), vector unit busy 41 % of the
// cycles, matrix unit 35 %, LDS bank conflicts in 26 %; two segments of 5000-6500 rows, 16
// heads of 64 over 4, with as many exponentials for half the products: 594-629 us, 440-463
// TFLOP/s, vector unit 56 %, matrix unit 25 %; with dropped probabilities 1094 us, of which
// the draws are 480 (8 heads of 128: 531).  fp32, 4096 rows, 8 heads of 128: 425-471 us,
// 146-162 TFLOP/s (library products: 154).
// Few rows: the keys' way from HBM bounds it, so they are dealt to parts, in workgroups of
// 64 rows, four a CU; one row of 8 heads of 128 against 60000 keys, bf16: 57-63 us, 3.9-4.3
// TB/s.  In fp32 it does not get there: 8 rows of 8 heads of 100 against 7000-8001 keys 522
// us, 0.7 TB/s (bf16: 62 us, 3.1).  The staging registers double with half the threads, and
// heads of 97-128 keep 348 bytes a lane in scratch memory (heads of 65-96: 216; bf16 heads of
// 97-128: 68); and of the two waves one works on rows that are not there.
// Molecules of 5 to 49 atoms: one short pass, waits one after the other (offsets, rows,
// keys, products), on that two-wave form: 64 of them, 8 heads of 72, fp32: 21.4-22.8 us.
// Heads above 128 fill the registers with one wave a SIMD, fp32 ones spill (372 bytes a lane
// at 193-256): 4001 rows, 4 heads of 200: bf16 176 us, 291 TFLOP/s, fp32 730 us, 70.
// With a bias by distance (see Buckets) a score takes twice the vector instructions, 20 instead of 10, or, with its
// bucket made ahead for all heads (gtp_attn_bytes.hip), 11 and an LDS read.  8192 rows, 8 heads of 128, 32 buckets,
// bf16: 549 us so, 447 with the buckets made ahead (their making 20 of it).  Molecules as above: 25.3 us.
// fp32, 8192 rows, 8 heads of 128: 1715 us (without a bias 1590), two of 1777-2001 rows, 8 heads of 64: 140 (122).  Few rows: 4
// against 15000-16001 keys, 8 heads over 2 of 64: bf16 28 us (22), fp32 66 (57); one against 60000, 8 heads of 128: bf16 123 (65),
// fp32 442 (381): workgroups of 64 rows, whose buckets and bias spill there (196 and 376 bytes a lane).
#pragma once

#include "gtp_attn_core.hpp"

namespace gtp {

// Tiles of 32 keys that the forward takes at a time.
constexpr int key_tiles(int DP, bool bf16) { return !bf16 && DP > 64 ? 1 : 2; }

namespace {

constexpr float kSlack = 8.0f;  // probabilities stay below 2^8: far from overflow in fp32 and bf16, and as exact

// Workgroup: 32 NW rows of one key head (a wave 32), keys in tiles of 32 KT.  Heads longer
// than 128 leave the registers room for one wave a SIMD only.
template <typename T, int DP, int KT, bool DROP, int BIAS, int NW>
__global__ __launch_bounds__(64 * NW, DP <= 128 ? 2 : 1) void k_attn_fwd(const AttnArgs a, int64_t n_wg, int tiles) {
  constexpr int NT = 64 * NW, BM = 32 * NW, BN = 32 * KT, NC = DP / 16, NDT = DP / 32;
  __shared__ __align__(16) char tk[tile_bytes<T, DP, BN>()];
  __shared__ __align__(16) char tv[tile_bytes<T, DP, BN>()];
  lds_poison(reinterpret_cast<float*>(tk), int(sizeof(tk) / 4));
  lds_poison(reinterpret_cast<float*>(tv), int(sizeof(tv) / 4));
  extern __shared__ __align__(16) float more[];  // kBias: positions of the tile's keys [3][BN]; a bias: it [G][bias_stride]
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
  // the scores' scale is taken positive, its sign into q: their maximum is then that of the products
  const float scale2 = fabsf(a.scale2);
  RowOperands<T, DP, long_rows<T, DP>()> qf;
  qf.load(static_cast<const T*>(a.q.p) + qi * a.q.row + h * a.q.head, there, hi, a.d, a.vec);
  if (a.scale2 < 0.0f) qf.negate();
  float px = 0.0f, py = 0.0f, pz = 0.0f;
  const float* table = nullptr;
  constexpr int POS = BIAS == kBias ? 3 * BN : 0;
  const u32x4* bytes = nullptr;
  u32x4 ahead[BIAS == kBiasBytes ? KT : 1];
  if constexpr (BIAS != kNoBias) {
    lds_poison(more, POS + a.G * bias_stride(a.buckets));
    table = more + POS + g * bias_stride(a.buckets);
    if constexpr (BIAS == kBias)
      px = a.q_pos[3 * qi], py = a.q_pos[3 * qi + 1], pz = a.q_pos[3 * qi + 2];
    else
      bytes = bucket_bytes(a.bytes, w.b, bytes_tiles(a.max_q), bytes_tiles(a.max_k), qi - qs, hi);
  }
  const Buckets bucket(a);
  f32x16 acc[NDT];
#pragma unroll
  for (int i = 0; i < NDT; ++i) acc[i] = zero16();
  // m: the reference of the row's exponentials in units of log 2, at most kSlack below its largest score so far;
  // l: this half's part of their sum
  float m = -INFINITY, l = 0.0f;
  Drop drop;
  if constexpr (DROP) drop.init(a, w.b, w.hk);

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
    if constexpr (BIAS == kBiasBytes)
#pragma unroll
      for (int t = 0; t < KT; ++t) ahead[t] = bytes[((j0 >> 5) + t) * 64];
    sk.fetch([&](int r) { return kb + (j0 + r < nk ? j0 + r : j0) * a.k.row; }, a.d, a.vec);
    sv.fetch([&](int r) { return vb + (j0 + r < nk ? j0 + r : j0) * a.v.row; }, a.d, a.vec);
  };
  int64_t j0 = w.split * per * BN;
  constexpr bool AHEAD = !long_rows<T, DP>();
  if (AHEAD && j0 < j_end) fetch(j0);
  if constexpr (BIAS != kNoBias) load_bias(a, w.hk, more + POS);  // behind the first tile's loads; the loop's barriers stand before its use
  for (; j0 < j_end; j0 += BN) {
    if (!AHEAD) fetch(j0);
    __syncthreads();
    const bool whole = !mask && j0 + BN <= nk;
    const uint64_t keys = here.rows(mask, j0, nk, lane);  // zeros stand for absent keys' rows
    sk.commit(tk, a.d, a.vec, whole, keys);
    sv.commit(tv, a.d, a.vec, whole, keys);
    if constexpr (BIAS == kBias) sp.commit(more);
    __syncthreads();
    u32x4 in[BIAS == kBiasBytes ? KT : 1];
    if constexpr (BIAS == kBiasBytes)
#pragma unroll
      for (int t = 0; t < KT; ++t) in[t] = ahead[t];
    if (AHEAD && j0 + BN < j_end) fetch(j0 + BN);  // in flight while this tile is worked on
    f32x16 s[KT];
    uint32_t ok[KT];
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < KT; ++t) s[t] = zero16();
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const Operand<T> q = qf(c);
      if constexpr (KT == 2)
        mma2<T>(tile_operand<T, DP, BN>(tk, l31, c, hi), q, s[0], tile_operand<T, DP, BN>(tk, 32 + l31, c, hi), q, s[1]);
      else
        mma<T>(tile_operand<T, DP, BN>(tk, l31, c, hi), q, s[0]);
    }
    if constexpr (BIAS == kBiasBytes) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = fmaf(s[t][r], scale2, word_at(table, bucket_byte(in[t], r)));
    }
    if constexpr (BIAS == kBias) {  // scores in units of log 2 from here on
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* const at = more + 32 * t + 8 * i + 4 * hi;
          const f32x4 x = *reinterpret_cast<const f32x4*>(at), y = *reinterpret_cast<const f32x4*>(at + BN),
                      z = *reinterpret_cast<const f32x4*>(at + 2 * BN);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float b = table[bucket(px - x[j], py - y[j], pz - z[j])];
            s[t][4 * i + j] = fmaf(s[t][4 * i + j], scale2, b);
          }
        }
    }
    if (!whole) {
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        ok[t] = uint32_t(keys >> (32 * t)) >> (4 * hi);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = (ok[t] >> tile_row(r, 0)) & 1u ? s[t][r] : -INFINITY;
      }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
    top = BIAS ? half_max(top) : half_max(top) * scale2;
    // the reference moves only where a score passes it by kSlack: the accumulators are seldom scaled
    if (__any(top > m + kSlack)) {
      const float m_new = fmaxf(m, top);
      const float f = m_new == m ? 1.0f : pow2(m - m_new);
      m = m_new;
      l *= f;
#pragma unroll
      for (int i = 0; i < NDT; ++i) acc[i] *= f;
    }
    const float ref = m == -INFINITY ? 0.0f : m;  // no score yet: every exponential below is zero
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      uint32_t keep = 0xffffu;
      if constexpr (DROP) keep = drop.keys_of_row(R0, j0 + 32 * t, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = pow2(BIAS ? s[t][r] - ref : fmaf(s[t][r], scale2, -ref));
      if (!whole) {  // also where scale is 0
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = (ok[t] >> tile_row(r, 0)) & 1u ? s[t][r] : 0.0f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        l += s[t][r];
        if constexpr (DROP) s[t][r] = Drop::kept(s[t][r], keep, r);
      }
      const Columns<T> p(s[t]);
      mma_turned<T, DP, BN>(tv, 32 * t, 0, p, lane, acc);
    }
  }
  l = half_sum(l);
  if (!there) return;
  if (BIAS != kNoBias && l == 0.0f)  // nothing within the cutoff: zeros, whatever v holds (0 times infinity would be NaN)
#pragma unroll
    for (int i = 0; i < NDT; ++i) acc[i] = zero16();
  const float inv = l == 0.0f ? 0.0f : (DROP ? a.keep / l : 1.0f / l);
  const float lse = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
  if (a.splits > 1) {
    const int64_t all = a.Tq * a.H, row = qi * a.H + h;
    store_columns<float>(part_row(a.part, w.split, all, row, a.d), acc, inv, 0, a.d, hi, a.d % 4 == 0);
    if (hi == 0) a.part[a.splits * all * a.d + w.split * all + row] = lse;
    return;
  }
  store_columns<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + qi * a.out.row + h * a.out.head, acc, inv, 0, a.d, hi,
                   a.vec);
  if (hi == 0) a.lse[qi * a.H + h] = lse;
}

template <typename T, int DP, bool DROP, int BIAS>
void launch_tiles(const AttnArgs& a, hipStream_t s) {
  constexpr int KT = key_tiles(DP, sizeof(T) == 2);
  const int64_t BM = rows_a_tile(a.max_q * a.G), tiles = (a.max_q * a.G + BM - 1) / BM, n = tiles * a.splits * a.Hk * a.B;
  const size_t lds = BIAS ? ((BIAS == kBias ? 3 * 32 * KT : 0) + size_t(a.G) * bias_stride(a.buckets)) * 4 : 0;
  if constexpr (BIAS == kBiasBytes)  // made for long segments only
    k_attn_fwd<T, DP, KT, DROP, BIAS, 4><<<uint32_t(n), 256, lds, s>>>(a, n, int(tiles));
  else if (BM == 64)
    k_attn_fwd<T, DP, KT, DROP, BIAS, 2><<<uint32_t(n), 128, lds, s>>>(a, n, int(tiles));
  else
    k_attn_fwd<T, DP, KT, DROP, BIAS, 4><<<uint32_t(n), 256, lds, s>>>(a, n, int(tiles));
}

template <typename T, int DP, int BIAS>
void launch_fwd_tiles(const AttnArgs& a, hipStream_t s) {
  if (a.threshold)
    launch_tiles<T, DP, true, BIAS>(a, s);
  else
    launch_tiles<T, DP, false, BIAS>(a, s);
}

template <int BIAS>
void launch_fwd_kernel(const AttnArgs& a, hipStream_t s) {
  switch (attn_padded(a.d)) {
    case 32: return a.bf16 ? launch_fwd_tiles<uint16_t, 32, BIAS>(a, s) : launch_fwd_tiles<float, 32, BIAS>(a, s);
    case 64: return a.bf16 ? launch_fwd_tiles<uint16_t, 64, BIAS>(a, s) : launch_fwd_tiles<float, 64, BIAS>(a, s);
    case 96: return a.bf16 ? launch_fwd_tiles<uint16_t, 96, BIAS>(a, s) : launch_fwd_tiles<float, 96, BIAS>(a, s);
    case 128: return a.bf16 ? launch_fwd_tiles<uint16_t, 128, BIAS>(a, s) : launch_fwd_tiles<float, 128, BIAS>(a, s);
    case 192: return a.bf16 ? launch_fwd_tiles<uint16_t, 192, BIAS>(a, s) : launch_fwd_tiles<float, 192, BIAS>(a, s);
    default: return a.bf16 ? launch_fwd_tiles<uint16_t, 256, BIAS>(a, s) : launch_fwd_tiles<float, 256, BIAS>(a, s);
  }
}

}  // namespace
}  // namespace gtp
