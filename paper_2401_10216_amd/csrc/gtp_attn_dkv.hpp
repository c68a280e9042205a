// Softmax attention, gradients of the keys and values: with P, dP, dS as for
// dq (gtp_attn_dq.hip),
//   dv = (P m)^T dout,  dk = scale dS^T q,
// summed over the rows of every query head that shares the key head, in order: the
// rows of a key head's G query heads are one axis of the loop, so shared heads cost
// no more and no atomics.
//
// A wave's 32 keys are the columns of its products, their k and v in registers, both
// accumulators too; rows of q and dout are staged for all waves.  The registers bound the
// long cases (8 d flops a row and key): two segments of 5000-6500 rows, 16 heads of 64 over
// 4, bf16, two waves a SIMD: 821-866 us, dropped 1300-1320; 4001 rows, 8 heads of 100, fp32,
// one wave a SIMD: 787-849 us, 121-130 TFLOP/s, matrix unit busy 42 % of the cycles, vector
// unit 33 %; 8192 rows, 8 heads of 128, bf16: 911-946 us, 581-604 TFLOP/s, matrix and vector
// unit 25 % each: two waves a SIMD cost it the tile ahead and 104 bytes a lane in scratch
// memory (heads of 97-128 on two-wave workgroups 140, of 65-96 there 80).
// With a bias by distance: two segments of 3500-4300 rows, 16 heads of 64 over 4, bf16 (the four rows of an atom share their
// bucket): 608 us; 1777-2001 rows, 8 heads of 64, fp32, buckets made ahead: 272 us (each made at its score: 309).
#pragma once

#include "gtp_attn_core.hpp"

namespace gtp {
namespace {

// Keys, values and both accumulators take twice what dq's rows do.
// With a bias, 16-bit heads of 97-128 on one wave with the tile ahead: two of 3500-4300 rows, 8 heads of 128, buckets made
// ahead, 859 us (two waves: 973), over 2, made at each score, 908 (1050); heads of 96, 8 over 2: 800 so, 715 on two.
template <typename T, int DP, int BIAS>
constexpr int dkv_waves() {
  return DP * int(sizeof(T)) <= 128 || (sizeof(T) == 2 && DP <= (BIAS ? 96 : 128)) ? 2 : 1;
}

// Workgroup: 32 NW keys of one key head (a wave 32), rows in tiles of 32.  Heads
// longer than 128 are dealt to `parts` workgroups by output elements (DO each):
// the accumulators of all of them would not fit the registers.
template <typename T, int DP, int DO, int RT, bool DROP, int BIAS, int NW>
__global__ __launch_bounds__(64 * NW, (dkv_waves<T, DP, BIAS>())) void k_attn_dkv(const AttnArgs a, int64_t n_wg, int tiles) {
  constexpr int NT = 64 * NW, BK = 32 * NW, BR = 32 * RT, NC = DP / 16, NDT = DO / 32, PARTS = DP / DO;
  __shared__ __align__(16) char tq[tile_bytes<T, DP, BR>()];
  __shared__ __align__(16) char tg[tile_bytes<T, DP, BR>()];
  __shared__ __align__(16) float t_ref[BR], t_delta[BR];
  __shared__ __align__(16) int t_head[BIAS == kBias ? BR : 4];  // where in `more` the bias of the row's head is
  extern __shared__ __align__(16) float more[];        // kBias: positions of the tile's rows [3][BR]; a bias: it [G][bias_stride]
  lds_poison(reinterpret_cast<float*>(tq), int(sizeof(tq) / 4));
  lds_poison(reinterpret_cast<float*>(tg), int(sizeof(tg) / 4));
  lds_poison(t_ref, BR);
  lds_poison(t_delta, BR);
  if constexpr (BIAS == kBias) lds_poison(reinterpret_cast<float*>(t_head), BR);
  const Work w(blockIdx.x, n_wg, tiles * PARTS, a.splits, a.Hk);
  const int tile = w.tile / PARTS, part = w.tile % PARTS;
  int64_t qs, nq, ks, nk;
  segment(a.q_off, w.b, a.max_q, a.Tq, qs, nq);
  segment(a.k_off, w.b, a.max_k, a.Tk, ks, nk);
  if (int64_t(tile) * BK >= nk) return;
  const int64_t rows = nq * a.G;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l31 = lane & 31, hi = lane >> 5;
  const int64_t j = int64_t(tile) * BK + wave * 32 + l31;
  const bool there = j < nk;
  const bool present = there && (!a.mask || a.mask[ks + j]);  // an absent key's row is not read; its gradients are zero
  RowOperands<T, DP, long_rows<T, DP>()> kf, vf;
  const int64_t jc = ks + (there ? j : nk - 1);
  kf.load(static_cast<const T*>(a.k.p) + jc * a.k.row + w.hk * a.k.head, present, hi, a.d, a.vec);
  vf.load(static_cast<const T*>(a.v.p) + jc * a.v.row + w.hk * a.v.head, present, hi, a.d, a.vec);
  f32x16 ak[NDT], av[NDT];
#pragma unroll
  for (int i = 0; i < NDT; ++i) ak[i] = zero16(), av[i] = zero16();
  Drop drop;
  if constexpr (DROP) drop.init(a, w.b, w.hk);
  float px = 0.0f, py = 0.0f, pz = 0.0f;
  constexpr int POS = BIAS == kBias ? 3 * BR : 0;
  const u32x4* bytes = nullptr;
  u32x4 ahead[BIAS == kBiasBytes ? RT : 1];
  if constexpr (BIAS != kNoBias) {
    lds_poison(more, POS + a.G * bias_stride(a.buckets));
    if constexpr (BIAS == kBias)
      px = a.k_pos[3 * jc], py = a.k_pos[3 * jc + 1], pz = a.k_pos[3 * jc + 2];
    else
      bytes = bucket_bytes(a.bytes_k, w.b, bytes_tiles(a.max_k), bytes_tiles(a.max_q), jc - ks, hi);
  }
  const Buckets bucket(a);

  const int64_t ntile = (rows + BR - 1) / BR, per = (ntile + a.splits - 1) / a.splits;
  const int64_t r_end = (w.split + 1) * per * BR < rows ? (w.split + 1) * per * BR : rows;
  const Group group(a.G);
  Stage<T, DP, BR, NT> sq, sg;
  float lse = 0.0f, delta = 0.0f;
  StagedPos<BR> sp;
  int head = 0;
  auto fetch = [&](int64_t r0) {
    auto row = [&](const AttnRows& t, int r) {
      int g;
      const int64_t i = group.row(r0 + r < rows ? r0 + r : r0, &g);
      return static_cast<const T*>(t.p) + (qs + i) * t.row + (w.hk * a.G + g) * t.head;
    };
    sq.fetch([&](int r) { return row(a.q, r); }, a.d, a.vec);
    sg.fetch([&](int r) { return row(a.dout, r); }, a.d, a.vec);
    int g;  // by every thread, wanted or not: under a condition these loads, and the tile's, were waited for here
    const int64_t rt = r0 + (threadIdx.x & (BR - 1)), i = group.row(rt < rows ? rt : r0, &g);
    const int64_t at = (qs + i) * a.H + w.hk * a.G + g;
    lse = a.lse[at];
    delta = a.delta[at];
    if constexpr (BIAS == kBias) {
      sp.fetch(a.q_pos, qs + i);
      head = POS + g * bias_stride(a.buckets);
    }
    if constexpr (BIAS == kBiasBytes)  // one query head a key head: rows are atoms
#pragma unroll
      for (int t = 0; t < RT; ++t) ahead[t] = bytes[((r0 >> 5) + t) * 64];
  };
  int64_t r0 = w.split * per * BR;
  constexpr bool AHEAD = !long_rows<T, DP>() && !(sizeof(T) == 2 && DP == 128 && BIAS == kNoBias);  // there the registers hold no more
  if (AHEAD && r0 < r_end) fetch(r0);
  if constexpr (BIAS != kNoBias) load_bias(a, w.hk, more + POS);  // behind the first tile's loads; the loop's barriers stand before its use
  for (; r0 < r_end; r0 += BR) {
    if (!AHEAD) fetch(r0);
    __syncthreads();
    const bool whole = r0 + BR <= rows;
    const uint64_t there_r = whole ? ~uint64_t(0) : (uint64_t(1) << (rows - r0)) - 1;  // fewer than 64 left
    sq.commit(tq, a.d, a.vec, whole, there_r);
    sg.commit(tg, a.d, a.vec, whole, there_r);
    if (threadIdx.x < BR) {
      const bool in = r0 + threadIdx.x < rows;
      t_ref[threadIdx.x] = !in || lse == -INFINITY ? INFINITY : lse * kLog2e;
      t_delta[threadIdx.x] = in ? delta : 0.0f;
      if constexpr (BIAS == kBias) t_head[threadIdx.x] = head;
    }
    if constexpr (BIAS == kBias) sp.commit(more);
    __syncthreads();
    u32x4 pairs[BIAS == kBiasBytes ? RT : 1];
    if constexpr (BIAS == kBiasBytes)
#pragma unroll
      for (int t = 0; t < RT; ++t) pairs[t] = ahead[t];
    if (AHEAD && r0 + BR < r_end) fetch(r0 + BR);  // in flight while this tile is worked on
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x16 s = zero16(), dp = zero16();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        mma2<T>(tile_operand<T, DP, BR>(tq, 32 * t + l31, c, hi), kf.template operator()<true>(c), s,
                tile_operand<T, DP, BR>(tg, 32 * t + l31, c, hi), vf.template operator()<true>(c), dp);
        if constexpr (long_rows<T, DP>()) __builtin_amdgcn_sched_barrier(0);  // a step's parts with the step: made ahead they spill
      }
      uint32_t keep = 0xffffu;
      if constexpr (DROP) keep = drop.rows_of_key(r0 + 32 * t, int64_t(tile) * BK + wave * 32, lane);
      f32x16 p;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        uint32_t in = 0;
        i32x4 head_at = {0, 0, 0, 0};
        const int row = 32 * t + 8 * g + 4 * hi;
        if constexpr (BIAS == kBias) head_at = *reinterpret_cast<const i32x4*>(t_head + row);
        const f32x4 rf = *reinterpret_cast<const f32x4*>(t_ref + 32 * t + 8 * g + 4 * hi);
        const f32x4 de = *reinterpret_cast<const f32x4*>(t_delta + 32 * t + 8 * g + 4 * hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * g + i;
          float e;
          if constexpr (BIAS == kBiasBytes) {
            e = pow2(fmaf(s[r], a.scale2, word_at(more, bucket_byte(pairs[t], r))) - rf[i]);
          } else if constexpr (BIAS == kBias) {
            // four rows of one atom, or two and two, have one distance
            if (i == 0 || (i == 2 ? (a.G & 3) != 0 : (a.G & 1) != 0))
              in = bucket(more[row + i] - px, more[BR + row + i] - py, more[2 * BR + row + i] - pz);
            e = pow2(fmaf(s[r], a.scale2, more[head_at[i] + in]) - rf[i]);
          } else {
            e = pow2(fmaf(s[r], a.scale2, -rf[i]));
          }
          if constexpr (DROP) {
            p[r] = Drop::kept(e, keep, r);
            s[r] = e * (Drop::kept(dp[r] * a.keep, keep, r) - de[i]);
          } else {
            p[r] = e;
            s[r] = e * (dp[r] - de[i]);
          }
        }
      }
      // rows past the end and rows without a key count nothing, whatever k and v
      // hold (a zero of theirs times an infinity would be NaN)
      if (__any(t_ref[32 * t + l31] == INFINITY)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t_ref[32 * t + tile_row(r, 0) + 4 * hi] == INFINITY) p[r] = s[r] = 0.0f;
      }
      {
        const Columns<T> pc(p);
        mma_turned<T, DP, BR>(tg, 32 * t, part * NDT, pc, lane, av);
      }
      const Columns<T> ds(s);
      mma_turned<T, DP, BR>(tq, 32 * t, part * NDT, ds, lane, ak);
    }
  }
  if (!there) return;
  if (!present)
#pragma unroll
    for (int i = 0; i < NDT; ++i) ak[i] = zero16(), av[i] = zero16();
  if (a.splits > 1) {
    const int64_t all = a.Tk * a.Hk, row = (ks + j) * a.Hk + w.hk;
    store_columns<float>(part_row(a.part, w.split, all, row, a.d), ak, a.scale, part * DO, a.d, hi, a.d % 4 == 0);
    store_columns<float>(part_row(a.part + a.splits * all * a.d, w.split, all, row, a.d), av, DROP ? a.keep : 1.0f,
                         part * DO, a.d, hi, a.d % 4 == 0);
    return;
  }
  if (a.dk.p)
    store_columns<T>(static_cast<T*>(const_cast<void*>(a.dk.p)) + (ks + j) * a.dk.row + w.hk * a.dk.head, ak, a.scale,
                     part * DO, a.d, hi, a.vec);
  if (a.dv.p)
    store_columns<T>(static_cast<T*>(const_cast<void*>(a.dv.p)) + (ks + j) * a.dv.row + w.hk * a.dv.head, av,
                     DROP ? a.keep : 1.0f, part * DO, a.d, hi, a.vec);
}

template <typename T, int DP, bool DROP, int BIAS>
void launch_tiles(const AttnArgs& a, hipStream_t s) {
  constexpr int DO = DP > 128 ? DP / 2 : DP, RT = DP * int(sizeof(T)) <= 128 ? 2 : 1;
  const int64_t BK = rows_a_tile(a.max_k), tiles = (a.max_k + BK - 1) / BK, n = tiles * (DP / DO) * a.splits * a.Hk * a.B;
  const size_t lds = BIAS ? ((BIAS == kBias ? 3 * 32 * RT : 0) + size_t(a.G) * bias_stride(a.buckets)) * 4 : 0;
  if constexpr (BIAS == kBiasBytes)  // made for long segments only
    k_attn_dkv<T, DP, DO, RT, DROP, BIAS, 4><<<uint32_t(n), 256, lds, s>>>(a, n, int(tiles));
  else if (BK == 64)
    k_attn_dkv<T, DP, DO, RT, DROP, BIAS, 2><<<uint32_t(n), 128, lds, s>>>(a, n, int(tiles));
  else
    k_attn_dkv<T, DP, DO, RT, DROP, BIAS, 4><<<uint32_t(n), 256, lds, s>>>(a, n, int(tiles));
}

template <typename T, int DP, int BIAS>
void launch_dkv_tiles(const AttnArgs& a, hipStream_t s) {
  if (a.threshold)
    launch_tiles<T, DP, true, BIAS>(a, s);
  else
    launch_tiles<T, DP, false, BIAS>(a, s);
}

template <int BIAS>
void launch_dkv_kernel(const AttnArgs& a, hipStream_t s) {
  switch (attn_padded(a.d)) {
    case 32: return a.bf16 ? launch_dkv_tiles<uint16_t, 32, BIAS>(a, s) : launch_dkv_tiles<float, 32, BIAS>(a, s);
    case 64: return a.bf16 ? launch_dkv_tiles<uint16_t, 64, BIAS>(a, s) : launch_dkv_tiles<float, 64, BIAS>(a, s);
    case 96: return a.bf16 ? launch_dkv_tiles<uint16_t, 96, BIAS>(a, s) : launch_dkv_tiles<float, 96, BIAS>(a, s);
    case 128: return a.bf16 ? launch_dkv_tiles<uint16_t, 128, BIAS>(a, s) : launch_dkv_tiles<float, 128, BIAS>(a, s);
    case 192: return a.bf16 ? launch_dkv_tiles<uint16_t, 192, BIAS>(a, s) : launch_dkv_tiles<float, 192, BIAS>(a, s);
    default: return a.bf16 ? launch_dkv_tiles<uint16_t, 256, BIAS>(a, s) : launch_dkv_tiles<float, 256, BIAS>(a, s);
  }
}

}  // namespace
}  // namespace gtp
