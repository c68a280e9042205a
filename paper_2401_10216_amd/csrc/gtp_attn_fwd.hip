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
#include <cmath>

#include "gtp_attn_core.hpp"

namespace gtp {
namespace {

constexpr float kSlack = 8.0f;  // probabilities stay below 2^8: far from overflow in fp32 and bf16, and as exact

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

// Workgroup: 32 NW rows of one key head (a wave 32), keys in tiles of 32 KT.  Heads longer
// than 128 leave the registers room for one wave a SIMD only.
template <typename T, int DP, int KT, bool DROP, int NW>
__global__ __launch_bounds__(64 * NW, DP <= 128 ? 2 : 1) void k_attn_fwd(const AttnArgs a, int64_t n_wg, int tiles) {
  constexpr int NT = 64 * NW, BM = 32 * NW, BN = 32 * KT, NC = DP / 16, NDT = DP / 32;
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
  // the scores' scale is taken positive, its sign into q: their maximum is then that of the products
  const float scale2 = fabsf(a.scale2);
  RowOperands<T, DP, long_rows<T, DP>()> qf;
  qf.load(static_cast<const T*>(a.q.p) + qi * a.q.row + h * a.q.head, there, hi, a.d, a.vec);
  if (a.scale2 < 0.0f) qf.negate();
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
    top = half_max(top) * scale2;
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
      for (int r = 0; r < 16; ++r) s[t][r] = pow2(fmaf(s[t][r], scale2, -ref));
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

// Tiles of 32 keys that the forward takes at a time.
constexpr int key_tiles(int DP, bool bf16) { return !bf16 && DP > 64 ? 1 : 2; }

template <typename T, int DP, bool DROP>
void launch_tiles(const AttnArgs& a, hipStream_t s) {
  constexpr int KT = key_tiles(DP, sizeof(T) == 2);
  const int64_t BM = rows_a_tile(a.max_q * a.G), tiles = (a.max_q * a.G + BM - 1) / BM, n = tiles * a.splits * a.Hk * a.B;
  if (BM == 64)
    k_attn_fwd<T, DP, KT, DROP, 2><<<uint32_t(n), 128, 0, s>>>(a, n, int(tiles));
  else
    k_attn_fwd<T, DP, KT, DROP, 4><<<uint32_t(n), 256, 0, s>>>(a, n, int(tiles));
}

template <typename T, int DP>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
  if (a.threshold)
    launch_tiles<T, DP, true>(a, s);
  else
    launch_tiles<T, DP, false>(a, s);
  if (a.splits > 1) {
    // four waves a row for many parts, whose loads one wave waits for eight at a time (32 rows
    // of 64: 64 parts by one wave 6.1 us, 125 by four 4.6); few parts of many rows want
    // fewer workgroups
    if (a.splits > 16)
      k_attn_join<T, 4><<<uint32_t(a.max_q * a.H * a.B), 256, 0, s>>>(a);
    else
      k_attn_join<T, 1><<<uint32_t((a.max_q * a.H + 3) / 4 * a.B), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

int attn_padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }

// Workgroups that a CU holds: by the waves a SIMD that the kernels' registers are cut for.
int attn_row_splits(const AttnArgs& a, bool backward) {
  const int BM = rows_a_tile(a.max_q * a.G), DP = attn_padded(a.d);
  const int waves = DP * (a.bf16 ? 2 : 4) <= 256 || (!backward && DP <= 128) ? 2 : 1;
  return parts_for((a.max_q * a.G + BM - 1) / BM * a.Hk * a.B, a.max_k, backward ? 32 : 32 * key_tiles(DP, a.bf16),
                   waves * 128 / BM, a.bf16);
}
int attn_key_splits(const AttnArgs& a) {
  const int BK = rows_a_tile(a.max_k), DP = attn_padded(a.d), bytes = DP * (a.bf16 ? 2 : 4);
  return parts_for((a.max_k + BK - 1) / BK * (DP > 128 ? 2 : 1) * a.Hk * a.B, a.max_q * a.G, bytes <= 128 ? 64 : 32,
                   (bytes <= (a.bf16 ? 256 : 128) ? 2 : 1) * 128 / BK, a.bf16);
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

hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t s) {
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
