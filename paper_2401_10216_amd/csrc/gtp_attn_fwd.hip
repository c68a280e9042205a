// Softmax attention, forward: o = softmax(scale q k^T) v over the keys of a
// row's segment, in one pass over the keys with the running maximum and sum of
// each row, and lse = log of the row's sum (the backward pass makes the
// probabilities again from it).
#include "gtp_attn_core.hpp"

namespace gtp {
namespace {

constexpr int NW = 4, NT = 64 * NW, BM = 32 * NW;

// Workgroup: 128 rows of one key head (4 waves x 32), keys in tiles of 32 KT.
template <typename T, int DP, int KT, bool DROP>
__global__ __launch_bounds__(NT) void k_attn_fwd(const AttnArgs a, int64_t n_wg, int tiles) {
  constexpr int BN = 32 * KT, NC = DP * int(sizeof(T)) / 32, NDT = DP / 32;
  __shared__ __align__(16) char tk[BN * tile_stride<T, DP>()];
  __shared__ __align__(16) char tv[BN * tile_stride<T, DP>()];
  lds_poison(reinterpret_cast<float*>(tk), int(sizeof(tk) / 4));
  lds_poison(reinterpret_cast<float*>(tv), int(sizeof(tv) / 4));
  const Work w(blockIdx.x, n_wg, tiles, a.splits, a.Hk);
  int64_t qs, nq, ks, nk;
  segment(a.q_off, w.b, a.max_q, a.Tq, qs, nq);
  segment(a.k_off, w.b, a.max_k, a.Tk, ks, nk);
  const int64_t rows = nq * a.G;
  if (int64_t(w.tile) * BM >= rows) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l31 = lane & 31, hi = lane >> 5;
  const int64_t R = int64_t(w.tile) * BM + wave * 32 + l31;
  const bool there = R < rows;
  const int64_t qi = there ? qs + R / a.G : 0;
  const int h = w.hk * a.G + (there ? int(R % a.G) : 0);
  u32x4 qf[NC];
  {
    const T* row = there ? static_cast<const T*>(a.q.p) + qi * a.q.row + h * a.q.head : nullptr;
#pragma unroll
    for (int c = 0; c < NC; ++c) qf[c] = load16<T>(row, 2 * c + hi, a.d, a.vec);
  }
  f32x16 acc[NDT];
#pragma unroll
  for (int i = 0; i < NDT; ++i) acc[i] = zero16();
  float m = -INFINITY, l = 0.0f;  // of the row's scores in units of log 2; this half's part of the sum
  Drop drop;
  if constexpr (DROP) drop.init(a, w.b, w.hk);

  const T* const kb = static_cast<const T*>(a.k.p) + ks * a.k.row + w.hk * a.k.head;
  const T* const vb = static_cast<const T*>(a.v.p) + ks * a.v.row + w.hk * a.v.head;
  const uint8_t* const mask = a.mask ? a.mask + ks : nullptr;
  const int64_t ntile = (nk + BN - 1) / BN, per = (ntile + a.splits - 1) / a.splits;
  const int64_t j_end = (w.split + 1) * per * BN < nk ? (w.split + 1) * per * BN : nk;
  Stage<T, DP, BN, NT> sk, sv;
  for (int64_t j0 = w.split * per * BN; j0 < j_end; j0 += BN) {
    // absent keys' rows are not read: zeros stand for them
    auto present = [&](int r) { return j0 + r < nk && (!mask || mask[j0 + r]); };
    sk.fetch([&](int r) { return present(r) ? kb + (j0 + r) * a.k.row : nullptr; }, a.d, a.vec);
    sv.fetch([&](int r) { return present(r) ? vb + (j0 + r) * a.v.row : nullptr; }, a.d, a.vec);
    __syncthreads();
    sk.commit(tk);
    sv.commit(tv);
    __syncthreads();
    f32x16 s[KT];
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      s[t] = zero16();
#pragma unroll
      for (int c = 0; c < NC; ++c) mma_chunk<T>(tile_chunk<T, DP>(tk, 32 * t + l31, c, hi), qf[c], s[t]);
      const uint32_t ok = uint32_t(__ballot(present(32 * t + l31))) >> (4 * hi);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[t][r] = (ok >> tile_row(r, 0)) & 1u ? s[t][r] * a.scale2 : -INFINITY;
        top = fmaxf(top, s[t][r]);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m_new = fmaxf(m, top);
    const float ref = m_new == -INFINITY ? 0.0f : m_new;  // no score yet: every exponential below is zero
    const float f = exp2f(m - ref);
    m = m_new;
    l *= f;
#pragma unroll
    for (int i = 0; i < NDT; ++i) acc[i] *= f;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      uint32_t keep = 0xffffu;
      if constexpr (DROP) keep = drop.keys_of_row(R, j0 + 32 * t, hi);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = exp2f(s[t][r] - ref);
        l += p;
        s[t][r] = DROP && !((keep >> r) & 1u) ? 0.0f : p;
      }
#pragma unroll
      for (int i = 0; i < NDT; ++i)
        mma_transposed<T, DP>(tv + 32 * t * tile_stride<T, DP>(), i, s[t], lane, acc[i]);
    }
  }
  l += __shfl_xor(l, 32);
  if (!there) return;
  const float inv = l == 0.0f ? 0.0f : (DROP ? a.keep / l : 1.0f / l);
  store_columns<T>(static_cast<T*>(const_cast<void*>(a.out.p)) + qi * a.out.row + h * a.out.head, acc, inv, 0, a.d, hi,
                   a.vec);
  if (hi == 0) a.lse[qi * a.H + h] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
}

template <typename T, int DP>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
  constexpr int KT = DP * int(sizeof(T)) > 512 ? 1 : 2;
  const int64_t tiles = (a.max_q * a.G + BM - 1) / BM, n = tiles * a.splits * a.Hk * a.B;
  if (a.threshold)
    k_attn_fwd<T, DP, KT, true><<<uint32_t(n), NT, 0, s>>>(a, n, int(tiles));
  else
    k_attn_fwd<T, DP, KT, false><<<uint32_t(n), NT, 0, s>>>(a, n, int(tiles));
  return hipGetLastError();
}

}  // namespace

int attn_padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }

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
