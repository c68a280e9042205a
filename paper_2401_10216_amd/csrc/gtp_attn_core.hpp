// What the attention kernels share: the matrix products on a wave's 32 x 32
// tile, the staging of row tiles in LDS, segments, and dropped probabilities.
//
// A wave takes 32 columns (query rows in the forward and in dq, keys in dk and
// dv) as the N index of every product, and walks the other axis in tiles of 32
// as the M index.  The 32 x 32 result of a product lies with column lane & 31
// in a lane, rows 8 (r / 4) + 4 (lane >> 5) + r % 4 in its registers r < 16: that
// is, up to the order of the summed index, the layout in which the next product
// takes its N-side operand.  So probabilities go from accumulator to operand
// without crossing lanes, a column's statistics live in one lane (and its
// partner, lane ^ 32), and the M-side operand follows the same order.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "gtp_attn.hpp"
#include "gtp_device.hpp"
#include "gtp_rng.hpp"

namespace gtp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Row r of a wave's 32 x 32 result in register r (0..15) of lane half hi.
__device__ __forceinline__ constexpr int tile_row(int r, int hi) { return 8 * (r >> 2) + 4 * hi + (r & 3); }

// 2^x by the hardware's exponential (1 unit in the last place; results below 2^-126 are zero).
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}

// max(v, v of lane ^ 32) and their sum.
__device__ __forceinline__ float half_max(float v) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// fp32 operands go to the matrix unit in three bf16 parts, v = v1 + v2 + v3 (24
// bits: exact down to 2^-110), a product as the six partial products of 2^-16 of it and
// up: what is left out is below 2^-24 of a product, an fp32 rounding, and no value's
// range matters, since bf16 has fp32's exponents.  Six 16-bit products of depth 16 take
// 192 cycles, the fp32 instructions for that depth 512.  bf16 operands are one part.
template <typename T>
constexpr int parts() {
  return sizeof(T) == 4 ? 3 : 1;
}
template <typename T>
struct Operand {
  u32x4 p[parts<T>()];  // eight values of the summed axis, each part
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // to nearest, ties to even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// Two values in three parts.  GUARD: a value is cut to the largest bf16 value before its
// first rounding, what that leaves is in the other parts.  An infinity is its third part,
// which meets no part of the other operand but the first: infinity times that is what the
// product is, where infinity times a second part of zero would be NaN.  Its own first part
// is a number of its sign near 1, so that the other operand's third part may be one too.
// NaN stays in the second and third.
template <bool GUARD>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&o)[3]) {
  constexpr float kMost = 0x1.fep127f;  // 0x7f7f
  if constexpr (GUARD)
    o[0] = pack_bf16(__builtin_amdgcn_fmed3f(a, -kMost, kMost), __builtin_amdgcn_fmed3f(b, -kMost, kMost));
  else
    o[0] = pack_bf16(a, b);
  const float ra = a - __uint_as_float(o[0] << 16), rb = b - __uint_as_float(o[0] & 0xffff0000u);
  if constexpr (GUARD) {
    const bool ia = fabsf(a) == INFINITY, ib = fabsf(b) == INFINITY;
    o[0] ^= (ia ? 0x4000u : 0u) | (ib ? 0x40000000u : 0u);  // 0x7f7f to 0x3f7f
    o[1] = pack_bf16(ia ? 0.0f : ra, ib ? 0.0f : rb);
  } else {
    o[1] = pack_bf16(ra, rb);
  }
  o[2] = pack_bf16(ra - __uint_as_float(o[1] << 16), rb - __uint_as_float(o[1] & 0xffff0000u));
}
__device__ __forceinline__ f32x16 mfma16(const u32x4& a, const u32x4& b, const f32x16& acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0,
                                                 0, 0);
}

// acc += A B over 16 values of the summed axis, of which the lane holds its half's
// eight: A's of row lane & 31, B's of column lane & 31.
template <typename T>
__device__ __forceinline__ void mma(const Operand<T>& a, const Operand<T>& b, f32x16& acc) {
  if constexpr (sizeof(T) == 4) {
    acc = mfma16(a.p[0], b.p[2], acc);  // the small ones first
    acc = mfma16(a.p[2], b.p[0], acc);
    acc = mfma16(a.p[1], b.p[1], acc);
    acc = mfma16(a.p[0], b.p[1], acc);
    acc = mfma16(a.p[1], b.p[0], acc);
  }
  acc = mfma16(a.p[0], b.p[0], acc);
}

// Two products at once, instruction by instruction: one's partial product runs while the
// other's waits for the sum before it.
template <typename T>
__device__ __forceinline__ void mma2(const Operand<T>& a, const Operand<T>& b, f32x16& acc, const Operand<T>& c,
                                     const Operand<T>& d, f32x16& acc2) {
  auto both = [&](int i, int j) {
    acc = mfma16(a.p[i], b.p[j], acc);
    acc2 = mfma16(c.p[i], d.p[j], acc2);
  };
  if constexpr (sizeof(T) == 4) {
    both(0, 2);
    both(2, 0);
    both(1, 1);
    both(0, 1);
    both(1, 0);
  }
  both(0, 0);
}

// A tile of rows in LDS: a plane for each part, rows of DP bf16 values, 16 bytes of
// padding behind each (the lanes of an operand's read take the same columns of 32 rows:
// an odd stride in units of 16 bytes spreads them over the banks).
template <int DP>
constexpr int row_bytes() {
  return DP * 2 + 16;
}
template <typename T, int DP, int ROWS>
constexpr int tile_bytes() {
  return parts<T>() * ROWS * row_bytes<DP>();
}

// The operand of columns 16 c .. 16 c + 15 of row `row` of a tile of ROWS rows.
template <typename T, int DP, int ROWS>
__device__ __forceinline__ Operand<T> tile_operand(const char* tile, int row, int c, int hi) {
  Operand<T> o;
#pragma unroll
  for (int p = 0; p < parts<T>(); ++p)
    o.p[p] = *reinterpret_cast<const u32x4*>(tile + (p * ROWS + row) * row_bytes<DP>() + 32 * c + 16 * hi);
  return o;
}

// A result as the N-side operand of the next product, summed over its 32 rows: 16
// values a lane, in bf16 one rounding of 2^-8 at most of each probability or score
// gradient (as the inputs' own), in fp32 none.
template <typename T>
struct Columns {
  Operand<T> s[2];
  __device__ __forceinline__ explicit Columns(const f32x16& v) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = v[8 * i + 2 * j], y = v[8 * i + 2 * j + 1];
        if constexpr (sizeof(T) == 4) {
          uint32_t o[3];
          split_pair<false>(x, y, o);
#pragma unroll
          for (int p = 0; p < 3; ++p) s[i].p[p][j] = o[p];
        } else {
          s[i].p[0][j] = pack_bf16(x, y);
        }
      }
  }
};

// The M-side operand of columns 32 dt .. 32 dt + 31 of rows r0 + 16 s .. r0 + 16 s + 15 of
// a tile, turned over, in the order in which a result holds its rows.
template <typename T, int DP, int ROWS>
__device__ __forceinline__ Operand<T> turned_operand(const char* tile, int r0, int dt, int s, int lane) {
  constexpr int S = row_bytes<DP>();
  // 16 lanes read a block of 4 rows x 16 columns, 8 bytes each, and each receives
  // the 4 rows of its own column
  const char* base = tile + (r0 + 16 * s + 4 * (lane >> 5) + ((lane & 15) >> 2)) * S +
                     (32 * dt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  typedef __attribute__((address_space(3))) s16x4* lds4;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  Operand<T> a;
#pragma unroll
  for (int p = 0; p < parts<T>(); ++p) {
    const char* at = base + p * ROWS * S;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at)));
    const u32x2 up = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * S)));
    a.p[p] = u32x4{lo[0], lo[1], up[0], up[1]};
  }
  return a;
}

// acc[i][d, column] += sum over rows r0 .. r0 + 31 of a tile of tile[row][32 (dt + i) + d] v[row, column].
template <typename T, int DP, int ROWS, int N>
__device__ __forceinline__ void mma_turned(const char* tile, int r0, int dt, const Columns<T>& v, int lane,
                                           f32x16 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 2)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Operand<T> a = turned_operand<T, DP, ROWS>(tile, r0, dt + i, s, lane);
      if (i + 1 < N)
        mma2<T>(a, v.s[s], acc[i], turned_operand<T, DP, ROWS>(tile, r0, dt + (i + 1 < N ? i + 1 : i), s, lane), v.s[s],
                acc[i + 1 < N ? i + 1 : i]);
      else
        mma<T>(a, v.s[s], acc[i]);
    }
}

// 16 bytes of a row of d elements, column `col` in units of 16 bytes: get() issues
// the load, always (a load under a condition would make every one wait for the one
// before it): of the row's last 16 bytes where the column passes the row's end; fix()
// moves what came into place and puts zeros past the end, and everywhere unless `ok`.
// vec: the row's columns are whole and its memory 16-byte aligned (else the load is
// of element-aligned memory).
template <typename T>
struct Load16 {
  static constexpr int E = 16 / int(sizeof(T));
  __device__ __forceinline__ static u32x4 get(const T* row, int col, int d, bool vec) {
    const int at = col * E;
    u32x4 v;
    if (vec) {
      v = *reinterpret_cast<const u32x4*>(row + (at < d ? at : 0));
    } else if (d >= E) {
      __builtin_memcpy(&v, row + (at < d - E ? at : d - E), 16);
    } else {  // shorter rows than one load
      v = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const T e = row[i < d ? i : 0];
        if constexpr (sizeof(T) == 4)
          v[i] = i < d ? __builtin_bit_cast(uint32_t, e) : 0u;
        else
          v[i >> 1] |= (i < d ? uint32_t(e) : 0u) << (16 * (i & 1));
      }
    }
    return v;
  }
  __device__ __forceinline__ static u32x4 fix(u32x4 v, int col, int d, bool vec, bool ok) {
    const int past = col * E + E - d;  // elements of this column behind the row's end
    if (!vec && d >= E && past > 0 && past < E) {
      const int bits = past * int(sizeof(T)) * 8;  // the load began as much too early
      uint64_t lo = uint64_t(v[1]) << 32 | v[0], up = uint64_t(v[3]) << 32 | v[2];
      if (bits >= 64) {
        lo = bits == 64 ? up : up >> (bits - 64);
        up = 0;
      } else {
        lo = lo >> bits | up << (64 - bits);
        up >>= bits;
      }
      v = u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(up), uint32_t(up >> 32)};
    }
    const bool in = ok && past < E;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = in ? v[i] : 0u;
    return v;
  }
};

// A lane's row as N-side operands, DP / 16 of them.  RAW: fp32 values kept as they
// are and split at each use, where the parts of them all would not fit the registers.
template <typename T, int DP, bool RAW>
struct RowOperands {
  static constexpr int NC = DP / 16;
  Operand<T> o[RAW ? 1 : NC];
  u32x4 raw[RAW ? NC : 1][2];
  __device__ __forceinline__ static Operand<T> split(const u32x4& a, const u32x4& b) {
    Operand<T> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4& v = j < 2 ? a : b;
      uint32_t q[3];
      split_pair<true>(__uint_as_float(v[2 * (j & 1)]), __uint_as_float(v[2 * (j & 1) + 1]), q);
#pragma unroll
      for (int p = 0; p < parts<T>(); ++p) r.p[p][j] = q[p];
    }
    return r;
  }
  // row: a valid row also where !ok (then zeros stand for it)
  __device__ __forceinline__ void load(const T* row, bool ok, int hi, int d, bool vec) {
    constexpr int W = sizeof(T) == 4 ? 2 : 1;
    u32x4 v[NC][W];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int k = 0; k < W; ++k) v[c][k] = Load16<T>::get(row, W * (2 * c + hi) + k, d, vec);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int k = 0; k < W; ++k) v[c][k] = Load16<T>::fix(v[c][k], W * (2 * c + hi) + k, d, vec, ok);
      if constexpr (sizeof(T) == 2)
        o[c].p[0] = v[c][0];
      else if constexpr (RAW)
        raw[c][0] = v[c][0], raw[c][1] = v[c][1];
      else
        o[c] = split(v[c][0], v[c][1]);
    }
  }
  __device__ __forceinline__ void negate() {
    if constexpr (RAW) {
#pragma unroll
      for (int c = 0; c < NC; ++c) raw[c][0] ^= 0x80000000u, raw[c][1] ^= 0x80000000u;
    } else {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int p = 0; p < parts<T>(); ++p) o[c].p[p] ^= 0x80008000u;
    }
  }
  // AGAIN: split at each use; else the compiler makes the parts once and keeps them in
  // scratch memory (dk, dv of heads of 217: 1565 us so and 1200 split again; dq of them 795 and 868).
  template <bool AGAIN = false>
  __device__ __forceinline__ Operand<T> operator()(int c) const {
    if constexpr (RAW) {
      u32x4 a = raw[c][0], b = raw[c][1];
      if constexpr (AGAIN) asm volatile("" : "+v"(a), "+v"(b));
      return split(a, b);
    } else {
      return o[c];
    }
  }
};

// ROWS rows from memory to an LDS tile by NT threads: fetch() issues the loads,
// commit() writes what came.  row(r, &ok): pointer to tile row r, a valid one also where
// there is none (ok = false: zeros stand for it).
template <typename T, int DP, int ROWS, int NT>
struct Stage {
  static constexpr int CPR = DP * int(sizeof(T)) / 16;
  static constexpr int ITER = (ROWS * CPR + NT - 1) / NT;
  static_assert(ROWS <= 64, "a bit for each row");
  u32x4 reg[ITER];
  template <typename F>
  __device__ __forceinline__ void fetch(F row, int d, bool vec) {
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      const int id = int(threadIdx.x) + i * NT;
      const T* p = row(ROWS * CPR % NT != 0 && id >= ROWS * CPR ? 0 : id / CPR);
      reg[i] = Load16<T>::get(p, id % CPR, d, vec);
    }
  }
  // rows: a bit for each row of the tile, zeros where it is not there; whole: all are
  __device__ __forceinline__ void commit(char* tile, int d, bool vec, bool whole, uint64_t rows) const {
    if (vec && whole && d == DP)
      write<true>(tile, d, vec, rows);
    else
      write<false>(tile, d, vec, rows);
  }
  template <bool PLAIN>
  __device__ __forceinline__ void write(char* tile, int d, bool vec, uint64_t rows) const {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      const int id = int(threadIdx.x) + i * NT;
      if (ROWS * CPR % NT != 0 && id >= ROWS * CPR) break;
      char* const at = tile + (id / CPR) * row_bytes<DP>();
      const u32x4 v = PLAIN ? reg[i] : Load16<T>::fix(reg[i], id % CPR, d, vec, (rows >> (id / CPR)) & 1u);
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x4*>(at + 16 * (id % CPR)) = v;
      } else {
        uint32_t a[3], b[3];
        split_pair<true>(__uint_as_float(v[0]), __uint_as_float(v[1]), a);
        split_pair<true>(__uint_as_float(v[2]), __uint_as_float(v[3]), b);
#pragma unroll
        for (int p = 0; p < 3; ++p)
          *reinterpret_cast<u32x2*>(at + p * ROWS * row_bytes<DP>() + 8 * (id % CPR)) = u32x2{a[p], b[p]};
      }
    }
  }
};

// Rows [start, start + n) of segment b among `total`, at most `most`; offsets
// outside the tensor are cut to it, so that no access leaves it.
__device__ __forceinline__ void segment(const int64_t* off, int64_t b, int64_t most, int64_t total, int64_t& start,
                                        int64_t& n) {
  int64_t s = off ? off[b] : b * most, e = off ? off[b + 1] : s + most;
  s = s < 0 ? 0 : (s > total ? total : s);
  e = e < s ? s : (e > total ? total : e);
  start = s;
  n = e - s < most ? e - s : most;
}

// Which keys of a tile are there: a lane loads the mask's byte of key lane % ROWS, ahead
// with the tile and whether or not there is a mask (a load under a condition is waited
// for on the spot; one for each staged piece of a row was most of a short call's time).
template <int ROWS>
struct Present {
  uint32_t byte = 0;
  // j0 < n; base: any memory of ours to read where there is no mask
  __device__ __forceinline__ void fetch(const uint8_t* mask, const void* base, int64_t j0, int64_t n, int lane) {
    const int64_t j = j0 + (lane & (ROWS - 1));
    byte = *(mask ? mask + (j < n ? j : j0) : static_cast<const uint8_t*>(base));
  }
  __device__ __forceinline__ uint64_t rows(const uint8_t* mask, int64_t j0, int64_t n, int lane) const {
    return __ballot(j0 + (lane & (ROWS - 1)) < n && (!mask || byte != 0));
  }
};

// Row R = i G + g of a key head's rows: i, and g in *g.  (64-bit divisions in the tile
// loop took longer than its products; R < 2^31 by the launch's limits.)
struct Group {
  uint32_t G, inv;
  __device__ __forceinline__ explicit Group(int g) : G(uint32_t(g)), inv(g > 1 ? 0xffffffffu / uint32_t(g) : 0) {}
  __device__ __forceinline__ int64_t row(int64_t R, int* g) const {
    if (G == 1) {
      *g = 0;
      return R;
    }
    uint32_t q = __umulhi(uint32_t(R), inv);  // at most two too few
    uint32_t r = uint32_t(R) - q * G;
    if (r >= G) ++q, r -= G;
    if (r >= G) ++q, r -= G;
    *g = int(r);
    return int64_t(q);
  }
};

// Element type of the tensors in memory.
template <typename T>
__device__ __forceinline__ float to_f32(T v) {
  if constexpr (sizeof(T) == 4)
    return v;
  else
    return __uint_as_float(uint32_t(v) << 16);
}

// d elements of one row from the results acc[dt] (column lane & 31 = the row,
// results' rows = the elements), times f.
template <typename T, int NDT>
__device__ __forceinline__ void store_columns(T* row, const f32x16 (&acc)[NDT], float f, int d0, int d, int hi,
                                              bool vec) {
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = d0 + 32 * dt + 8 * g + 4 * hi;
      if (e >= d) continue;
      if constexpr (sizeof(T) == 4) {
        const f32x4 o = {acc[dt][4 * g] * f, acc[dt][4 * g + 1] * f, acc[dt][4 * g + 2] * f, acc[dt][4 * g + 3] * f};
        if (vec)
          *reinterpret_cast<f32x4*>(row + e) = o;
        else
          for (int i = 0; i < 4; ++i)
            if (e + i < d) row[e + i] = o[i];
      } else {
        bf16x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = static_cast<__bf16>(acc[dt][4 * g + i] * f);
        if (vec)
          *reinterpret_cast<bf16x4*>(row + e) = o;
        else
          for (int i = 0; i < 4; ++i) {
            const __bf16 one = o[i];
            if (e + i < d) row[e + i] = __builtin_bit_cast(uint16_t, one);
          }
      }
    }
}

// Dropped probabilities.  The rows of a key head's G query heads count together
// (row R = i G + g of the segment), in blocks of 4 rows x 4 keys: block
// ((b Hk + hk) ceil(max_q G / 4) + R / 4) ceil(max_k / 4) + j / 4 takes calls 2 block
// (rows 0, 1) and 2 block + 1 (rows 2, 3) of the generator, element (R, j) halfword
// 4 (R % 2) + j % 4.
struct Drop {
  uint64_t seed, offset, base, nc;
  uint32_t threshold;
  __device__ __forceinline__ void init(const AttnArgs& a, int64_t b, int hk) {
    seed = a.rng[0];
    offset = a.rng[1];
    threshold = a.threshold;
    nc = uint64_t(a.max_k + 3) >> 2;
    const uint64_t nr = uint64_t(a.max_q * a.G + 3) >> 2;
    base = (uint64_t(b) * a.Hk + hk) * nr * nc;
  }
  // The draws of a 32 x 32 tile whose first row is R0 and first key j0, in the two
  // layouts of a result.  A lane's run of four elements (register group g) is one row
  // or column of a block; the four lanes of a quad need the same four blocks, so lane
  // q makes the two calls of block g = q alone and they trade: 16 draws a lane cost two
  // calls, not eight.
  //
  // Bit r: whether element (row R0 + lane & 31, key j0 + tile_row(r, hi)) is kept.
  __device__ __forceinline__ uint32_t keys_of_row(int64_t R0, int64_t j0, int lane) const {
    const int q = lane & 3;
    const uint64_t block =
        base + uint64_t((R0 + (lane & 28)) >> 2) * nc + uint64_t((j0 + 8 * q + 4 * (lane >> 5)) >> 2);
    uint32_t bits = 0;  // of block q: nibble r = row r's four keys
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4];
      philox(2 * block + h, seed, offset, w);
      bits |= kept8(w) << (8 * h);
    }
    return trade(bits, q);
  }
  // Bit r: whether element (row R0 + tile_row(r, hi), key j0 + lane & 31) is kept.
  __device__ __forceinline__ uint32_t rows_of_key(int64_t R0, int64_t j0, int lane) const {
    const int q = lane & 3;
    const uint64_t block =
        base + uint64_t((R0 + 8 * q + 4 * (lane >> 5)) >> 2) * nc + uint64_t((j0 + (lane & 28)) >> 2);
    uint32_t bits = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4];
      philox(2 * block + h, seed, offset, w);
      bits |= kept8(w) << (8 * h);
    }
    // the 4 x 4 bits turned over: nibble j = key j's four rows
    uint32_t t = (bits ^ (bits >> 3)) & 0x0a0au;
    bits ^= t ^ (t << 3);
    t = (bits ^ (bits >> 6)) & 0x00ccu;
    bits ^= t ^ (t << 6);
    return trade(bits, q);
  }
  // Bit h: whether draw h of a call keeps.
  __device__ __forceinline__ uint32_t kept8(const uint32_t (&w)[4]) const {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const uint16_t below = uint16_t(threshold - 1);  // threshold > 0 where anything is dropped
    uint32_t b = 0;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      // both halves at once: draw - (threshold - 1), at least 0 and at most 1
      const u16x2 over = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, w[h]), u16x2{below, below});
      const uint32_t one = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(over, u16x2{1, 1}));
      b |= ((one | one >> 15) & 3u) << (2 * h);
    }
    return b;
  }
  // v where bit r of keep is set, else 0.
  __device__ __forceinline__ static float kept(float v, uint32_t keep, int r) {
    return __uint_as_float(__float_as_uint(v) & uint32_t(__builtin_amdgcn_sbfe(int(keep), r, 1)));
  }
  // Lane q of a quad holds block q's nibbles; it gets nibble q of each block g, at bits 4 g.
  __device__ __forceinline__ static uint32_t trade(uint32_t bits, int q) {
    uint32_t out = 0;
    auto take = [&](auto ctrl, int g) {
      const uint32_t b = uint32_t(
          __builtin_amdgcn_update_dpp(0, int(bits), decltype(ctrl)::value, 0xf, 0xf, true));
      out |= ((b >> (4 * q)) & 0xfu) << (4 * g);
    };
    take(std::integral_constant<int, 0x00>{}, 0);  // quad_perm 0 0 0 0
    take(std::integral_constant<int, 0x55>{}, 1);  // 1 1 1 1
    take(std::integral_constant<int, 0xaa>{}, 2);
    take(std::integral_constant<int, 0xff>{}, 3);
    return out;
  }
};

// The learned bias of a score, by the distance of its two positions: bucket
//   0 where d2 < r0^2,  1 + (number(d2) - number(r0^2)) >> shift,  at most buckets - 1,
// number(x) the place of a positive fp32 number among them all, its bits: 2^(23 - shift)
// buckets for each doubling of d2, evenly spaced between powers of two.  d2 = dx^2 + dy^2 + dz^2
// with one rounding for each difference, for dx^2 and for each sum, so that every pass, and
// whoever computes it elsewhere, finds the same bucket.  NaN is above every number, whatever its sign bit.
// Three instructions from d2 to the bucket; an exact logarithm, or a search among edges in
// LDS, would be several times that beside the 10-20 that a score takes in all.
struct Buckets {
  uint32_t near, far, shift;  // numbers of the first bucket's and the last's first d2 (near: a step below r0^2)
  __device__ __forceinline__ explicit Buckets(const AttnArgs& a) : near(a.near), far(a.far), shift(a.step) {}
  __device__ __forceinline__ uint32_t operator()(float dx, float dy, float dz) const {
    const float d2 = fmaf(dz, dz, fmaf(dy, dy, __fmul_rn(dx, dx)));
    uint32_t v;  // the middle one of three: the compiler takes two instructions
    asm("v_med3_u32 %0, %1, %2, %3" : "=v"(v) : "v"(d2), "v"(near), "v"(far));
    return (v - near) >> shift;
  }
};

// What the kernels take of a bias.
constexpr int kNoBias = 0, kBias = 1, kBiasBytes = 2;

// The buckets made ahead: for each segment, block of 32 columns (a wave's: rows or keys, `at` in the segment) and tile of
// 32 of the other side, a lane's 16 buckets in the order of a result's registers, four times the bucket each: 16 bytes a lane,
// 1 KB a wave and tile.  blocks, tiles: of a segment.
__device__ __forceinline__ const u32x4* bucket_bytes(const uint8_t* bytes, int64_t b, int64_t blocks, int64_t tiles,
                                                     int64_t at, int hi) {
  return reinterpret_cast<const u32x4*>(bytes) + ((b * blocks + (at >> 5)) * tiles) * 64 + (at & 31) + 32 * hi;
}
// The byte of register r.
__device__ __forceinline__ uint32_t bucket_byte(const u32x4& v, int r) { return (v[r >> 2] >> (8 * (r & 3))) & 0xffu; }
// The word that lies `byte` bytes behind p.
__device__ __forceinline__ float word_at(const float* p, uint32_t byte) {
  return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p) + byte);
}

// The bias of key head hk's query heads in LDS, in units of log 2: [G][bias_stride].
__device__ __forceinline__ void load_bias(const AttnArgs& a, int hk, float* table) {
  const int n = a.G * a.buckets, stride = bias_stride(a.buckets);
  const float* const from = a.bias + int64_t(hk) * n;
  for (int i = threadIdx.x; i < n; i += int(blockDim.x)) table[i / a.buckets * stride + i % a.buckets] = from[i] * kLog2e;
}

// Positions of a tile's rows, one after the other x, y, z [ROWS] each in LDS: a lane fetches row lane % ROWS's.
template <int ROWS>
struct StagedPos {
  float x, y, z;
  __device__ __forceinline__ void fetch(const float* pos, int64_t row) {
    x = pos[3 * row];
    y = pos[3 * row + 1];
    z = pos[3 * row + 2];
  }
  __device__ __forceinline__ void commit(float* tile) const {
    if (threadIdx.x < ROWS) {
      tile[threadIdx.x] = x;
      tile[ROWS + threadIdx.x] = y;
      tile[2 * ROWS + threadIdx.x] = z;
    }
  }
};

// Waves a SIMD that a kernel's registers are cut for: two hide each other's
// waits (one issues vector instructions while the matrix unit works for the
// other), where rows, accumulators and a prefetched tile of a four-wave workgroup fit
// 256 registers.  (Two-wave workgroups stage twice as much a lane: fp32 heads of 33-64
// keep 24 bytes a lane in scratch memory there, 116 with draws.)
template <typename T, int DP>
constexpr int waves_per_simd() {
  return DP * int(sizeof(T)) <= 256 ? 2 : 1;
}
// fp32 rows longer than that stay unsplit, and the next tile is not fetched ahead.
template <typename T, int DP>
constexpr bool long_rows() {
  return sizeof(T) == 4 && DP > 128;
}

// Parts of a split call: part s of element (row, i), rows counted over all heads.
__device__ __forceinline__ float* part_row(float* part, int split, int64_t rows, int64_t row, int d) {
  return part + (int64_t(split) * rows + row) * d;
}

// Work of a workgroup: tiles fastest, then splits, key heads, segments; XCD-aware,
// so that the workgroups that read one segment's rows share an L2.
struct Work {
  int tile, split, hk;
  int64_t b;
  __device__ __forceinline__ Work(int64_t w, int64_t n, int tiles, int splits, int Hk) {
    int64_t id = xcd_product(w, n);
    tile = int(id % tiles);
    id /= tiles;
    split = int(id % splits);
    id /= splits;
    hk = int(id % Hk);
    b = id / Hk;
  }
};

}  // namespace gtp
