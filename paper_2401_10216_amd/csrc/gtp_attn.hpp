// Softmax attention over packed segments and its gradient: what the C entries
// (gtp_layers.hip) hand to the kernels (gtp_attn_fwd.hip, gtp_attn_dq.hip,
// gtp_attn_dkv.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace gtp {

// Rows of a tensor [rows, heads, d]: element (t, h, i) at p[t row + h head + i].
struct AttnRows {
  const void* p;
  int64_t row, head;
};

struct AttnArgs {
  AttnRows q, k, v, o, dout;  // inputs (o and dout in the backward)
  AttnRows out;               // o of the forward, dq of the backward (p = null: not asked for)
  AttnRows dk, dv;            // null: not asked for
  const int64_t *q_off, *k_off;  // [B + 1] or null: equal segments of max_q, max_k rows
  const uint8_t* mask;           // [Tk] or null
  float* lse;                    // [Tq, H]: written by the forward, read by the backward
  float* delta;                  // [Tq, H]: rows' sums of dout o
  float* part;                   // results of the parts of a split call, [splits, rows, d] (forward: then [splits, rows]
                                 // of lse; dk, dv: one behind the other)
  const uint64_t* rng;           // {seed, offset}, with threshold > 0
  const float *bias, *q_pos, *k_pos;  // [H, buckets] added to the scores by distance; positions [Tq, 3], [Tk, 3]; or null
  float* dbias;                  // [H, buckets]: gradient asked for, or null
  float* bias_part;              // bias_part_floats, for dbias
  int64_t B, Tq, Tk, max_q, max_k;
  int H, Hk, G, d;               // query heads, key heads, H / Hk, head length
  int buckets;                   // of the bias
  uint32_t near, far, step;      // bucket of a squared distance: see Buckets
  uint8_t *bytes, *bytes_k;      // the pairs' buckets made ahead (see bias_bytes), for rows and for keys; null: made at each score
  int splits;                    // parts that a row's keys (or a key's rows) are dealt to
  float scale, scale2;           // of the scores; times log2(e)
  uint32_t threshold;            // 0: nothing is dropped
  float keep;                    // factor of what is kept
  bool bf16, vec;                // vec: every row of every tensor starts 16-byte aligned, d a multiple of 16 bytes
};

// Rows (keys in dk, dv) that a workgroup takes, a wave 32: 128, or 64 where no segment has
// more, so that short ones do not leave half the waves idle.
inline int rows_a_tile(int64_t most) { return most <= 64 ? 64 : 128; }
// Tiles of 32 of a segment's longest side in the buckets made ahead: an even number, since kernels take two at a time.
__host__ __device__ inline int64_t bytes_tiles(int64_t most) { return (most + 63) / 64 * 2; }
constexpr int kMaxBias = 4096, kMaxBiasHeads = 256;  // of the bias of a key head's query heads, in LDS
// From one head's to the next: odd, so that heads that share a distance (lanes side by side) read different banks.
__host__ __device__ inline int bias_stride(int buckets) { return buckets | 1; }
// Of dq.  A bias's sums beside the longest fp32 tiles fit the LDS of 64 rows only; where two workgroups of 128 rows do not
// fit a CU's and one of 256 does, that keeps two waves on a SIMD (two of 3500-4300 rows, 8 heads of 128, 64 buckets, bf16:
// 540 us, of 128 rows 770).
int dq_rows_a_tile(const AttnArgs& a);
int attn_padded(int d);  // the head length that the kernels are instantiated at, >= d
// Parts that the keys of each row (the rows of each key) are dealt to: 1 where the
// workgroups fill the chip without.
int attn_row_splits(const AttnArgs& a, bool backward);  // its parts: of the forward, of dq
int attn_key_splits(const AttnArgs& a);
hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t s);
// With a bias (instantiations of their own, gtp_attn_bias_*.hip).
void launch_attn_fwd_bias(const AttnArgs& a, hipStream_t s);
void launch_attn_dq_bias(const AttnArgs& a, hipStream_t s);
void launch_attn_dkv_bias(const AttnArgs& a, hipStream_t s);
// With the buckets made ahead (gtp_attn_bytes_*.hip).
void launch_attn_fwd_bytes(const AttnArgs& a, hipStream_t s);
void launch_attn_dq_bytes(const AttnArgs& a, hipStream_t s);
void launch_attn_dkv_bytes(const AttnArgs& a, hipStream_t s);
// Bytes of the buckets of all pairs of a segment's rows and keys, one for each, if they are worth making ahead for every
// head at once (0: not).
int64_t bias_bytes(const AttnArgs& a);
bool bias_bytes_for_keys(const AttnArgs& a);  // whether dk, dv take them too, turned
hipError_t launch_bias_bytes(const AttnArgs& a, bool keys, hipStream_t s);
// Workgroups of dq with a bias that work on one key head, floats for what each leaves of
// dbias and for their sums, and the sum of them all (a.splits: of dq).
int64_t attn_bias_parts(const AttnArgs& a);
int64_t bias_part_floats(const AttnArgs& a);
hipError_t launch_attn_bias_sum(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_delta(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_dq(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_dkv(const AttnArgs& a, hipStream_t s);
// Sums the parts of dq (keys = false), dk or dv (keys = true) into out.
hipError_t launch_attn_sum(const AttnArgs& a, const float* part, int splits, bool keys, const AttnRows& out,
                           hipStream_t s);

}  // namespace gtp
