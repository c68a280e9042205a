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
  int64_t B, Tq, Tk, max_q, max_k;
  int H, Hk, G, d;               // query heads, key heads, H / Hk, head length
  int splits;                    // parts that a row's keys (or a key's rows) are dealt to
  float scale, scale2;           // of the scores; times log2(e)
  uint32_t threshold;            // 0: nothing is dropped
  float keep;                    // factor of what is kept
  bool bf16, vec;                // vec: every row of every tensor starts 16-byte aligned, d a multiple of 16 bytes
};

// Rows (keys in dk, dv) that a workgroup takes, a wave 32: 128, or 64 where no segment has
// more, so that short ones do not leave half the waves idle.
inline int rows_a_tile(int64_t most) { return most <= 64 ? 64 : 128; }
int attn_padded(int d);  // the head length that the kernels are instantiated at, >= d
// Parts that the keys of each row (the rows of each key) are dealt to: 1 where the
// workgroups fill the chip without.
int attn_row_splits(const AttnArgs& a, bool backward);  // its parts: of the forward, of dq
int attn_key_splits(const AttnArgs& a);
hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_delta(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_dq(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_dkv(const AttnArgs& a, hipStream_t s);
// Sums the parts of dq (keys = false), dk or dv (keys = true) into out.
hipError_t launch_attn_sum(const AttnArgs& a, const float* part, int splits, bool keys, const AttnRows& out,
                           hipStream_t s);

}  // namespace gtp
