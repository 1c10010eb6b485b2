// Arguments of the kernels behind functional.py: rotary positions (rotary.hip),
// attention with a window and sinks (attention.hip), distillation (distill.hip).
// All pointers are device pointers; strides are in elements.  Entry points return
// 0, -1 (a size they do not take) or -5 (HIP error).
#pragma once
#include <stdint.h>

namespace compact {

// One tensor (b, l, heads, hd) of a rotary call; the last dimension is dense.
struct RotaryTensor {
  const void* src;
  void* dst;                     // may be src
  int64_t src_b, src_l, src_h;
  int64_t dst_b, dst_l, dst_h;
  int32_t heads;
  int32_t rotate;                // 0: copied
};

struct RotaryArgs {
  RotaryTensor t[3];
  const double* turns;           // [dims / 2] revolutions per position
  const void* positions;         // int64 or int32, or NULL: offset + index in the sequence
  int64_t pos_b, pos_l;          // its strides
  int64_t offset;
  int64_t tokens;                // b l
  int32_t l, hd, dims, count;    // count: tensors
  int32_t interleaved, inverse, pos32, f32;
  float magnitude;
};

struct AttnArgs {
  const uint16_t *q, *k, *v;     // (b, heads, lq, hd), (b, kv, lk, hd) twice
  uint16_t* o;
  float* lse;                    // [b heads][lq]: log2 of the sum of 2^(scale log2(e) q.k); +inf: no key
  int8_t* o_low;                 // [b heads][lq][hd]: what o's rounding took off, in 127ths of half its last place; or NULL
  const int32_t* lengths;        // [b] keys of each sequence, or NULL: lk
  int64_t qs[3], ks[3], vs[3], os[3];  // strides: sequence, head, row
  int32_t b, heads, kv, lq, lk, hd;
  int32_t window, sinks;         // key j of position p: j <= p and (p - j < window or j < sinks)
  float scale;
  int32_t splits;                // > 0: this many ranges of keys apart, then joined
  int32_t waves;                 // split form of few rows: a wave for 32 rows of the heads that share keys
  float* part_o;                 // with splits: [splits][b heads lq][hd]
  float* part_lse;               // [splits][b heads lq]
};

struct AttnGradArgs {
  AttnArgs f;                    // o and lse of the forward
  const uint16_t* go;            // gradient of o
  uint16_t *dq, *dk, *dv;        // dq of q's shape, dk and dv of k's
  float* delta;                  // [b heads][lq] scratch
  int64_t gs[3], dqs[3], dks[3], dvs[3];
  float* part;                   // [compact_attention_bwd_scratch()]
  int32_t parts, near_keys, chunks, far_keys, fine;  // set by the entry point
};

struct DistillArgs {
  const void* x;                 // [rows][V] bf16 or fp32 (f32)
  const void* top;               // [rows][K] bf16 or fp32 (top32), rows top_ld apart
  const void* ids;               // [rows][K] int64 or int32 (ids32), rows ids_ld apart; < 0: no entry
  const int64_t* target;         // [rows] or NULL
  float* count;                  // rows that count (target given)
  float* loss_row;               // [rows], or NULL: no loss
  float* loss;                   // their mean
  void* dx;                      // gradient of x, or NULL
  const float* dloss;            // NULL: 1
  float* entries;                // [rows][K + 1] pairs of scratch
  float* stats;                  // [rows] pairs of scratch
  int64_t rows, V, top_ld, ids_ld, ignore_index;
  int32_t K, f32, top32, ids32;
  int32_t unless_one;            // with dloss: nothing to do where that is 1
  int32_t ready;                 // entries, stats and count are those of an earlier call
  float temperature, weight;
};

}  // namespace compact
