// The attention weights that a cache's tokens receive from a step's rows: what its kernels share.
#pragma once

#include "attend.cuh"

namespace spf {

struct WeighArgs {
  AttendArgs a;                   // its lse is read; `out` is not used
  CUtensorMap k_map, k_scale_map, weight_map;   // few rows; the second: 4 bits
  CUtensorMap q_map;              // many rows
  float* weight;                  // [n_blocks][n_kv_heads][block_tokens]
  int32_t* position;              // the same; may be null
  const int32_t* positions;       // [n_rows]; null: a token's place
  float decay;
  int last_rows;                  // of a sequence's new tokens, those that count; 0: all
};

// A sequence's part in the call: its rows that count, and the places of its new tokens.
struct WeighSpan {
  SeqSpan rows;                   // row0, n_new and pos0 of the rows that count
  int fresh, fresh_row;           // place and row of the first new token
};
__device__ __forceinline__ WeighSpan weigh_span(const WeighArgs& w, int b) {
  WeighSpan s;
  s.rows = seq_span(w.a, b);
  s.fresh = s.rows.pos0;
  s.fresh_row = s.rows.row0;
  const int skip = w.last_rows > 0 ? max(s.rows.n_new - w.last_rows, 0) : 0;
  s.rows.row0 += skip;
  s.rows.pos0 += skip;
  s.rows.n_new -= skip;
  return s;
}

// What a key has received: `got` joins what the ledger holds, or replaces it where the token is one of the step's.
__device__ __forceinline__ void book(const WeighArgs& w, int64_t cell, float held, float got, int key, int fresh, int fresh_row) {
  if (key < fresh) {
    w.weight[cell] = w.decay != 0.f ? fmaf(held, w.decay, got) : got;      // memory that was never written may hold NaN
    return;
  }
  w.weight[cell] = got;
  const int64_t row = (int64_t)fresh_row + key - fresh;
  if (w.position != nullptr) w.position[cell] = w.positions != nullptr && row < w.a.step.n_rows ? __ldg(w.positions + row) : key;
}

// The kernel for many rows a key head and sequence; that for few is weigh.cu's own.
bool weigh_prompt_prepare(WeighArgs& w, int n_q_heads, int head_dim);       // false: its copies cannot read the queries
int32_t weigh_prompt_launch(const WeighArgs& w, int head_dim, int sm_count, cudaStream_t stream);

}  // namespace spf
