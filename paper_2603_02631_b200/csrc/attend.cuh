// Attention of a step's tokens over the paged cache: what its kernels share.
#pragma once

#include <cuda_fp16.h>

#include "kv.cuh"
#include "tc_ptx.cuh"

namespace spf {

struct AttendArgs {
  KvView kv;
  StepView step;
  RowsView q, out;
  float* lse;                     // may be null; element (row, head) at row * lse_stride_row + head * lse_stride_head
  int64_t lse_stride_row, lse_stride_head;
  const int32_t* first_keys;      // may be null: [n_seqs]
  int group, causal;
  float c;                        // softmax scale * log2(e)
  int32_t* dev_status;
};

// A sequence's part in the step.
struct SeqSpan {
  int row0, n_new;                // its rows
  int pos0;                       // place of the first of them (negative: fewer tokens than rows, reported)
  int first, end;                 // keys of the cache that any of its rows may see: [first, end)
};

__device__ __forceinline__ SeqSpan seq_span(const AttendArgs& a, int b) {
  SeqSpan s;
  s.row0 = max(__ldg(a.step.row_start + b), 0);
  s.n_new = max(min(__ldg(a.step.row_start + b + 1), a.step.n_rows) - s.row0, 0);
  const int len = __ldg(a.step.seq_lens + b);
  s.pos0 = len - (__ldg(a.step.row_start + b + 1) - s.row0);
  s.end = max((int)min((int64_t)len, (int64_t)a.step.table_stride * a.kv.block_tokens), 0);
  s.first = a.first_keys != nullptr ? min(max(__ldg(a.first_keys + b), 0), s.end) : 0;
  if (s.n_new > 0 && (s.end != len || s.pos0 < 0)) report_cache(a.dev_status);
  return s;
}

// Row of the pool (as the tensor maps count them, over blocks and heads) of a token's key; a place outside the pool is a row
// outside the map, which reads as zeros.
__device__ __forceinline__ int pool_row(const AttendArgs& a, int seq, int head, int pos) {
  const int64_t block = pool_block(a.kv, a.step, seq, pos);
  if (block < 0) {
    report_cache(a.dev_status);
    return 0x7fffff00;
  }
  return (int)((block * a.kv.n_kv_heads + head) * a.kv.block_tokens + pos % a.kv.block_tokens);
}

// Factor of a group of 64 tokens, 1 outside the pool (its bytes then read as zeros).
__device__ __forceinline__ float group_scale(const float* scale, int pool_row, int64_t rows) {
  return pool_row < rows ? __ldg(scale + pool_row / kScaleTokens) : 1.f;
}

// One copy of a tile of pool rows, all spans of them, completing `bar`.
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
               : "memory");
}

// Waits, a second at most, for a copy that an aborting CTA still has in flight.
__device__ __forceinline__ void drain_copy(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = global_timer();
  while (!mbar_test_wait(bar, parity) && global_timer() - t0 < 1000000000ull) {}
}

// Tensor map of a pool: rows of d elements seen as spans of at most 128 bytes, `tile_rows` rows a copy.
int32_t encode_pool_map(const char* who, const spf_kv_cache* cache, void* pool, int tile_rows, CUtensorMap* map);

// The two kernels: a few rows a head and sequence, keys split over the chip; many rows.
size_t attend_step_workspace_bytes(const spf_kv_cache* cache, int group, int max_new, int sm_count);
int32_t attend_step_launch(const AttendArgs& a, const spf_kv_cache* cache, int max_new, int sm_count, void* workspace, cudaStream_t stream);

}  // namespace spf
