// The draft model's paged cache and a step's tokens, as the kernels that write and read them see them, and the host's checks.
#pragma once

#include "common.cuh"

namespace spf {

constexpr int kScaleTokens = SPF_KV_SCALE_TOKENS, kScaleDims = SPF_KV_SCALE_DIMS;

struct KvView {
  uint8_t *k, *v;              // pools: bf16, E4M3 or codes [n_blocks][n_kv_heads][block_tokens][d]
  float *k_scale, *v_scale;    // 8-bit pools: [n_blocks][n_kv_heads][block_tokens / 64]
  uint16_t *k_scale4, *v_scale4;    // 4-bit pools: bf16 [n_blocks][n_kv_heads][block_tokens][d / 32]
  int64_t n_blocks;
  int block_tokens, n_kv_heads;
  int bits;                    // 16, 8 or 4
};

struct StepView {
  const int32_t *row_start, *seq_lens, *table;
  int n_seqs, n_rows, table_stride;
};

struct RowsView {
  __nv_bfloat16* data;
  int64_t stride_row, stride_head;
};

// Device-side conditions of the cache calls: the first one stays.
__device__ __forceinline__ void report_cache(int32_t* dev_status) {
  if (dev_status != nullptr) atomicCAS(dev_status, 0, (int32_t)SPF_ERR_CACHE);
}

// Place in its sequence of a token that has `behind` tokens from it on: below zero where the sequence is shorter than that, and kept where
// 2^30 rows more stay below zero, whatever the length says.
__device__ __forceinline__ int place_from_end(int len, int64_t behind) { return (int)min(max(len - behind, -(int64_t)(1 << 30)), (int64_t)0x7fffffff); }

// Pool block of a token, -1 where the table or the pool has no such place.
__device__ __forceinline__ int64_t pool_block(const KvView& kv, const StepView& st, int seq, int pos) {
  const int j = pos / kv.block_tokens;
  if (pos < 0 || j >= st.table_stride) return -1;
  const int b = __ldg(st.table + (int64_t)seq * st.table_stride + j);
  return b >= 0 && b < kv.n_blocks ? b : -1;
}

// Bits of a cache's elements; the caller has checked it.
inline int cache_bits(const spf_kv_cache* c) { return c->bits != 0 ? c->bits : c->k_scale != nullptr ? 8 : 16; }

// Host checks, shared by the calls on the cache; they leave the reason in the error text.
int32_t check_cache(const char* who, const spf_kv_cache* cache, KvView* out);
int32_t check_step(const char* who, const spf_kv_step* step, StepView* out);
int32_t check_ledger(const char* who, const spf_kv_ledger* ledger);
int32_t check_rows(const char* who, const char* name, const spf_rows* rows, int n_heads, int head_dim, bool written, RowsView* out);
// Whether rows `a` that a call reads and rows `b` that it writes (`n_rows` of either, of so many heads) have an element in common.
bool rows_meet(const RowsView& a, int a_heads, const RowsView& b, int b_heads, int n_rows, int head_dim);
int32_t device_sm_count(int* out);

}  // namespace spf
