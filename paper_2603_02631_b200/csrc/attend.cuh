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
  s.pos0 = place_from_end(len, (int64_t)__ldg(a.step.row_start + b + 1) - s.row0);
  s.end = max((int)min((int64_t)len, (int64_t)a.step.table_stride * a.kv.block_tokens), 0);
  s.first = a.first_keys != nullptr ? min(max(__ldg(a.first_keys + b), 0), s.end) : 0;
  if (s.n_new > 0 && (s.end != len || s.pos0 < 0)) report_cache(a.dev_status);
  return s;
}

// Row of the pool (as the tensor maps count them, over blocks and heads) of a token's key; a place outside the pool is a row
// outside every map (pools have at most 2^31 - 128 rows), which reads as zeros.
__device__ __forceinline__ int pool_row(const AttendArgs& a, int seq, int head, int pos) {
  const int64_t block = pool_block(a.kv, a.step, seq, pos);
  if (block < 0) {
    report_cache(a.dev_status);
    return 0x7fffff80;
  }
  return (int)((block * a.kv.n_kv_heads + head) * a.kv.block_tokens + pos % a.kv.block_tokens);
}

// Factor of the group of 64 tokens at `key` (pool row `row`): 1 outside the pool, whose bytes then read as zeros, and for groups that
// no row sees, whose factor may be anything.
__device__ __forceinline__ float group_scale(const float* scale, const SeqSpan& s, int key, int row, int64_t rows) {
  return row < rows && key < s.end && key + kScaleTokens > s.first ? __ldg(scale + row / kScaleTokens) : 1.f;
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

// ---------------------------------------------------------------------------------------------- what both kernels compute with
constexpr float kLazy = 8.f;            // how far logits may exceed their reference
constexpr float kNoReference = -1.5e38f;   // of a row that has seen no key: finite, so that no difference of two is NaN
constexpr float kShift = 7.f;           // 8-bit values: their reference is that much lower: weights reach 2^15, below fp16's 65504
constexpr float kFar = 64.f;            // 8-bit values: how far the sum's weights may be above the products' and be made of them (RowStats)

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Four E4M3 bytes as two pairs of fp16, bytes 0 and 2, bytes 1 and 3, each times kWiden.  A byte s eeee mmm moved to the bits
// s 0eeee mmm0000000 of a half is its value times 2^-8, subnormals included.  The product with 9 * 2^12 (exact: 4 + 4 significant
// bits) leaves 448 at 64512, inside fp16, and takes the NaN patterns, which look like 480, to infinity.
constexpr float kWiden = 144.f;
__device__ __forceinline__ void widen4(uint32_t four, uint32_t& even, uint32_t& odd) {
  const __half2 up = __half2half2(__ushort_as_half(0x7880));
  const uint32_t e = (four & 0x00ff00ffu) * 128u + (four & 0x00800080u) * 128u;
  const uint32_t o = ((four >> 1) & 0x3f803f80u) | (four & 0x80008000u);
  const __half2 he = __hmul2(*reinterpret_cast<const __half2*>(&e), up), ho = __hmul2(*reinterpret_cast<const __half2*>(&o), up);
  even = *reinterpret_cast<const uint32_t*>(&he);
  odd = *reinterpret_cast<const uint32_t*>(&ho);
}
// What is not finite in an 8-bit pool can only have been NaN.
template <bool FP8>
__device__ __forceinline__ float nan_if_infinite(float x) {
  return FP8 && !(fabsf(x) <= 3.402823466e38f) ? __int_as_float(0x7fffffff) : x;
}

// Eight elements of a query row, whose largest magnitude is `top`, as bytes of two terms: x 2^e = hi (E4M3) + lo (E5M2).  2^e takes
// `top` to (224, 448]; e is clipped where 2^e or its inverse would leave fp32's normal range.
__device__ __forceinline__ void two_terms(const float (&f)[8], float top, int* e_out, uint2* hi_out, uint2* lo_out) {
  const uint32_t bits = __float_as_uint(top);
  const int e = top > 0.f && top < INFINITY ? min(max(135 - (int)(bits >> 23) - ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -120), 120) : 0;
  // a row with an infinite element has no softmax: NaN, not the largest finite byte
  const float up = __uint_as_float(top == INFINITY ? 0x7fffffffu : (uint32_t)(e + 127) << 23);
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = f[2 * i] * up, y = f[2 * i + 1] * up;
    uint32_t near;
    asm("{\n.reg .b16 t;\ncvt.rn.satfinite.e4m3x2.f32 t, %3, %2;\ncvt.u32.u16 %0, t;\ncvt.rn.f16x2.e4m3x2 %1, t;\n}" : "=r"(hi[i]), "=r"(near) : "f"(x), "f"(y));
    const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&near));
    asm("{\n.reg .b16 t;\ncvt.rn.satfinite.e5m2x2.f32 t, %2, %1;\ncvt.u32.u16 %0, t;\n}" : "=r"(lo[i]) : "f"(x - t.x), "f"(y - t.y));
  }
  *e_out = e;
  *hi_out = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
  *lo_out = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
}

// A row's references and the sum of its weights.  bf16: weights are 2^(z - m) in the products and in the sum, m_sum is m.  8 bits: they
// are 2^(z + log2 s_v - m) in the products, s_v being the scale of a group's values, and 2^(z - m_sum) in the sum.  Value scales may lie
// 2^200 apart (that of zeros is 2^-100), so that no reference holds both in fp32's range.  A group's sum of the former times
// 2^above_weights() is its part of the latter; where that factor is above 2^kFar, weights that fp32 has flushed to zero (below 2^-126)
// could matter, and the part is made of exponentials of its own.
struct RowStats {
  float m, m_sum, l;
};
// `off`: what a group's logits have added in the exponents of the products' weights.
__device__ __forceinline__ float above_weights(float off, float m_sum) { return -off - m_sum; }

// What a row's weighted values are multiplied by besides 1 / l.
template <bool FP8>
__device__ __forceinline__ float output_factor(const RowStats& s) {
  return FP8 ? fast_exp2(above_weights(-s.m, s.m_sum)) * (1.f / kWiden) : 1.f;
}

// 8 bits: factor from a row's accumulated products to base-2 logits.  Keys of the smallest scale under a tiny query take it below fp32's
// range, where it would make NaN of the -inf of masked keys, and the largest beyond it, where it would of zeros: it stays inside.
__device__ __forceinline__ float logit_factor(float k_scale, float q_factor) {
  float f;                                               // a NaN scale stays one
  asm("max.NaN.f32 %0, %1, 0f00800000;" : "=f"(f) : "f"(k_scale * q_factor));
  asm("min.NaN.f32 %0, %1, 0f7F7FFFFF;" : "=f"(f) : "f"(f));
  return f;
}

// Log-sum-exp (natural) of a row.
__device__ __forceinline__ float row_lse(const RowStats& s) { return s.l == 0.f ? -INFINITY : (s.m_sum + log2f(s.l)) * kLn2; }

// ---------------------------------------------------------------------------------------------- parts of a triple
// A triple (sequence, row tile, key head) whose tiles several CTAs share leaves partial sums: slot 2 c of CTA c for what an earlier
// CTA began, slot 2 c + 1 for what it began itself.
struct AttendParts {
  float* sums;                    // [2 ctas][R][D]
  float4* stats;                  // [2 ctas][R] RowStats
  int4* headers;                  // [ctas][2]: CTAs behind this one with parts of its last triple (0: none), row0, head, row tile; rows
};
struct PartsLayout {
  size_t sums, stats, headers, total;
};
inline PartsLayout parts_layout(int rows, int d, int ctas) {
  PartsLayout w;
  w.sums = 0;
  w.stats = align_up((size_t)2 * ctas * rows * d * sizeof(float), 256);
  w.headers = w.stats + align_up((size_t)2 * ctas * rows * sizeof(float4), 256);
  w.total = w.headers + align_up((size_t)2 * ctas * sizeof(int4), 256);
  return w;
}
inline AttendParts parts_at(void* workspace, int rows, int d, int ctas) {
  const PartsLayout w = parts_layout(rows, d, ctas);
  char* base = static_cast<char*>(workspace);
  return AttendParts{reinterpret_cast<float*>(base + w.sums), reinterpret_cast<float4*>(base + w.stats), reinterpret_cast<int4*>(base + w.headers)};
}
// Launches the kernel that joins parts, behind the one that leaves them.  `live`: rows that a tile of `rows` is expected to have at
// most; with more the kernel does its work in several rounds.
int32_t attend_join_launch(const AttendArgs& a, const AttendParts& parts, int rows, int live, int head_dim, bool fp8, int ctas, cudaStream_t stream);

// The two kernels: a few rows a head and sequence, keys split over the chip; many rows.
size_t attend_prompt_workspace_bytes(const spf_kv_cache* cache, int sm_count);
int32_t attend_prompt_launch(const AttendArgs& a, const spf_kv_cache* cache, int sm_count, void* workspace, cudaStream_t stream);
// Rows a key head and sequence up to which the first is taken.  Over 131072 keys and 8 heads, first against second, 32 rows: 61 us
// against 81 (64 dimensions), 80 against 91 (64, 8 bits), 109 against 114 (128), 157 against 139 (128, 8 bits, whose values' widening
// then takes longer than their read); 64 rows: 99 against 85, 134 against 97, 189 against 119, 281 against 148.  32 rows elsewhere, 8 heads,
// in the same order but for the last form, of which the first kernel has none: 32 sequences of 2000 keys 42 against 53, 52 against 63,
// 73 against 73; of 16000 keys 176 against 269, 246 against 302, 375 against 445; 256 sequences of 500 keys 87 against 119, 122 against 142,
// 165 against 153.  One sequence of 2000 keys and one of 16000 differ by 2 us or less but with 128 dimensions (18 against 16.5, 30 against 27).  With
// one key head, over 2000 to 131072 keys of one sequence, the second is up to 9 us the quicker one (34 against 25: 128 dimensions, 16000).
// 16 rows, 128 dimensions, 8 bits: 88 against 138 over 131072 keys, 288 against 473 for 32 sequences of 16000, 16 against 21 for one of 2000.
inline int step_rows(const spf_kv_cache* cache) { return cache->k_scale != nullptr && cache->head_dim == 128 ? 16 : 32; }
size_t attend_step_workspace_bytes(const spf_kv_cache* cache, int group, int max_new, int sm_count);
int32_t attend_step_launch(const AttendArgs& a, const spf_kv_cache* cache, int max_new, int sm_count, void* workspace, cudaStream_t stream);

}  // namespace spf
