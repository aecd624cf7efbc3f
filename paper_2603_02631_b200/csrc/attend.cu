// Host side of spf_attend: checks, workspace, choice of the kernel.
#include <algorithm>
#include <cmath>

#include "attend.cuh"

namespace spf {
namespace {

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) == cudaSuccess && found == cudaDriverEntryPointSuccess;
    return reinterpret_cast<EncodeFn>(ok ? p : nullptr);
  }();
  return fn;
}

// Enough for every step with up to `max_new` new tokens a sequence.
size_t workspace_for(const spf_kv_cache* cache, int group, int max_new, int sm_count) {
  const size_t few = attend_step_workspace_bytes(cache, group, max_new, sm_count);
  return (int64_t)group * max_new > step_rows(cache) ? std::max(few, attend_prompt_workspace_bytes(cache, sm_count)) : few;
}

}  // namespace

int32_t check_heads(const char* who, const spf_kv_cache* cache, int32_t n_q_heads, int* group) {
  if (n_q_heads < 1) return fail(SPF_ERR_INVALID_ARG, "%s: n_q_heads must be positive", who);
  if (n_q_heads % cache->n_kv_heads != 0)
    return fail(SPF_ERR_UNSUPPORTED, "%s: n_q_heads %d is not a multiple of n_kv_heads %d", who, n_q_heads, cache->n_kv_heads);
  *group = n_q_heads / cache->n_kv_heads;
  return SPF_OK;
}

int32_t attend_settings(const char* who, const spf_kv_cache* cache, const spf_kv_step* step, int32_t n_q_heads, float softmax_scale,
                        const spf_attend_options* options, AttendArgs* a) {
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)cache->head_dim);
  a->c = scale * kLog2e;
  if (!std::isfinite(a->c)) return fail(SPF_ERR_INVALID_ARG, "%s: softmax_scale is too large", who);
  a->causal = 1;
  if (options != nullptr) {
    a->causal = options->see_all == 0;
    a->first_keys = options->first_keys;
    a->lse = options->lse;
    a->lse_stride_row = options->lse_stride_row;
    a->lse_stride_head = options->lse_stride_head;
    if (a->lse != nullptr && (a->lse_stride_row < 0 || a->lse_stride_head < 0 || (n_q_heads > 1 && a->lse_stride_head < 1) || (step->n_rows > 1 && a->lse_stride_row < 1)))
      return fail(SPF_ERR_INVALID_ARG, "%s: the strides of lse must be positive", who);
  }
  return SPF_OK;
}

static cuuint64_t pool_rows(const spf_kv_cache* cache) {
  return (cuuint64_t)cache->n_pool_blocks * (cuuint64_t)cache->n_kv_heads * (cuuint64_t)cache->block_tokens;
}

int32_t encode_pool_map(const char* who, const spf_kv_cache* cache, void* pool, int tile_rows, CUtensorMap* map) {
  const EncodeFn encode = encoder();
  if (encode == nullptr) return fail(SPF_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available from the driver", who);
  const int bits = cache_bits(cache);
  const int es = bits == 16 ? 2 : 1, row = cache->head_dim * bits / 8, span = std::min(row, 128);
  const cuuint64_t rows = pool_rows(cache);
  const cuuint64_t dims[3] = {(cuuint64_t)(span / es), rows, (cuuint64_t)(row / span)};
  const cuuint64_t strides[2] = {(cuuint64_t)row, (cuuint64_t)span};
  const cuuint32_t box[3] = {(cuuint32_t)(span / es), (cuuint32_t)tile_rows, (cuuint32_t)(row / span)}, ones[3] = {1, 1, 1};
  const CUresult r = encode(map, bits == 16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, pool, dims, strides, box, ones,
                            CU_TENSOR_MAP_INTERLEAVE_NONE,
                            span == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                            : span == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                         : CU_TENSOR_MAP_SWIZZLE_32B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(SPF_ERR_CUDA, "%s: encoding a pool's tensor map failed (CUresult %d)", who, (int)r);
  return SPF_OK;
}

int32_t encode_rows_map(const char* who, const RowsView& rows, int n_rows, int n_heads, int head_dim, int tokens, int heads, CUtensorMap* map) {
  const EncodeFn encode = encoder();
  if (encode == nullptr) return fail(SPF_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available from the driver", who);
  const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)n_heads, (cuuint64_t)n_rows};
  const cuuint64_t strides[2] = {(cuuint64_t)(n_heads > 1 ? rows.stride_head : head_dim) * 2, (cuuint64_t)(n_rows > 1 ? rows.stride_row : head_dim) * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)tokens}, ones[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, rows.data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(SPF_ERR_CUDA, "%s: encoding a tensor map of rows failed (CUresult %d)", who, (int)r);
  return SPF_OK;
}
// Rows of `words` 32-bit words, one behind the other.
static int32_t encode_words(const char* who, void* data, cuuint64_t words, cuuint64_t rows, CUtensorMap* map) {
  const EncodeFn encode = encoder();
  if (encode == nullptr) return fail(SPF_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available from the driver", who);
  const cuuint64_t dims[2] = {words, rows}, strides[1] = {words * 4};
  const cuuint32_t box[2] = {(cuuint32_t)words, 1}, ones[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(SPF_ERR_CUDA, "%s: encoding a tensor map of scales or weights failed (CUresult %d)", who, (int)r);
  return SPF_OK;
}
int32_t encode_scale_map(const char* who, const spf_kv_cache* cache, void* scales, CUtensorMap* map) {
  return encode_words(who, scales, (cuuint64_t)(128 * cache->head_dim / kScaleDims / 2), pool_rows(cache) / 128, map);
}
int32_t encode_ledger_map(const char* who, const spf_kv_cache* cache, float* numbers, int tile_rows, CUtensorMap* map) {
  return encode_words(who, numbers, (cuuint64_t)tile_rows, pool_rows(cache) / (cuuint64_t)tile_rows, map);
}

}  // namespace spf

using namespace spf;

extern "C" size_t spf_attend_workspace_bytes(const spf_kv_cache* cache, int32_t n_q_heads, int32_t max_new) {
  const char* who = "spf_attend_workspace_bytes";
  clear_error();
  KvView kv;
  int group = 0, sm_count = 0;
  if (check_cache(who, cache, &kv) != SPF_OK || check_heads(who, cache, n_q_heads, &group) != SPF_OK) return 0;
  if (max_new < 1) return fail(SPF_ERR_INVALID_ARG, "%s: max_new must be positive", who), 0;
  if (device_sm_count(&sm_count) != SPF_OK) return 0;
  return workspace_for(cache, group, max_new, sm_count);
}

extern "C" int32_t spf_attend(const spf_kv_cache* cache, const spf_kv_step* step, const spf_rows* q, const spf_rows* out, int32_t n_q_heads,
                              float softmax_scale, const spf_attend_options* options, void* workspace, size_t workspace_bytes,
                              int32_t* dev_status, void* cuda_stream) {
  const char* who = "spf_attend";
  clear_error();
  AttendArgs a{};
  int32_t st = check_cache(who, cache, &a.kv);
  if (st == SPF_OK) st = check_step(who, step, &a.step);
  if (st == SPF_OK) st = check_heads(who, cache, n_q_heads, &a.group);
  if (st != SPF_OK) return st;
  if (step->n_rows == 0) return SPF_OK;
  st = check_rows(who, "q", q, n_q_heads, cache->head_dim, false, &a.q);
  if (st == SPF_OK) st = check_rows(who, "out", out, n_q_heads, cache->head_dim, true, &a.out);
  if (st != SPF_OK) return st;
  if (rows_meet(a.q, n_q_heads, a.out, n_q_heads, step->n_rows, cache->head_dim)) return fail(SPF_ERR_INVALID_ARG, "%s: out overlaps q", who);
  st = attend_settings(who, cache, step, n_q_heads, softmax_scale, options, &a);
  if (st != SPF_OK) return st;
  a.dev_status = dev_status;
  int sm_count = 0;
  st = device_sm_count(&sm_count);
  if (st != SPF_OK) return st;
  const size_t need = workspace_for(cache, a.group, step->max_new, sm_count);
  if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(SPF_ERR_WORKSPACE, "%s: workspace is null or not 256-byte aligned", who);
  if (workspace_bytes < need) return fail(SPF_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if ((int64_t)a.group * step->max_new > step_rows(cache)) return attend_prompt_launch(a, cache, sm_count, workspace, stream);
  return attend_step_launch(a, cache, step->max_new, sm_count, workspace, stream);
}
