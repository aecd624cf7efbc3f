// Joins the parts of triples (sequence, row tile, key head) that several CTAs of an attention kernel computed.
#include "attend.cuh"

namespace spf {
namespace {

// Joins the parts of the triples that CTA blockIdx.x began and others went on with: a warp per row.
template <int D, bool FP8, int R>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendParts args) {
  grid_wait();
  const int4 head = args.headers[2 * blockIdx.x];
  const int r = blockIdx.y * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (head.x <= 0 || r >= args.headers[2 * blockIdx.x + 1].x) return;
  const int parts = head.x + 1;
  auto slot = [&](int i) { return i == 0 ? 2 * (int)blockIdx.x + 1 : 2 * ((int)blockIdx.x + i); };
  float top = -INFINITY;
  for (int i = lane; i < parts; i += 32) top = fmaxf(top, args.stats[slot(i) * R + r].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  constexpr int V = D / 32;                              // columns of a lane
  float x[V] = {}, l = 0.f;
  for (int i0 = 0; i0 < parts; i0 += 32) {
    // a lane has the statistics of one of 32 parts; the sums' loads then wait for nothing
    float2 s = make_float2(-INFINITY, 0.f);
    if (i0 + lane < parts) s = args.stats[slot(i0 + lane) * R + r];
    const float f = s.x == -INFINITY ? 0.f : fast_exp2(s.x - top);
    l += s.y * f;
#pragma unroll 8
    for (int i = 0; i < min(32, parts - i0); ++i) {
      const float w = __shfl_sync(0xffffffffu, f, i);
      float v[V];
      const float* src = args.sums + ((int64_t)slot(i0 + i) * R + r) * D + lane * V;
      if constexpr (V == 4) {
        const float4 t = __ldcg(reinterpret_cast<const float4*>(src));
        v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
      } else {
        const float2 t = __ldcg(reinterpret_cast<const float2*>(src));
        v[0] = t.x, v[1] = t.y;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] += v[j] * w;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  const int rr = head.w * R + r;
  const int64_t row = head.y + rr / a.group;
  const int h = head.z * a.group + rr % a.group;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint32_t* dst = reinterpret_cast<uint32_t*>(a.out.data + row * a.out.stride_row + h * a.out.stride_head) + lane * (V / 2);
#pragma unroll
  for (int j = 0; j < V / 2; ++j) dst[j] = pack_bf16(nan_if_infinite<FP8>(x[2 * j]) * inv, nan_if_infinite<FP8>(x[2 * j + 1]) * inv);
  if (a.lse != nullptr && lane == 0)
    a.lse[row * a.lse_stride_row + h * a.lse_stride_head] = row_lse<FP8>(top, l);
}

template <int D, bool FP8, int R>
int32_t launch(const AttendArgs& a, const AttendParts& parts, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t config{};
  config.gridDim = dim3((unsigned)ctas, R / 4);
  config.blockDim = dim3(128);
  config.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  config.attrs = &attr;
  config.numAttrs = 1;
  SPF_CUDA_CHECK(cudaLaunchKernelEx(&config, attend_join_kernel<D, FP8, R>, a, parts));
  return SPF_OK;
}

template <int D, bool FP8>
int32_t launch_rows(const AttendArgs& a, const AttendParts& parts, int rows, int ctas, cudaStream_t stream) {
  switch (rows) {
    case 8: return launch<D, FP8, 8>(a, parts, ctas, stream);
    case 16: return launch<D, FP8, 16>(a, parts, ctas, stream);
    case 32: return launch<D, FP8, 32>(a, parts, ctas, stream);
    case 64: return launch<D, FP8, 64>(a, parts, ctas, stream);
    default: return launch<D, FP8, 256>(a, parts, ctas, stream);
  }
}

}  // namespace

int32_t attend_join_launch(const AttendArgs& a, const AttendParts& parts, int rows, int head_dim, bool fp8, int ctas, cudaStream_t stream) {
  if (head_dim == 64) return fp8 ? launch_rows<64, true>(a, parts, rows, ctas, stream) : launch_rows<64, false>(a, parts, rows, ctas, stream);
  return fp8 ? launch_rows<128, true>(a, parts, rows, ctas, stream) : launch_rows<128, false>(a, parts, rows, ctas, stream);
}

}  // namespace spf
