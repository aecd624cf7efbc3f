// Joins the parts of triples (sequence, row tile, key head) that several CTAs of an attention kernel computed.
#include <algorithm>

#include "attend.cuh"

namespace spf {
namespace {

// Joins the parts of the triple that CTA blockIdx.x began and others went on with, row by row.  Four warps share a row's parts (at
// 8000 tokens of one sequence a triple has 32), each with its loads in flight together: what the kernel takes is their latency.
template <int D, bool FP8, int R>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendParts args) {
  constexpr int V = D / 32;                              // columns of a lane
  __shared__ float sums[4][D], weights[4];
  grid_wait();
  const int4 head = args.headers[2 * blockIdx.x];
  if (head.x <= 0) return;
  const int live = args.headers[2 * blockIdx.x + 1].x, parts = head.x + 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto slot = [&](int i) { return i == 0 ? 2 * (int)blockIdx.x + 1 : 2 * ((int)blockIdx.x + i); };
  for (int r = blockIdx.y; r < live; r += gridDim.y) {
    RowStats all{-INFINITY, -INFINITY, 0.f};             // references are finite, also of parts whose keys the row does not see
    for (int i = lane; i < parts; i += 32) {
      const float2 s = __ldcg(reinterpret_cast<const float2*>(&args.stats[slot(i) * R + r]));
      all.m = fmaxf(all.m, s.x);
      all.m_sum = fmaxf(all.m_sum, s.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      all.m = fmaxf(all.m, __shfl_xor_sync(0xffffffffu, all.m, o));
      if (FP8) all.m_sum = fmaxf(all.m_sum, __shfl_xor_sync(0xffffffffu, all.m_sum, o));
    }
    if (!FP8) all.m_sum = all.m;
    float x[V] = {}, l = 0.f;
    for (int i0 = warp; i0 < parts; i0 += 128) {
      // the warp's parts i0, i0 + 4, ...: a lane has the statistics of one of 32
      float f = 0.f;
      if (i0 + 4 * lane < parts) {
        const float4 s = __ldcg(&args.stats[slot(i0 + 4 * lane) * R + r]);
        f = fast_exp2(s.x - all.m);
        l += s.z * (FP8 ? fast_exp2(s.y - all.m_sum) : f);
      }
#pragma unroll 8
      for (int i = 0; i < 32 && i0 + 4 * i < parts; ++i) {
        const float w = __shfl_sync(0xffffffffu, f, i);
        float v[V];
        const float* src = args.sums + ((int64_t)slot(i0 + 4 * i) * R + r) * D + lane * V;
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
#pragma unroll
    for (int j = 0; j < V; ++j) sums[warp][lane * V + j] = x[j];
    if (lane == 0) weights[warp] = l;
    __syncthreads();
    all.l = (weights[0] + weights[1]) + (weights[2] + weights[3]);
    const int rr = head.w * R + r, t = 2 * threadIdx.x;
    const int64_t row = head.y + rr / a.group;
    const int h = head.z * a.group + rr % a.group;
    const float inv = all.l == 0.f ? 0.f : 1.f / all.l, factor = output_factor<FP8>(all);
    if (t < D) {
      const float u = (sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]);
      const float v = (sums[0][t + 1] + sums[1][t + 1]) + (sums[2][t + 1] + sums[3][t + 1]);
      *reinterpret_cast<uint32_t*>(a.out.data + row * a.out.stride_row + h * a.out.stride_head + t) =
          pack_bf16(nan_if_infinite<FP8>(u) * inv * factor, nan_if_infinite<FP8>(v) * inv * factor);
    }
    if (a.lse != nullptr && threadIdx.x == 0) a.lse[row * a.lse_stride_row + h * a.lse_stride_head] = row_lse(all);
    __syncthreads();
  }
}

template <int D, bool FP8, int R>
int32_t launch(const AttendArgs& a, const AttendParts& parts, int live, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t config{};
  config.gridDim = dim3((unsigned)ctas, (unsigned)std::min(std::min(R, live), 64));
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
int32_t launch_rows(const AttendArgs& a, const AttendParts& parts, int rows, int live, int ctas, cudaStream_t stream) {
  switch (rows) {
    case 8: return launch<D, FP8, 8>(a, parts, live, ctas, stream);
    case 16: return launch<D, FP8, 16>(a, parts, live, ctas, stream);
    case 32:
      if constexpr (!(D == 128 && FP8)) return launch<D, FP8, 32>(a, parts, live, ctas, stream);   // else such steps have their tiles of 256
      break;
  }
  return launch<D, FP8, 256>(a, parts, live, ctas, stream);
}

}  // namespace

int32_t attend_join_launch(const AttendArgs& a, const AttendParts& parts, int rows, int live, int head_dim, bool fp8, int ctas, cudaStream_t stream) {
  if (head_dim == 64) return fp8 ? launch_rows<64, true>(a, parts, rows, live, ctas, stream) : launch_rows<64, false>(a, parts, rows, live, ctas, stream);
  return fp8 ? launch_rows<128, true>(a, parts, rows, live, ctas, stream) : launch_rows<128, false>(a, parts, rows, live, ctas, stream);
}

}  // namespace spf
