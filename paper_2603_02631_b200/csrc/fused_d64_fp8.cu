// Instantiations of the fused scoring kernel: head dimension 64, E4M3 keys.
#include "fused.cuh"

namespace spf {
int32_t fused_launch_d64_fp8(const FusedArgs& args, const FusedLaunch& l, cudaStream_t stream) {
  return l.scale_groups ? fused_launch_d64_fp8_groups(args, l, stream) : fused_launch<64, 1>(args, l, stream);
}
}  // namespace spf
