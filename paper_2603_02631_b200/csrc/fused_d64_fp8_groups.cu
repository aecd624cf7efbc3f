// Instantiations of the fused scoring kernel: head dimension 64, E4M3 keys with scales for groups of 64.
#include "fused.cuh"

namespace spf {
int32_t fused_launch_d64_fp8_groups(const FusedArgs& args, const FusedLaunch& l, cudaStream_t stream) { return fused_launch<64, 2>(args, l, stream); }
}  // namespace spf
