// Instantiations of the fused scoring kernel: head dimension 128, E4M3 keys with scales for groups of 64.
#include "fused.cuh"

namespace spf {
int32_t fused_launch_d128_fp8_groups(const FusedArgs& args, const FusedLaunch& l, cudaStream_t stream) { return fused_launch<128, 2>(args, l, stream); }
}  // namespace spf
