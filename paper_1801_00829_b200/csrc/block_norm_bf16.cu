// Block norm and its gradient: stream of __nv_bfloat16, block of __nv_bfloat16.
#define FO_BLOCK_NORM_DEFINE
#include "block_norm_launch.cuh"

namespace fo {
template cudaError_t launch_block_norm<__nv_bfloat16, __nv_bfloat16>(const BlockNormParams &, cudaStream_t);
template cudaError_t launch_block_norm_grad<__nv_bfloat16, __nv_bfloat16>(BlockNormGradParams, int, int *, cudaStream_t);
}  // namespace fo
