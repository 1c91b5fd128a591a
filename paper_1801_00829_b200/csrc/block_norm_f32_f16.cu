// Block norm and its gradient: stream of float, block of __half.
#define FO_BLOCK_NORM_DEFINE
#include "block_norm_launch.cuh"

namespace fo {
template cudaError_t launch_block_norm<float, __half>(const BlockNormParams &, cudaStream_t);
template cudaError_t launch_block_norm_grad<float, __half>(BlockNormGradParams, int, int *, cudaStream_t);
}  // namespace fo
