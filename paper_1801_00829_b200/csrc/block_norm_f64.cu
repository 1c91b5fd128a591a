// Block norm and its gradient: stream of double, block of double.
#define FO_BLOCK_NORM_DEFINE
#include "block_norm_launch.cuh"

namespace fo {
template cudaError_t launch_block_norm<double, double>(const BlockNormParams &, cudaStream_t);
template cudaError_t launch_block_norm_grad<double, double>(BlockNormGradParams, int, int *, cudaStream_t);
}  // namespace fo
