// Head norms with rotation: the kernels for float.
#include "head_norm_launch.cuh"

namespace fo {

template cudaError_t launch_head_norm<float>(const HeadParams &, int, int, bool, bool, int, cudaStream_t);

}  // namespace fo
