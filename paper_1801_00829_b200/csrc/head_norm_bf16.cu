// Head norms with rotation: the kernels for __nv_bfloat16.
#include "head_norm_launch.cuh"

namespace fo {

template cudaError_t launch_head_norm<__nv_bfloat16>(const HeadParams &, int, int, bool, bool, int, cudaStream_t);

}  // namespace fo
