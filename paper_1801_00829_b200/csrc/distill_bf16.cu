// Distillation loss and gradient: the kernels for logits of __nv_bfloat16.
#include "distill_launch.cuh"

namespace fo {

template cudaError_t launch_distill<__nv_bfloat16>(DistillParams, DistillWay, cudaStream_t);

}  // namespace fo
