// Distillation loss and gradient: the kernels for logits of __half.
#include "distill_launch.cuh"

namespace fo {

template cudaError_t launch_distill<__half>(DistillParams, DistillWay, cudaStream_t);

}  // namespace fo
