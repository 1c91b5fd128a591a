// Distillation loss and gradient: the kernels for logits of float.
#include "distill_launch.cuh"

namespace fo {

template cudaError_t launch_distill<float>(DistillParams, DistillWay, cudaStream_t);

}  // namespace fo
