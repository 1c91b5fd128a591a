// Distillation loss and gradient: the kernels for logits of double.
#include "distill_launch.cuh"

namespace fo {

template cudaError_t launch_distill<double>(DistillParams, DistillWay, cudaStream_t);

}  // namespace fo
