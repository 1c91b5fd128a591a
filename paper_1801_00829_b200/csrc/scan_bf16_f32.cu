// Gated linear recurrence: the kernels for x of __nv_bfloat16 with gates of float.
#include "scan_launch.cuh"

namespace fo {

template cudaError_t launch_scan<__nv_bfloat16, float>(ScanParams, bool, void *, cudaStream_t);

}  // namespace fo
