// Gated linear recurrence: the kernels for x of __nv_bfloat16 with gates of __nv_bfloat16.
#include "scan_launch.cuh"

namespace fo {

template cudaError_t launch_scan<__nv_bfloat16, __nv_bfloat16>(ScanParams, bool, void *, cudaStream_t);

}  // namespace fo
