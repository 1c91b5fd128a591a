// Gated linear recurrence: the kernels for x of __half with gates of float.
#include "scan_launch.cuh"

namespace fo {

template cudaError_t launch_scan<__half, float>(ScanParams, bool, void *, cudaStream_t);

}  // namespace fo
