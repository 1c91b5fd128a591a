// Gated linear recurrence: the kernels for x of float with gates of float.
#include "scan_launch.cuh"

namespace fo {

template cudaError_t launch_scan<float, float>(ScanParams, bool, void *, cudaStream_t);

}  // namespace fo
