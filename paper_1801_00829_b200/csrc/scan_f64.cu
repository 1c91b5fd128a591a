// Gated linear recurrence: the kernels for x of double with gates of double.
#include "scan_launch.cuh"

namespace fo {

template cudaError_t launch_scan<double, double>(ScanParams, bool, void *, cudaStream_t);

}  // namespace fo
