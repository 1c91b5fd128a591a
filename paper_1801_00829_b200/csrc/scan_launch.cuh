// How a recurrence is cut into CTAs and clusters, for one pair of element types.
#pragma once

#include <stdlib.h>
#include "launch.cuh"
#include "scan.cuh"

namespace fo {

// Channels of a lane and tokens of a segment.
template <class T> constexpr int scan_channels() { return sizeof(T) == 8 ? 1 : 2; }
template <class T> constexpr int scan_tokens() { return sizeof(T) == 2 ? 8 : 4; }

template <class T, class G>
cudaError_t launch_scan(ScanParams p, bool grad, long long batch, cudaStream_t st)
{
    constexpr int V = scan_channels<T>(), S = scan_tokens<T>();
    using Shared = ScanShared<typename ScanUnit<Acc<T>, V>::U>;
    using Ring = ScanRing<T, G, V, S>;
    static OncePerGpu once[2];
    const auto kernel = grad ? scan_grad_kernel<T, G, V, S> : scan_kernel<T, G, V, S>;
    const cudaError_t e = once[grad].allow(kernel, Ring::bytes(kScanMostWarps, grad) + Shared::bytes(kScanMostWarps, kScanMostCluster));
    if (e != cudaSuccess) return e;
    p.tiles = (int)((p.channels + 32 * V - 1) / (32 * V));
    const long long items = p.tiles * batch;
    const int sms = sm_count();
    const char *tw = getenv("SCAN_W") ? getenv("SCAN_W") : "", *tk = getenv("SCAN_K") ? getenv("SCAN_K") : "";
    int warps = 1, cluster = 1;
    const int most = tw[0] ? atoi(tw) : kScanMostWarps;
    while (warps < most && warps * S < p.tokens) warps *= 2;
    // a round of all CTAs together is to occupy the GPU, and no more than that
    while (cluster < kScanMostCluster && items * cluster * 2 <= (long long)sms * 3 && cluster * warps * S < p.tokens) cluster *= 2;
    if (tk[0]) cluster = atoi(tk);
    return launch_beside(kernel, dim3((unsigned)(items * cluster)), 32 * warps, st, Ring::bytes(warps, grad) + Shared::bytes(warps, cluster), p, cluster);
}

}  // namespace fo
