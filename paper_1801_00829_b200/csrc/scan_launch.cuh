// How a recurrence is cut into CTAs and clusters, for one pair of element types.
#pragma once

#include <algorithm>

#include <stdlib.h>
#include "launch.cuh"
#include "scan.cuh"

namespace fo {

// Channels of a lane and tokens of a segment.
template <class T> constexpr int scan_channels() { return sizeof(T) == 8 ? 1 : 2; }
template <class T> constexpr int scan_tokens(bool grad) { return (sizeof(T) == 2 ? 8 : 4) * (grad || sizeof(T) == 8 ? 1 : 2); }

template <class T, class G, bool GRAD>
cudaError_t scan_launch(ScanParams p, long long batch, cudaStream_t st)
{
    constexpr int V = scan_channels<T>(), S = scan_tokens<T>(GRAD);
    using Shared = ScanShared<typename ScanUnit<Acc<T>, V>::U>;
    using Ring = ScanRing<T, G, V, S>;
    static OncePerGpu once;
    void (*kernel)(ScanParams);
    if constexpr (GRAD) kernel = scan_grad_kernel<T, G, V, S>;
    else kernel = scan_kernel<T, G, V, S>;
    const cudaError_t e = once.allow(kernel, Ring::bytes(kScanMostWarps, GRAD) + Shared::bytes(kScanMostWarps, kScanMostCluster));
    if (e != cudaSuccess) return e;
    p.tiles = (int)((p.channels + 32 * V - 1) / (32 * V));
    const long long items = p.tiles * batch;
    const int sms = sm_count();
    int warps = 1;
    // as many warps as leave two CTAs room on an SM
    const int most = Ring::bytes(kScanMostWarps, GRAD) <= 100 * 1024 ? kScanMostWarps : kScanMostWarps / 2;
    while (warps < most && warps * S < p.tokens) warps *= 2;
    // as many CTAs as can work at once, two on an SM, where the sequences are long enough
    long long cluster = std::min<long long>(kScanMostCluster, 2LL * sms / items);
    cluster = std::max<long long>(1, std::min<long long>(cluster, (p.tokens + warps * S - 1) / (warps * S)));
    if (getenv("SCAN_W")) warps = atoi(getenv("SCAN_W"));
    if (getenv("SCAN_K")) cluster = atoi(getenv("SCAN_K"));
    return launch_beside(kernel, dim3((unsigned)(items * cluster)), 32 * warps, st, Ring::bytes(warps, GRAD) + Shared::bytes(warps, (int)cluster), p, (int)cluster);
}

template <class T, class G>
cudaError_t launch_scan(ScanParams p, bool grad, long long batch, cudaStream_t st)
{
    return grad ? scan_launch<T, G, true>(p, batch, st) : scan_launch<T, G, false>(p, batch, st);
}

}  // namespace fo
