// How a recurrence is cut into CTAs and clusters, for one pair of element types.
#pragma once

#include "launch.cuh"
#include "scan.cuh"

namespace fo {

// Tokens of a segment: as many as leave a thread its registers.
template <class T, class G>
constexpr int scan_tokens(bool grad)
{
    return sizeof(T) == 8 ? 4 : grad ? (sizeof(T) == 2 && sizeof(G) == 2 ? 8 : 4) : 8;
}

template <class T, class G, int V, bool GRAD>
cudaError_t scan_launch(ScanParams p, long long batch, cudaStream_t st)
{
    constexpr int S = scan_tokens<T, G>(GRAD);
    p.tiles = (p.channels + 32 * V - 1) / (32 * V);
    const long long items = p.tiles * batch;
    if (items > 0x7fffffffLL / kScanMostCluster) return cudaErrorInvalidConfiguration;
    const int sms = sm_count();
    int warps = 1, cluster = 1;
    while (warps < 8 && (long long)warps * S < p.tokens) warps *= 2;
    // a round of all CTAs together is to occupy the GPU, and no more than that
    while (cluster < kScanMostCluster && items * cluster * 2 <= (long long)sms * 3 && (long long)cluster * warps * S < p.tokens) cluster *= 2;
    const size_t shared = ScanShared<Acc<T>, V>::bytes(warps, cluster);
    const dim3 grid((unsigned)(items * cluster));
    if constexpr (GRAD) return launch_beside(scan_grad_kernel<T, G, V, S>, grid, 32 * warps, st, shared, p, cluster);
    else return launch_beside(scan_kernel<T, G, V, S>, grid, 32 * warps, st, shared, p, cluster);
}

// wide: channels can move in pairs (16-bit types)
template <class T, class G>
cudaError_t launch_scan(const ScanParams &p, bool wide, bool grad, long long batch, cudaStream_t st)
{
    if constexpr (sizeof(T) == 2)
        if (wide) return grad ? scan_launch<T, G, 2, true>(p, batch, st) : scan_launch<T, G, 2, false>(p, batch, st);
    return grad ? scan_launch<T, G, 1, true>(p, batch, st) : scan_launch<T, G, 1, false>(p, batch, st);
}

}  // namespace fo
