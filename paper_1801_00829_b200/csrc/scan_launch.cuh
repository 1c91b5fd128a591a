// How a recurrence is cut into CTAs and clusters, for one pair of element types.
#pragma once

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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(items * cluster));
    cfg.blockDim = dim3((unsigned)(32 * warps));
    cfg.dynamicSmemBytes = ScanShared<Acc<T>, V>::bytes(warps, cluster);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if constexpr (GRAD) return cudaLaunchKernelEx(&cfg, scan_grad_kernel<T, G, V, S>, p);
    else return cudaLaunchKernelEx(&cfg, scan_kernel<T, G, V, S>, p);
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
