// How a recurrence is cut into CTAs and clusters, for one pair of element types.
#pragma once

#include <algorithm>
#include <atomic>

#include "launch.cuh"
#include "scan.cuh"

namespace fo {

// Channels of a lane, and tokens of a segment: forwards 16 of 16-bit x (8 x 4096 x 2048 in bfloat16 77 us, with 8 tokens 97), backwards
// half of that, by the registers that their decays take.
template <class T> constexpr int scan_channels() { return sizeof(T) == 8 ? 1 : 2; }
template <class T> constexpr int scan_tokens(bool grad) { return (sizeof(T) == 2 ? 8 : 4) * (grad || sizeof(T) == 8 ? 1 : 2); }

// How many clusters of 1 .. kScanMostCluster CTAs the GPU works on at once, asked once for each GPU, kernel and number of warps.
// What does not fit runs after the rest, and doubles the time (65536 x 2560: 6 CTAs a cluster 301 us, 7 486).
template <class K>
class ScanFit {
    std::atomic<int> known_[64][kScanMostCluster + 1] = {};

public:
    int clusters(K kernel, int gpu, int threads, size_t shared, int cluster)
    {
        if (gpu < 0 || gpu >= 64) return 0;
        std::atomic<int> &at = known_[gpu][cluster];
        int n = at.load(std::memory_order_relaxed);
        if (n) return n - 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)cluster);
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = shared;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {(unsigned)cluster, 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) cudaGetLastError(), n = 0;
        at.store(n + 1, std::memory_order_relaxed);
        return n;
    }
};

template <class T, class G, bool GRAD>
cudaError_t scan_launch(ScanParams p, cudaStream_t st)
{
    constexpr int V = scan_channels<T>(), S = scan_tokens<T>(GRAD);
    using Shared = ScanShared<typename ScanUnit<Acc<T>, V>::U>;
    using Ring = ScanRing<T, G, V, S, GRAD>;
    using Kernel = void (*)(ScanParams);
    static OncePerGpu once;
    static ScanFit<Kernel> fit;
    Kernel kernel;
    if constexpr (GRAD) kernel = scan_grad_kernel<T, G, V, S>;
    else kernel = scan_kernel<T, G, V, S>;
    cudaError_t e = once.allow(kernel, Ring::kBytes * kScanMostWarps + Shared::bytes(kScanMostWarps, kScanMostCluster));
    int gpu = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&gpu);
    if (e != cudaSuccess) return e;
    p.tiles = (int)((p.channels + 32 * V - 1) / (32 * V));
    const long long items = p.tiles * p.batch;
    int warps = 1, cluster = 1;
    while (warps < kScanMostWarps && warps * S < p.tokens) warps *= 2;
    const auto shared = [&](int k) { return Ring::kBytes * warps + Shared::bytes(warps, k); };
    // longer sequences of few channels over as many CTAs as all work at once
    if (warps == kScanMostWarps)
        while (cluster < kScanMostCluster && items <= 1000 && cluster * warps * S < p.tokens
               && fit.clusters(kernel, gpu, 32 * warps, shared(cluster + 1), cluster + 1) >= items)
            ++cluster;
    return launch_beside(kernel, dim3((unsigned)(items * cluster)), 32 * warps, st, shared(cluster), p, cluster);
}

template <class T, class G>
cudaError_t launch_scan(ScanParams p, bool grad, cudaStream_t st)
{
    // a decoding step takes 5.9 us this way, 8.9 by segments (64 x 1 x 4096)
    if (!grad && p.tokens <= 4) {
        constexpr int V = scan_channels<T>();
        const long long threads = p.batch * ((p.channels + V - 1) / V);
        return launch_beside(scan_step_kernel<T, G, V>, dim3((unsigned)((threads + kScanCta - 1) / kScanCta)), kScanCta, st, (size_t)0, p);
    }
    return grad ? scan_launch<T, G, true>(p, st) : scan_launch<T, G, false>(p, st);
}

}  // namespace fo
