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

// Whether a call's sequences are cut into chunks.  `room`: CTAs for each 32 V channels of a sequence that find a place at once; `rounds`: how
// many the largest clusters would take.  Below eight the two more launches and the second reading cost more than they give
// (bfloat16, 1 x 2048 x 512: in clusters 10 us forwards and 20 backwards, in chunks 16 and 24; 1 x 8192 x 1024: 33 and 70, 26 and
// 40), and forwards, where all inputs are read twice, so it is when the clusters fill the GPU (1 x 65536 x 2560, side by side: 374 and 440;
// backwards, where two of four are, 660 and 478).
inline bool scan_chunked(bool grad, long long room, long long rounds) { return rounds >= 8 && room >= (grad ? 4 : 16); }
constexpr int kScanLeastChunk = 4;      // rounds; 1 x 65536 x 32 forwards: with four 39 us, two 41, eight 54

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
cudaError_t scan_launch(ScanParams p, void *ws, cudaStream_t st)
{
    constexpr int V = scan_channels<T>(), S = scan_tokens<T>(GRAD);
    using A = Acc<T>;
    using Shared = ScanShared<typename ScanUnit<A, V>::U>;
    using Ring = ScanRing<T, G, V, S, GRAD>;
    using Kernel = void (*)(ScanParams);
    static OncePerGpu once, cluster_once;
    static ScanFit<Kernel> fit;
    Kernel kernel, cluster_kernel;
    if constexpr (GRAD) kernel = scan_grad_kernel<T, G, V, S, false>, cluster_kernel = scan_grad_kernel<T, G, V, S, true>;
    else kernel = scan_kernel<T, G, V, S, false>, cluster_kernel = scan_kernel<T, G, V, S, true>;
    const size_t most_shared = Ring::kBytes * kScanMostWarps + Shared::bytes(kScanMostWarps, kScanMostCluster);
    cudaError_t e = once.allow(kernel, most_shared);
    if (e == cudaSuccess) e = cluster_once.allow(cluster_kernel, most_shared);
    int gpu = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&gpu);
    if (e != cudaSuccess) return e;
    p.tiles = (int)((p.channels + 32 * V - 1) / (32 * V));
    const long long items = p.tiles * p.batch;
    int warps = 1, cluster = 1;
    while (warps < kScanMostWarps && warps * S < p.tokens) warps *= 2;
    const auto shared = [&](int k) { return Ring::kBytes * warps + Shared::bytes(warps, k); };
    const long long room = 2LL * std::min(sm_count(), kScanMostSms) / items;             // chunks that find room at once
    p.chunks = 1, p.chunk = p.tokens;
    if (p.tokens >= kScanLeastChunked && scan_chunked(GRAD, room, p.tokens / (kScanMostCluster * kScanMostWarps * S))) {
        const int round = warps * S, most = (int)std::min<long long>(room, p.tokens / (kScanLeastChunk * round));
        p.chunk = ((p.tokens + most - 1) / most + round - 1) / round * round;
        p.chunks = (p.tokens + p.chunk - 1) / p.chunk;
    }
    if (p.chunks > 1) {
        static OncePerGpu map_once;
        const size_t states = (size_t)p.batch * p.chunks * p.channels * sizeof(A), rings = ScanMapRing<T, G, V>::kBytes * kScanMostWarps;
        char *const at = static_cast<char *>(ws) + sizeof(WsHead);
        p.map_a = at, p.map_h = at + states, p.carry = at + 2 * states, p.map_drops = reinterpret_cast<int *>(at + 3 * states);
        e = map_once.allow(scan_map_kernel<T, G, V, GRAD>, rings);
        if (e == cudaSuccess) e = launch_beside(scan_map_kernel<T, G, V, GRAD>, dim3((unsigned)(items * p.chunks)), kScanCta, st, rings, p);
        const unsigned ctas = (unsigned)((p.batch * p.channels + kScanCta - 1) / kScanCta);
        if (e == cudaSuccess) e = launch_beside(scan_carry_kernel<A, GRAD>, dim3(ctas), kScanCta, st, (size_t)0, p);
        if (e != cudaSuccess) return e;
    } else if (warps == kScanMostWarps) {
        // longer sequences of few channels over as many CTAs as all work at once
        while (cluster < kScanMostCluster && items <= 1000 && cluster * warps * S < p.tokens
               && fit.clusters(cluster_kernel, gpu, 32 * warps, shared(cluster + 1), cluster + 1) >= items)
            ++cluster;
    }
    return launch_beside(cluster > 1 ? cluster_kernel : kernel, dim3((unsigned)(items * p.chunks * cluster)), 32 * warps, st, shared(cluster), p, cluster);
}

template <class T, class G>
cudaError_t launch_scan(ScanParams p, bool grad, void *ws, cudaStream_t st)
{
    // a decoding step takes 5.9 us this way, 8.9 by segments (64 x 1 x 4096)
    if (!grad && p.tokens <= 4) {
        constexpr int V = scan_channels<T>();
        const long long threads = p.batch * ((p.channels + V - 1) / V);
        return launch_beside(scan_step_kernel<T, G, V>, dim3((unsigned)((threads + kScanCta - 1) / kScanCta)), kScanCta, st, (size_t)0, p);
    }
    return grad ? scan_launch<T, G, true>(p, ws, st) : scan_launch<T, G, false>(p, ws, st);
}

}  // namespace fo
