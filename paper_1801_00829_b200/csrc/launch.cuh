// Launches with shared memory, clusters, and beside the kernel before them on the stream (such a kernel calls wait_for_earlier()).
#pragma once

#include <atomic>

#include "elem.cuh"

namespace fo {

// Lets a kernel have more than 48 KB of shared memory, once for each GPU.
class OncePerGpu {
    std::atomic<unsigned long long> done_{0};

public:
    template <class K>
    cudaError_t allow(K kernel, size_t bytes)
    {
        int gpu = 0;
        cudaError_t e = cudaGetDevice(&gpu);
        if (e != cudaSuccess) return e;
        const unsigned long long bit = gpu < 64 ? 1ull << gpu : 0;
        if (done_.load(std::memory_order_relaxed) & bit) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e == cudaSuccess) done_.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};

template <class P>
cudaError_t launch_beside(void (*kernel)(P), dim3 grid, int cta, cudaStream_t st, size_t shared, const P &params, int cluster = 1)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)cta);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, params);
}

}  // namespace fo
