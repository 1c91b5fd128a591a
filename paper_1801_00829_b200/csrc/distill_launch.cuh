// How rows are spread over CTAs and clusters, for one element type.
#pragma once

#include <atomic>

#include "distill.cuh"

namespace fo {

constexpr int kDistillMostBytes = 196640;                 // of a row in one CTA's shared memory

// Lets a kernel have more than 48 KB of shared memory, once for each GPU.
template <class K>
cudaError_t distill_allow(K kernel, std::atomic<unsigned long long> &done)
{
    int gpu = 0;
    cudaError_t e = cudaGetDevice(&gpu);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (gpu & 63);
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDistillMostBytes + 20 * FO_DISTILL_MAX_TOP);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <class T, bool STEP>
cudaError_t distill_row_launch(DistillParams p, cudaStream_t st)
{
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = distill_allow(distill_kernel<T, STEP>, done);
    if (e != cudaSuccess) return e;
    // a row may begin anywhere in its first piece
    const long long pieces = ((long long)p.vocab * (int)sizeof(T) + 15 - (int)sizeof(T)) / 16 + 1;
    int cluster = 1;
    while (cluster < 8 && (pieces + cluster - 1) / cluster > 65536 / 16) cluster *= 2;
    p.slice = (int)((pieces + cluster - 1) / cluster);
    const int threads = p.slice >= 2048 ? 512 : p.slice >= 512 ? 256 : 128;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * cluster));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)p.slice * 16 + (size_t)p.top * 20;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, distill_kernel<T, STEP>, p);
}

template <class T>
cudaError_t launch_distill(DistillParams p, DistillWay way, cudaStream_t st)
{
    if (way == kDistillLoss) return distill_row_launch<T, false>(p, st);
    if (way == kDistillStep) return distill_row_launch<T, true>(p, st);
    const long long pieces = ((long long)p.vocab * (int)sizeof(T) + 15 - (int)sizeof(T)) / 16 + 1;
    constexpr int kThreads = 256, kMost = kThreads * 8;
    const int parts = (int)((pieces + kMost - 1) / kMost);
    p.slice = (int)((pieces + parts - 1) / parts);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.rows, (unsigned)parts);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)p.top * 20;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, distill_grad_kernel<T>, p);
}

}  // namespace fo
