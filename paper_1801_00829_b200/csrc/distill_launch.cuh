// How rows are spread over CTAs and clusters, for one element type.
#pragma once

#include "distill.cuh"
#include "launch.cuh"

namespace fo {

constexpr int kDistillMostBytes = 196640;                 // of a row in one CTA's shared memory

template <class T, bool STEP>
cudaError_t distill_row_launch(DistillParams p, cudaStream_t st)
{
    static OncePerGpu once;
    cudaError_t e = once.allow(distill_kernel<T, STEP>, kDistillMostBytes + kTeacherBytes * FO_DISTILL_MAX_TOP);
    if (e != cudaSuccess) return e;
    // a row may begin anywhere in its first piece
    const long long pieces = ((long long)p.vocab * (int)sizeof(T) + 15 - (int)sizeof(T)) / 16 + 1;
    int cluster = 1;
    while (cluster < 8 && (pieces + cluster - 1) / cluster > 32768 / 16) cluster *= 2;
    p.slice = (int)((pieces + cluster - 1) / cluster);
    const int threads = p.slice >= 512 ? kDistillCta : 128;
    return launch_beside(distill_kernel<T, STEP>, dim3((unsigned)(p.rows * cluster)), threads, st, (size_t)p.slice * 16 + (size_t)(p.top + 3) / 4 * 4 * kTeacherBytes, p, cluster);
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
    return launch_beside(distill_grad_kernel<T>, dim3((unsigned)p.rows, (unsigned)parts), kThreads, st, (size_t)(p.top + 3) / 4 * 4 * kTeacherBytes, p);
}

}  // namespace fo
