// Which instance of the head norm's kernels a call takes, for one element type.
#pragma once

#include "head_norm.cuh"
#include "launch.cuh"

namespace fo {

template <class T, int V, int I, int TENSORS>
cudaError_t head_go(void (*kernel)(HeadParams), const HeadParams &p, int grid, cudaStream_t st, OncePerGpu &once)
{
    // the ring; in its place at the end the gradient's sums, a line for every group of lanes
    constexpr size_t lines = TENSORS == 2 ? (size_t)kHeadWarps * 64 * I * V * sizeof(Acc<T>) : 0, ring = HeadRing<T, V, I, TENSORS>::kBytes;
    constexpr size_t bytes = ring > lines ? ring : lines;
    if (bytes + (FO_HEAD_MAX_DIM + 16) * sizeof(double) > 48 * 1024) {        // with the weights
        const cudaError_t e = once.allow(kernel, bytes);
        if (e != cudaSuccess) return e;
    }
    return launch_beside(kernel, dim3((unsigned)grid), kHeadCta, st, bytes, p);
}

template <class T, int V, int I, int PAIRING>
cudaError_t head_launch(const HeadParams &p, bool grad, bool bias, int grid, cudaStream_t st)
{
    static OncePerGpu once[3];
    if (!grad) return head_go<T, V, I, 1>(head_norm_kernel<T, V, I, PAIRING>, p, grid, st, once[0]);
    if (bias) return head_go<T, V, I, 2>(head_norm_grad_kernel<T, V, I, PAIRING, true>, p, grid, st, once[1]);
    return head_go<T, V, I, 2>(head_norm_grad_kernel<T, V, I, PAIRING, false>, p, grid, st, once[2]);
}

template <class T, int V, int I>
cudaError_t head_paired(const HeadParams &p, int pairing, bool grad, bool bias, int grid, cudaStream_t st)
{
    return pairing == FO_PAIR_HALVES ? head_launch<T, V, I, FO_PAIR_HALVES>(p, grad, bias, grid, st)
                                     : head_launch<T, V, I, FO_PAIR_NEIGHBOURS>(p, grad, bias, grid, st);
}

// A vector is 32 lanes times I items at most; head_lanes() (head_norm.cu) has chosen the lanes for the same I.
template <class T>
cudaError_t launch_head_norm(const HeadParams &p, int piece, int pairing, bool grad, bool bias, int grid, cudaStream_t st)
{
    constexpr int kWhole = 16 / (int)sizeof(T);
    if (piece == kWhole) {
        if (p.dim <= 64 * kWhole) return head_paired<T, kWhole, 1>(p, pairing, grad, bias, grid, st);
        if constexpr (sizeof(T) >= 4) return head_paired<T, kWhole, (int)sizeof(T) / 2>(p, pairing, grad, bias, grid, st);
    }
    if constexpr (sizeof(T) == 2)
        if (piece == 4) return head_paired<T, 4, 1>(p, pairing, grad, bias, grid, st);
    if (p.dim <= 128) return head_paired<T, 1, 2>(p, pairing, grad, bias, grid, st);
    return head_paired<T, 1, 8>(p, pairing, grad, bias, grid, st);
}

}  // namespace fo
