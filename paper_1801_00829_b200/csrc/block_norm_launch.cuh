// Which kernel shape a row length takes, per pair of element types.  Every pair is compiled in a
// file of its own (block_norm_*.cu).
#pragma once

#include "block_norm.cuh"

namespace fo {

// How the gradient's column sums are laid out in the workspace: at most `max_lines` lines of partial sums, and
// behind them `room` bytes for CTAs whose sums do not fit shared memory.
struct GradSpace {
    int max_lines, lines;                    // lines: written by the launch
    void *sums;
};

template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st);
template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, GradSpace *space, cudaStream_t st);

// Calls go(T, C, E) with the shape for `cols` columns: 16 elements a thread where a row has them.  A sum
// over the group costs every thread about 25 instructions, which 16 elements share; 16 is also what 64 to 80
// registers hold of a row's matrices.  Beyond 512 threads a row takes a cluster: CTAs of 1024 threads have
// 64 registers a thread, and spill.
template <class Go>
cudaError_t with_row_shape(int cols, Go go)
{
#define FO_SHAPE(t, c, e) \
    go(std::integral_constant<int, t>(), std::integral_constant<int, c>(), std::integral_constant<int, e>())
    if (cols <= 64) return FO_SHAPE(8, 1, 8);
    if (cols <= 128) return FO_SHAPE(8, 1, 16);
    if (cols <= 256) return FO_SHAPE(16, 1, 16);
    if (cols <= 512) return FO_SHAPE(32, 1, 16);
    if (cols <= 1024) return FO_SHAPE(64, 1, 16);
    if (cols <= 2048) return FO_SHAPE(128, 1, 16);
    if (cols <= 4096) return FO_SHAPE(256, 1, 16);
    if (cols <= 8192) return FO_SHAPE(512, 1, 16);
    if (cols <= 16384) return FO_SHAPE(512, 2, 16);
    return FO_SHAPE(512, 4, 16);
#undef FO_SHAPE
}

#ifdef FO_BLOCK_NORM_DEFINE
template <class Params>
cudaError_t launch_rows(void (*kern)(Params), const Params &p, long long grid, int cta, int cluster, size_t smem,
                        cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)cta);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st)
{
    return with_row_shape(p.cols, [&](auto tc, auto cc, auto ec) -> cudaError_t {
        constexpr int T = decltype(tc)::value, C = decltype(cc)::value, E = decltype(ec)::value;
        constexpr int kCta = T > 32 ? T : kGroupCta;
        const long long grid = (p.rows + kCta / T - 1) / (kCta / T) * C;
        auto go = [&](auto vec) {
            constexpr bool VEC = decltype(vec)::value;
            return p.f ? launch_rows(block_norm_kernel<TS, TB, T, C, E, VEC, true>, p, grid, kCta, C, 0, st)
                       : launch_rows(block_norm_kernel<TS, TB, T, C, E, VEC, false>, p, grid, kCta, C, 0, st);
        };
        return p.vec ? go(std::true_type()) : go(std::false_type());
    });
}

// What a kernel needs to be asked once per device.
struct GradKernelFacts {
    bool known;
    int per_sm[kGradSlots + 1];              // resident CTAs by number of sums in shared memory, 0: they do not fit
};

template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, GradSpace *space, cudaStream_t st)
{
    return with_row_shape(p.cols, [&](auto tc, auto cc, auto ec) -> cudaError_t {
        constexpr int T = decltype(tc)::value, C = decltype(cc)::value, E = decltype(ec)::value;
        constexpr int kCta = T > 32 ? T : kGroupCta;
        constexpr size_t kSum = (size_t)kCta * E * sizeof(Acc<TB>);
        auto go = [&](auto vec, auto blk) -> cudaError_t {
            const auto kern = block_norm_grad_kernel<TS, TB, T, C, E, decltype(vec)::value, decltype(blk)::value>;
            static GradKernelFacts facts[64];                // the same whoever asks first
            int dev = 0;
            cudaError_t e = cudaGetDevice(&dev);
            if (e != cudaSuccess) return e;
            GradKernelFacts &f = facts[dev & 63];
            if (!f.known) {
                constexpr int kFit = (int)((size_t)(220 * 1024) / kSum);
                constexpr int kMost = kFit < kGradSlots ? kFit : kGradSlots;
                e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kMost * kSum));
                for (int n = 0; n <= kGradSlots && e == cudaSuccess; ++n) {
                    f.per_sm[n] = 0;
                    if (n <= kMost) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&f.per_sm[n], kern, kCta, n * kSum);
                }
                if (e != cudaSuccess) return e;
                f.known = true;
            }
            const int n = __builtin_popcount(p.slots);
            const bool fits = f.per_sm[n] > 0;
            p.sums = fits ? nullptr : space->sums;
            long long lines = (long long)sm_count() * (fits ? f.per_sm[n] : 1) / C;
            const long long groups = (p.rows + kCta / T - 1) / (kCta / T);
            if (lines > groups) lines = groups;
            if (lines > space->max_lines) lines = space->max_lines;
            if (lines < 1) lines = 1;
            space->lines = (int)lines;
            return launch_rows(kern, p, lines * C, kCta, C, fits ? n * kSum : 0, st);
        };
        auto by_block = [&](auto vec) -> cudaError_t {
            return p.f ? go(vec, std::true_type()) : go(vec, std::false_type());
        };
        return p.vec ? by_block(std::true_type()) : by_block(std::false_type());
    });
}
#endif

}  // namespace fo
