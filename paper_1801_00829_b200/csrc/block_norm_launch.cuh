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

// Calls go(T, C, E, threads) with the shape for `cols` columns in pieces of V: T threads of a warp and CTAs of
// kGroupCta, or (T = 0) C CTAs of `threads` a row; 16 elements a thread where a row has them.  A sum over the
// group costs every thread about 25 instructions, which 16 elements share; 16 is also what 64 (the gradient: 128)
// registers hold of a row's matrices.  Beyond 512 threads a row takes a cluster: CTAs of 1024 threads would
// have 64 registers a thread, and spill.
template <int V, class Go>
cudaError_t with_row_shape(int cols, Go go)
{
#define FO_SHAPE(t, c, e, n) \
    go(std::integral_constant<int, t>(), std::integral_constant<int, c>(), std::integral_constant<int, e>(), n)
    if (cols <= 64) return FO_SHAPE(8, 1, 8, kGroupCta);
    if (cols <= 128) return FO_SHAPE(8, 1, 16, kGroupCta);
    if (cols <= 256) return FO_SHAPE(16, 1, 16, kGroupCta);
    if (cols <= 512) return FO_SHAPE(32, 1, 16, kGroupCta);
    const int c = cols <= 8192 ? 1 : cols <= 16384 ? 2 : 4, pieces = (cols + V - 1) / V;
    const int per_cta = 16 / V * c, threads = ((pieces + per_cta - 1) / per_cta + 31) / 32 * 32;
    if (c == 1) return FO_SHAPE(0, 1, 16, threads);
    if (c == 2) return FO_SHAPE(0, 2, 16, threads);
    return FO_SHAPE(0, 4, 16, threads);
#undef FO_SHAPE
}

// The same for the gradient: 8 elements a thread, for more threads (32768 x 1024 mixed 153 us, with 16 elements 165;
// 8192 x 5120 252 us, with 16 290).  Beyond 8192 columns that takes clusters of 4 and 8, and 16 elements are better
// where half as many threads nearly fill an SM's 512 (16384 columns: 236 us, with 8 374; 20000: 577, with 8 417).
template <int V, class Go>
cudaError_t with_grad_shape(int cols, Go go)
{
#define FO_SHAPE(t, c, e, n) \
    go(std::integral_constant<int, t>(), std::integral_constant<int, c>(), std::integral_constant<int, e>(), n)
    if (cols <= 64) return FO_SHAPE(8, 1, 8, kGroupCta);
    if (cols <= 128) return FO_SHAPE(16, 1, 8, kGroupCta);
    if (cols <= 256) return FO_SHAPE(32, 1, 8, kGroupCta);
    const int pieces = (cols + V - 1) / V;
    auto threads = [&](int c, int e) { return ((pieces + e / V * c - 1) / (e / V * c) + 31) / 32 * 32; };
    if (cols <= 4096) return FO_SHAPE(0, 1, 8, threads(1, 8));
    if (cols <= 8192) return FO_SHAPE(0, 2, 8, threads(2, 8));
    if (cols <= 16384) {
        if (threads(2, 16) >= 448) return FO_SHAPE(0, 2, 16, threads(2, 16));
        return FO_SHAPE(0, 4, 8, threads(4, 8));
    }
    if (threads(4, 16) >= 448) return FO_SHAPE(0, 4, 16, threads(4, 16));
    return FO_SHAPE(0, 8, 8, threads(8, 8));
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
    return with_row_shape<16 / (int)sizeof(TB)>(p.cols, [&](auto tc, auto cc, auto ec, int cta) -> cudaError_t {
        constexpr int T = decltype(tc)::value, C = decltype(cc)::value, E = decltype(ec)::value;
        constexpr int kGroups = T > 0 ? kGroupCta / kDivisor<T> : 1;
        const long long grid = (p.rows + kGroups - 1) / kGroups * C;
        auto go = [&](auto aligned) {
            constexpr bool ALIGNED = decltype(aligned)::value;
            return p.f ? launch_rows(block_norm_kernel<TS, TB, T, C, E, ALIGNED, true>, p, grid, cta, C, 0, st)
                       : launch_rows(block_norm_kernel<TS, TB, T, C, E, ALIGNED, false>, p, grid, cta, C, 0, st);
        };
        return p.aligned ? go(std::true_type()) : go(std::false_type());
    });
}

// Resident CTAs of a gradient kernel with `sums` column sums in shared memory, 0: they do not fit.  Asked once per
// device and size of CTA.
template <void (*KERNEL)(BlockNormGradParams)>
cudaError_t grad_residency(int cta, int sums, size_t sum_bytes, int *per_sm)
{
    constexpr size_t kRoom = 200 * 1024;
    static short cache[16][kMostCta / 32 + 1][kGradSlots + 1];       // + 1; the same whoever asks first
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    short &known = cache[dev & 15][cta / 32][sums];
    if (known == 0) {
        int found = 0;
        if (sums * sum_bytes <= kRoom) {
            e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRoom);
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&found, KERNEL, cta, sums * sum_bytes);
            if (e != cudaSuccess) return e;
        }
        known = (short)(found + 1);
    }
    *per_sm = known - 1;
    return cudaSuccess;
}

template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, GradSpace *space, cudaStream_t st)
{
    return with_grad_shape<16 / (int)sizeof(TB)>(p.cols, [&](auto tc, auto cc, auto ec, int cta) -> cudaError_t {
        constexpr int T = decltype(tc)::value, C = decltype(cc)::value, E = decltype(ec)::value;
        constexpr int kGroups = T > 0 ? kGroupCta / kDivisor<T> : 1;
        auto go = [&](auto aligned, auto blk, auto form) -> cudaError_t {
            constexpr auto kern = block_norm_grad_kernel<TS, TB, T, C, E, decltype(aligned)::value, decltype(blk)::value,
                                                         decltype(form)::value>;
            // as many groups as 512 threads hold, while there are rows for them on every SM
            const int sms = sm_count();
            int groups = kGroups, threads = cta;
            if (T == 0 && C == 1) {
                const long long each = (p.rows + sms - 1) / (sms > 0 ? sms : 1);
                groups = kMostCta / cta;
                if (groups > each) groups = (int)each;
                threads = groups * cta;
            }
            p.group = cta;
            const size_t sum_bytes = (size_t)threads * E * sizeof(Acc<TB>);
            const int n = __builtin_popcount(p.slots);
            int per_sm = 0;
            const cudaError_t e = grad_residency<kern>(threads, n, sum_bytes, &per_sm);
            if (e != cudaSuccess) return e;
            p.sums = per_sm > 0 ? nullptr : space->sums;
            long long lines = (long long)sms * (per_sm > 0 ? per_sm : 1) / C;
            const long long turns = (p.rows + groups - 1) / groups;
            if (lines > turns) lines = turns;
            if (lines > space->max_lines) lines = space->max_lines;
            if (lines < 1) lines = 1;
            space->lines = (int)lines;
            return launch_rows(kern, p, lines * C, threads, C, per_sm > 0 ? n * sum_bytes : 0, st);
        };
        using Any = std::integral_constant<int, kGradAny>;
        using Lean = std::integral_constant<int, kGradLean>;
        using LeanGate = std::integral_constant<int, kGradLeanGate>;
        const bool pre = p.dy && p.dx && p.pre.kind == FO_NORM_RMS && p.pre.weight && (p.slots & (1u << kPreW));
        if (!p.f) {
            if (p.aligned && pre && p.slots == (1u << kPreW)) return go(std::true_type(), std::false_type(), Lean());
            return p.aligned ? go(std::true_type(), std::false_type(), Any()) : go(std::false_type(), std::false_type(), Any());
        }
        const unsigned both = (1u << kPreW) | (1u << kPostW);
        if (p.aligned && pre && p.df && p.post.kind == FO_NORM_RMS && p.post.weight && !p.post.bias
            && (p.slots & ~(1u << kColScale)) == both) {
            if (p.gate_access < 0) return go(std::true_type(), std::true_type(), Lean());
            if (p.gate_access == FO_AT_CELL) return go(std::true_type(), std::true_type(), LeanGate());
        }
        return p.aligned ? go(std::true_type(), std::true_type(), Any()) : go(std::false_type(), std::true_type(), Any());
    });
}
#endif

}  // namespace fo
