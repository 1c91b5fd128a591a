// Which kernel shape a row length takes, per pair of element types.  Every pair is compiled in a
// file of its own (block_norm_*.cu).
#pragma once

#include "block_norm.cuh"

namespace fo {

template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st);
template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, int form, int max_ctas, int *ctas, cudaStream_t st);

// Calls go(T, E) with the shape for `cols` columns: as few threads as hold the row with 8 elements
// each, up to a CTA of 512; then 16 and 32 elements a thread.
template <class Go>
cudaError_t with_row_shape(int cols, Go go)
{
#define FO_SHAPE(t, e) go(std::integral_constant<int, t>(), std::integral_constant<int, e>())
    if (cols <= 64) return FO_SHAPE(8, 8);
    if (cols <= 128) return FO_SHAPE(16, 8);
    if (cols <= 256) return FO_SHAPE(32, 8);
    if (cols <= 512) return FO_SHAPE(32, 16);
    if (cols <= 1024) return FO_SHAPE(128, 8);
    if (cols <= 2048) return FO_SHAPE(256, 8);
    if (cols <= 4096) return FO_SHAPE(512, 8);
    if (cols <= 8192) return FO_SHAPE(512, 16);
    if (cols <= 16384) return FO_SHAPE(1024, 16);
    return FO_SHAPE(1024, 32);
#undef FO_SHAPE
}

#ifdef FO_BLOCK_NORM_DEFINE
template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st)
{
    return with_row_shape(p.cols, [&](auto tc, auto ec) -> cudaError_t {
        constexpr int T = decltype(tc)::value, E = decltype(ec)::value;
        constexpr int kCta = T > 32 ? T : kGroupCta;
        const long long grid = (p.rows + kCta / T - 1) / (kCta / T);
        if (p.f) block_norm_kernel<TS, TB, T, E, true><<<(unsigned)grid, kCta, 0, st>>>(p);
        else block_norm_kernel<TS, TB, T, E, false><<<(unsigned)grid, kCta, 0, st>>>(p);
        return cudaGetLastError();
    });
}

template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, int form, int max_ctas, int *ctas, cudaStream_t st)
{
    return with_row_shape(p.cols, [&](auto tc, auto ec) -> cudaError_t {
        constexpr int T = decltype(tc)::value, E = decltype(ec)::value;
        constexpr int kCta = T > 32 ? T : kGroupCta;
        auto go = [&](auto kern) -> cudaError_t {
            int per_sm = 0;
            cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, kCta, 0);
            if (e != cudaSuccess) return e;
            long long grid = (p.rows + kCta / T - 1) / (kCta / T);
            const long long resident = (long long)sm_count() * (per_sm > 0 ? per_sm : 1);
            if (grid > resident) grid = resident;
            if (grid > max_ctas) grid = max_ctas;
            *ctas = (int)grid;
            kern<<<(unsigned)grid, kCta, 0, st>>>(p);
            return cudaGetLastError();
        };
        if (form == kGradStream) return go(block_norm_grad_kernel<TS, TB, T, E, kGradStream>);
        if (form == kGradLean) return go(block_norm_grad_kernel<TS, TB, T, E, kGradLean>);
        return go(block_norm_grad_kernel<TS, TB, T, E, kGradAll>);
    });
}
#endif

}  // namespace fo
