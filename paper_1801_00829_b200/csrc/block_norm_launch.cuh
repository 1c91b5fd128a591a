// Which kernel shape a row length takes, per pair of element types.  Every pair is compiled in a
// file of its own (block_norm_*.cu).
#pragma once

#include "block_norm.cuh"

namespace fo {

template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st);
template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, int form, int max_ctas, int *ctas, cudaStream_t st);

// Calls go(T, E) with the shape for `cols` columns: 16 elements a thread where a row has them.  A sum
// over the group costs every thread about 25 instructions, which 16 elements share; 16 is also what 64 to 80
// registers hold of a row's matrices.
template <class Go>
cudaError_t with_row_shape(int cols, Go go)
{
#define FO_SHAPE(t, e) go(std::integral_constant<int, t>(), std::integral_constant<int, e>())
    if (cols <= 64) return FO_SHAPE(8, 8);
    if (cols <= 128) return FO_SHAPE(8, 16);
    if (cols <= 256) return FO_SHAPE(16, 16);
    if (cols <= 512) return FO_SHAPE(32, 16);
    if (cols <= 1024) return FO_SHAPE(64, 16);
    if (cols <= 2048) return FO_SHAPE(128, 16);
    if (cols <= 4096) return FO_SHAPE(256, 16);
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
        auto go = [&](auto vec) {
            constexpr bool VEC = decltype(vec)::value;
            if (p.f) block_norm_kernel<TS, TB, T, E, VEC, true><<<(unsigned)grid, kCta, 0, st>>>(p);
            else block_norm_kernel<TS, TB, T, E, VEC, false><<<(unsigned)grid, kCta, 0, st>>>(p);
        };
        if (p.vec) go(std::true_type());
        else go(std::false_type());
        return cudaGetLastError();
    });
}

template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, int form, int max_ctas, int *ctas, cudaStream_t st)
{
    return with_row_shape(p.cols, [&](auto tc, auto ec) -> cudaError_t {
        constexpr int T = decltype(tc)::value, E = decltype(ec)::value;
        constexpr int kCta = T > 32 ? T : kGroupCta;
        auto go = [&](auto vec, auto form_c) -> cudaError_t {
            const auto kern = block_norm_grad_kernel<TS, TB, T, E, decltype(vec)::value, decltype(form_c)::value>;
            static int per_sm[64] = {0};                     // of this kernel, per device; the same whoever asks first
            int dev = 0;
            cudaError_t e = cudaGetDevice(&dev);
            if (e != cudaSuccess) return e;
            int &n = per_sm[dev & 63];
            if (n == 0) {
                int found = 0;
                e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&found, kern, kCta, 0);
                if (e != cudaSuccess) return e;
                n = found > 0 ? found : 1;
            }
            long long grid = (p.rows + kCta / T - 1) / (kCta / T);
            const long long resident = (long long)sm_count() * n;
            if (grid > resident) grid = resident;
            if (grid > max_ctas) grid = max_ctas;
            *ctas = (int)grid;
            kern<<<(unsigned)grid, kCta, 0, st>>>(p);
            return cudaGetLastError();
        };
        auto by_form = [&](auto vec) -> cudaError_t {
            if (form == kGradStream) return go(vec, std::integral_constant<int, kGradStream>());
            if (form == kGradLean) return go(vec, std::integral_constant<int, kGradLean>());
            return go(vec, std::integral_constant<int, kGradAll>());
        };
        return p.vec ? by_form(std::true_type()) : by_form(std::false_type());
    });
}
#endif

}  // namespace fo
