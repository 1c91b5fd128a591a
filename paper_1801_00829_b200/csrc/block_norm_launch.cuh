// Which kernel shape a row length takes, per pair of element types.  Every pair is compiled in a
// file of its own (block_norm_*.cu).
#pragma once

#include "block_norm.cuh"

namespace fo {

template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st);
template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, int max_lines, int *lines, cudaStream_t st);   // of partial sums

// Calls go(T, C, E, threads) with the shape for `cols` columns in pieces of V: T threads of a warp and CTAs of
// kGroupCta, or (T = 0) C CTAs of `threads` a row; 16 elements a thread where a row has them.  A sum over the
// group costs every thread about 25 instructions, which 16 elements share; 16 is also what 64
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

// The same for the gradient, go(T, C, threads): 8 elements a thread, for more threads (32768 x 1024 mixed 153 us, with
// 16 elements and half the threads 165; 8192 x 5120 252 us, with 16 290; only rows that fill clusters of 4 or 8 CTAs
// would be faster with 16).
template <int V, class Go>
cudaError_t with_grad_shape(int cols, Go go)
{
#define FO_SHAPE(t, c, n) go(std::integral_constant<int, t>(), std::integral_constant<int, c>(), n)
    if (cols <= 64) return FO_SHAPE(8, 1, kGroupCta);
    if (cols <= 128) return FO_SHAPE(16, 1, kGroupCta);
    if (cols <= 256) return FO_SHAPE(32, 1, kGroupCta);
    const int c = cols <= 4096 ? 1 : cols <= 8192 ? 2 : cols <= 16384 ? 4 : 8;
    const int pieces = (cols + V - 1) / V, per_cta = kGradE / V * c;
    const int threads = ((pieces + per_cta - 1) / per_cta + 31) / 32 * 32;
    if (c == 1) return FO_SHAPE(0, 1, threads);
    if (c == 2) return FO_SHAPE(0, 2, threads);
    if (c == 4) return FO_SHAPE(0, 4, threads);
    return FO_SHAPE(0, 8, threads);
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
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // the kernels wait for the one before them themselves
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

template <class TS, class TB>
cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t st)
{
    return with_row_shape<16 / (int)sizeof(TB)>(p.cols, [&](auto tc, auto cc, auto ec, int cta) -> cudaError_t {
        constexpr int T = decltype(tc)::value, C = decltype(cc)::value, E = decltype(ec)::value;
        constexpr int kGroups = T > 0 ? kGroupCta / kDivisor<T> : 1;
        const long long grid = (p.rows + kGroups - 1) / kGroups * C;
        auto go = [&](auto aligned, auto blk, auto gate, auto lean) {
            return launch_rows(block_norm_kernel<TS, TB, T, C, E, decltype(aligned)::value, decltype(blk)::value,
                                                 decltype(gate)::value, decltype(lean)::value>, p, grid, cta, C, 0, st);
        };
        auto with_gate = [&](auto aligned, auto lean) -> cudaError_t {
            if (p.gate_access < 0) return go(aligned, std::true_type(), std::integral_constant<int, kNoGate>(), lean);
            if (p.gate_access == FO_AT_CELL)
                return go(aligned, std::true_type(), std::integral_constant<int, kCellGate>(), lean);
            return go(aligned, std::true_type(), std::integral_constant<int, kSharedGate>(), lean);
        };
        const auto none = std::integral_constant<int, kNoGate>();
        const bool lean_pre = p.aligned && p.x && p.y && p.pre.kind == FO_NORM_RMS && p.pre.weight && !p.pre.bias;
        if (!p.f) {
            if (lean_pre && !p.h) return go(std::true_type(), std::false_type(), none, std::true_type());
            return p.aligned ? go(std::true_type(), std::false_type(), none, std::false_type())
                             : go(std::false_type(), std::false_type(), none, std::false_type());
        }
        if (lean_pre && p.h && p.post.kind == FO_NORM_RMS && p.post.weight && !p.post.bias)
            return with_gate(std::true_type(), std::true_type());
        return p.aligned ? with_gate(std::true_type(), std::false_type()) : with_gate(std::false_type(), std::false_type());
    });
}

// Resident CTAs of a gradient kernel with `sums` column sums in shared memory.  Asked once per device and size of CTA.
template <void (*KERNEL)(BlockNormGradParams)>
cudaError_t grad_residency(int cta, int sums, size_t sum_bytes, int *per_sm)
{
    static short cache[16][kMostCta / 32 + 1][kGradSlots + 1];       // the same whoever asks first
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    short &known = cache[dev & 15][cta / 32][sums];
    if (known == 0) {
        int found = 0;
        constexpr int kMost = kGradSlots * kMostCta * kGradE * 8;    // of float64: 192 KB
        e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&found, KERNEL, cta, sums * sum_bytes);
        if (e != cudaSuccess) return e;
        known = (short)(found > 0 ? found : 1);
    }
    *per_sm = known;
    return cudaSuccess;
}

template <class TS, class TB>
cudaError_t launch_block_norm_grad(BlockNormGradParams p, int max_lines, int *lines, cudaStream_t st)
{
    return with_grad_shape<16 / (int)sizeof(TB)>(p.cols, [&](auto tc, auto cc, int cta) -> cudaError_t {
        constexpr int T = decltype(tc)::value, C = decltype(cc)::value;
        constexpr int kGroups = T > 0 ? kGroupCta / kDivisor<T> : 1;
        auto go = [&](auto aligned, auto blk, auto gate, auto lean) -> cudaError_t {
            constexpr auto kern = block_norm_grad_kernel<TS, TB, T, C, decltype(aligned)::value, decltype(blk)::value,
                                                         decltype(gate)::value, decltype(lean)::value>;
            // as many groups as a CTA holds, while there are rows for them on every SM
            const int sms = sm_count();
            int groups = kGroups, threads = cta;
            if (T == 0 && C == 1) {
                const long long each = (p.rows + sms - 1) / (sms > 0 ? sms : 1);
                groups = kMostCta / cta;
                if (groups > each) groups = (int)each;
                threads = groups * cta;
            }
            p.group = cta;
            const size_t sum_bytes = (size_t)threads * kGradE * sizeof(Acc<TB>);
            const int n = __builtin_popcount(p.slots);
            int per_sm = 0;
            const cudaError_t e = grad_residency<kern>(threads, n, sum_bytes, &per_sm);
            if (e != cudaSuccess) return e;
            long long count = (long long)sms * per_sm / C;
            const long long turns = (p.rows + groups - 1) / groups;
            if (count > turns) count = turns;
            if (count > max_lines) count = max_lines;
            if (count < 1) count = 1;
            *lines = (int)count;
            return launch_rows(kern, p, count * C, threads, C, n * sum_bytes, st);
        };
        auto with_gate = [&](auto aligned, auto lean) -> cudaError_t {
            if (p.gate_access < 0) return go(aligned, std::true_type(), std::integral_constant<int, kNoGate>(), lean);
            if (p.gate_access == FO_AT_CELL)
                return go(aligned, std::true_type(), std::integral_constant<int, kCellGate>(), lean);
            return go(aligned, std::true_type(), std::integral_constant<int, kSharedGate>(), std::false_type());
        };
        const auto none = std::integral_constant<int, kNoGate>();
        const bool lean_pre = p.aligned && p.dy && p.dx && p.pre.kind == FO_NORM_RMS && p.pre.weight;
        if (!p.f) {
            if (lean_pre && p.slots == (1u << kPreW)) return go(std::true_type(), std::false_type(), none, std::true_type());
            return p.aligned ? go(std::true_type(), std::false_type(), none, std::false_type())
                             : go(std::false_type(), std::false_type(), none, std::false_type());
        }
        const bool lean = lean_pre && p.df && p.post.kind == FO_NORM_RMS && p.post.weight && !p.post.bias
                          && (p.slots & ~(1u << kColScale)) == ((1u << kPreW) | (1u << kPostW));
        if (lean) return with_gate(std::true_type(), std::true_type());
        return p.aligned ? with_gate(std::true_type(), std::false_type()) : with_gate(std::false_type(), std::false_type());
    });
}
#endif

}  // namespace fo
