// How rows are spread over CTAs, for one element type.
#pragma once

#include "distill.cuh"
#include <algorithm>

#include "launch.cuh"

namespace fo {

template <class T, bool STEP>
cudaError_t distill_row_launch(DistillParams p, cudaStream_t st)
{
    static OncePerGpu once;
    constexpr size_t most = FO_DISTILL_MAX_VOCAB / 8 + 16 + kTeacherBytes * FO_DISTILL_MAX_TOP;
    const cudaError_t e = once.allow(distill_kernel<T, STEP>, most);
    if (e != cudaSuccess) return e;
    // the entries, and a bit for each of the row's places and those before it in its first piece
    const size_t shared = (size_t)(p.top + 3) / 4 * 4 * kTeacherBytes + (size_t)(p.vocab + 16 / (int)sizeof(T) - 1 + 127) / 128 * 16;
    // as many threads as have 32 pieces each, or more: what a row costs besides is hidden by other rows on the SM (16384 x 8192 in
    // bfloat16 with 8 pieces each 261 us, with 32 162).  Where every row has an SM of its own, as many as have 8
    const int pieces = (int)(((long long)p.vocab * (int)sizeof(T) + 15) / 16);
    const bool few = p.rows <= sm_count();
    p.team = 32, p.shared = (int)shared;
    while (p.team < (few ? kDistillRow : kDistillCta) && p.team * (few ? 8 : 32) < pieces) p.team *= 2;
    int teams = few ? 1 : kDistillCta / p.team;
    while (teams > 1 && teams * shared > 64 * 1024) teams /= 2;
    return launch_beside(distill_kernel<T, STEP>, dim3((unsigned)((p.rows + teams - 1) / teams)), p.team * teams, st, shared * teams, p);
}

template <class T>
cudaError_t launch_distill(DistillParams p, DistillWay way, cudaStream_t st)
{
    if (way == kDistillLoss) return distill_row_launch<T, false>(p, st);
    if (way == kDistillStep) return distill_row_launch<T, true>(p, st);
    const long long pieces = ((long long)p.vocab * (int)sizeof(T) + 15 - (int)sizeof(T)) / 16 + 1;
    // As many pieces a thread as pay for what a CTA does besides: 24 of short rows (16384 x 8192 in bfloat16 with four 154 us, with 24 102),
    // up to 32 of long ones (4096 x 128000: with eight 445 us, with 32 358); but of few rows so few, down to eight, that there are
    // CTAs for all SMs (8 x 128000: 7 us, with 32 13).
    int threads = 32;
    while (threads < kDistillCta && threads * 24 < pieces) threads *= 2;
    const long long least = (pieces + threads * 32 - 1) / (threads * 32), most = (pieces + threads * 8 - 1) / (threads * 8);
    const int parts = (int)std::max(least, std::min(most, (5LL * sm_count() + p.rows - 1) / p.rows));
    p.slice = (int)((pieces + parts - 1) / parts);
    return launch_beside(distill_grad_kernel<T>, dim3((unsigned)p.rows, (unsigned)parts), threads, st, (size_t)(p.top + 3) / 4 * 4 * kTeacherBytes, p);
}

}  // namespace fo
