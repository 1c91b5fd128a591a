// The distillation loss from a teacher's top logits and its gradient.
//
// Loss, or loss and gradient at once: a row of logits belongs to a cluster of 1 to 8 CTAs, whose shared memory holds it while the
// sums are made and the gradient is written, so that it is read once.  The row lies there as it does in memory, at the same
// offset from a 16-byte boundary, so that rows that begin anywhere move in whole 16-byte pieces but for their ends.  The entries' logits are
// taken out of the row (and replaced by minus infinity) before the sum is made: what the teacher's entries leave is then added up by itself, not as
// 1 minus their sum, and the entries, which hold most of the probability, are summed in 64 bits.
// The gradient alone is elementwise from the saved statistics, a CTA to a part of a row.
#pragma once

#include <math_constants.h>

#include "elem.cuh"
#include "../../include/fusedops_lm.h"

namespace fo {

constexpr int kDistillCta = 256;

struct DistillParams {
    long long rows;
    int vocab, top;
    int ids_long, wide_values;
    int slice;                          // pieces of a CTA
    long long ld_logits, ld_ids, ld_values, ld_dz;
    const void *logits, *ids, *values, *tail, *dloss;
    void *loss, *stats, *dz;
    double inv_t;
};

// exp(v): of v in units of log 2 for 16-bit logits by the hardware's exponential (relative error 2^-22), else by CUDA's function
template <class T> __device__ __forceinline__ float distill_exp(float v)
{
    if constexpr (sizeof(T) == 2) {
        float r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
        return r;
    } else return expf(v);
}
template <class T> __device__ __forceinline__ double distill_exp(double v) { return exp(v); }
template <class T>
__device__ __forceinline__ Acc<T> distill_unit(double inv_t)
{
    return Acc<T>(sizeof(T) == 2 ? inv_t * 1.4426950408889634074 : inv_t);
}
template <class A> __device__ __forceinline__ A distill_floor() { return -A(CUDART_INF); }

__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }

__device__ __forceinline__ double distill_warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double distill_warp_max(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// Sums s relative to maxima m, added up over each half of a warp (the rests', and the entries'): relative to each half's maximum,
// which m becomes.
__device__ __forceinline__ double distill_halves(double &m, double s, double inv_t)
{
    const double own = m;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (s != 0.0) s *= exp((own - m) * inv_t);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// The teacher's entries of one row, in shared memory.
struct Teacher {
    int *id;                            // -1: no entry; padded to a multiple of 4
    double *p, *share, *z;              // shares, those of a place, and the student's logits
    int *place;                         // of an entry that is the first of its place; -1
};

constexpr int kTeacherBytes = 32;       // of an entry in shared memory
__device__ __forceinline__ Teacher teacher_at(void *memory, int top)
{
    const int room = (top + 3) / 4 * 4;
    Teacher t;
    t.p = static_cast<double *>(memory), t.share = t.p + room, t.z = t.share + room;
    t.id = reinterpret_cast<int *>(t.z + room), t.place = t.id + room;
    return t;
}

template <class T>
__device__ __forceinline__ double teacher_value(const DistillParams &p, long long row, int k)
{
    const long long at = row * p.ld_values + k;
    const double v = p.wide_values ? (double)static_cast<const float *>(p.values)[at] : (double)widen(static_cast<const T *>(p.values)[at]);
    return v * p.inv_t;
}

// What all threads need to know of the entries besides the arrays.
struct TeacherSums {
    double top_max, log_sum;            // log p = v / temperature - top_max - log_sum
    double sum, rest;                   // of p, and P
};
// The first warp's part: ids, shares and their sums.  An id that is no place of the row makes the sum NaN, and with it everything.
template <class T>
__device__ __forceinline__ void teacher_shares(const DistillParams &p, long long row, const Teacher &t, TeacherSums &out)
{
    const int lane = threadIdx.x & 31;
    double most = -CUDART_INF, sum = 0.0;
    bool bad = false;
    for (int k = lane; k < p.top; k += 32) {
        const long long at = row * p.ld_ids + k;
        const long long id = p.ids_long ? static_cast<const long long *>(p.ids)[at] : static_cast<const int *>(p.ids)[at];
        const double v = teacher_value<T>(p, row, k);
        t.id[k] = id < 0 || id >= p.vocab ? -1 : (int)id;
        t.z[k] = v;
        bad = bad || id >= p.vocab;
        if (id >= 0) most = fmax(most, v);
    }
    if (lane < ((4 - p.top % 4) & 3)) t.id[p.top + lane] = -1;
    const double reference = p.tail ? (double)static_cast<const Acc<T> *>(p.tail)[row] : distill_warp_max(most);
    for (int k = lane; k < p.top; k += 32) {
        const double e = t.id[k] >= 0 ? exp(t.z[k] - reference) : 0.0;
        t.p[k] = e, sum += e;
    }
    sum = distill_warp_sum(bad ? CUDART_NAN : sum);
    TeacherSums s = {reference, 0.0, sum, 0.0};
    if (p.tail) {
        s.rest = sum < 1.0 ? 1.0 - sum : sum >= 1.0 ? 0.0 : sum;
    } else if (sum != 0.0) {                              // 0: no entries
        const double inverse = 1.0 / sum;
        for (int k = lane; k < p.top; k += 32) t.p[k] *= inverse;
        s.log_sum = log(sum), s.sum = sum * inverse;
    }
    if (lane == 0) out = s;
}
// Of entries with the same place the first one takes the shares of all, the others have no place.
__device__ __forceinline__ void teacher_places(const Teacher &t, int top)
{
    for (int k = threadIdx.x; k < top; k += blockDim.x) {
        const int id = t.id[k];
        t.share[k] = t.p[k], t.place[k] = id;
        if (id < 0) continue;
        int same = 0, first = k;
        const int4 *const four = reinterpret_cast<const int4 *>(t.id);
#pragma unroll 4
        for (int j = 0; j < (top + 3) / 4; ++j) {
            const int4 v = four[j];
            const int hits = (v.x == id) | (v.y == id) << 1 | (v.z == id) << 2 | (v.w == id) << 3;
            same += __popc(hits);
            if (hits) first = min(first, 4 * j + __ffs(hits) - 1);
        }
        if (same == 1) continue;
        if (first != k) {
            t.place[k] = -1;
            continue;
        }
        double all = 0.0;
        for (int j = 0; j < top; ++j)
            if (t.id[j] == id) all += t.p[j];
        t.share[k] = all;
    }
}

// Where a row lies: pieces of 16 bytes from the boundary before its first element.
template <class T>
struct RowPieces {
    static constexpr int E = 16 / (int)sizeof(T);
    int skip;                           // elements of the first piece that are not the row's
    int pieces, end;                    // end: skip + the row's elements
    __device__ __forceinline__ RowPieces(const T *row, int vocab)
        : skip((int)(((uintptr_t)row & 15u) / sizeof(T))), pieces((skip + vocab + E - 1) / E), end(skip + vocab)
    {
    }
    __device__ __forceinline__ bool whole(int i) const { return i * E >= skip && (i + 1) * E <= end; }
    __device__ __forceinline__ bool holds(int e) const { return e >= skip && e < end; }
};

template <class T>
__device__ __forceinline__ void distill_zero(T *dz, int vocab, int first, int count)
{
    const RowPieces<T> out(dz, vocab);
    T *const base = dz - out.skip;
    const uint32_t none[4] = {0, 0, 0, 0};
    for (int i = first + threadIdx.x; i < min(first + count, out.pieces); i += blockDim.x) {
        if (out.whole(i)) store16(base + i * RowPieces<T>::E, none);
        else
            for (int e = i * RowPieces<T>::E; e < (i + 1) * RowPieces<T>::E; ++e)
                if (out.holds(e)) base[e] = narrow<T>(Acc<T>(0));
    }
}

// A piece of the gradient: whole where both rows lie alike, else element by element.
template <class T>
__device__ __forceinline__ void distill_put(const RowPieces<T> &at, int i, T *dz, bool alike, const Packed<T, 16 / sizeof(T)> &v)
{
    constexpr int E = 16 / (int)sizeof(T);
    T *const base = dz - at.skip;
    if (alike && at.whole(i)) {
        store16(base + i * E, v.w);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at.holds(i * E + e)) base[i * E + e] = v.raw(e);
    }
}

// The largest value of a piece and `most`; a NaN is passed over (the sum finds it).
template <class T>
__device__ __forceinline__ Acc<T> distill_largest(const Packed<T, 16 / sizeof(T)> &v, Acc<T> most)
{
    if constexpr (std::is_same<T, __nv_bfloat16>::value || std::is_same<T, __half>::value) {
        using Pair = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        const Pair *const w = reinterpret_cast<const Pair *>(v.w);
        const Pair m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
        return larger(most, larger(widen(m.x), widen(m.y)));
    } else {
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) most = larger(most, v.get(e));
        return most;
    }
}

// What the CTAs of a cluster tell each other.
struct DistillPart {
    double rest_max, rest_sum, top_max, top_sum, entries;
};

template <class T, bool STEP>
__global__ void __launch_bounds__(kDistillCta, sizeof(T) == 8 ? 2 : 5) distill_kernel(const __grid_constant__ DistillParams p)
{
    using A = Acc<T>;
    constexpr int E = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char distill_memory[];
    __shared__ DistillPart warp_parts[kDistillCta / 32], parts[8];
    __shared__ double result[3];
    __shared__ TeacherSums teacher;
    unsigned rank, cluster;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
    if (cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    wait_for_earlier();
    const long long row = blockIdx.x / cluster;
    const T *z = static_cast<const T *>(p.logits) + row * p.ld_logits;
    T *dz = STEP ? static_cast<T *>(p.dz) + row * p.ld_dz : nullptr;
    const int first_piece = (int)rank * p.slice;
    A weight = A(1);
    if (STEP) {
        if (p.dloss) weight = static_cast<const A *>(p.dloss)[row];
        if (weight == A(0)) {                                 // the row is not looked at
            if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            // one piece more than the logits' can be the gradient's, at another offset: the last CTA has it
            distill_zero(dz, p.vocab, first_piece, rank + 1 == cluster ? p.slice + 1 : p.slice);
            if (rank == 0 && threadIdx.x == 0) static_cast<A *>(p.loss)[row] = A(0);
            return;
        }
    }
    const RowPieces<T> at(z, p.vocab);
    const int count = max(0, min(p.slice, at.pieces - first_piece));
    T *const held = reinterpret_cast<T *>(distill_memory);
    const Teacher t = teacher_at(distill_memory + (size_t)p.slice * 16, p.top);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const T *const base = z - at.skip;
    // whole pieces of this CTA's part: [begin, stop); of the others there is at most one at each end
    const int begin = max(0, (at.skip ? 1 : 0) - first_piece), stop = max(begin, min(count, at.end / E - first_piece));
    {
        unsigned to = (unsigned)__cvta_generic_to_shared(held) + (begin + threadIdx.x) * 16;
        const T *source = base + (long long)(first_piece + begin + threadIdx.x) * E;
        for (int i = begin + threadIdx.x; i < stop; i += blockDim.x, to += blockDim.x * 16, source += blockDim.x * E)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(source) : "memory");
        for (int i = threadIdx.x < 2 ? (threadIdx.x ? stop : 0) : count; i < count && (i < begin || i >= stop); i += count)
            for (int e = 0; e < E; ++e) {
                const int j = (first_piece + i) * E + e;
                held[i * E + e] = at.holds(j) ? base[j] : narrow<T>(distill_floor<A>());
            }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (warp == 0) teacher_shares<T>(p, row, t, teacher);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();

    // the entries in this CTA's part are taken out of the row
    const int from = first_piece * E - at.skip, to = from + count * E;      // elements of the row
    const auto here = [&](int place) { return place >= 0 && place >= from && place < to; };
    const bool with_entries = warp * 32 < p.top;
    double entries = 0.0, top_max = -CUDART_INF, top_sum = 0.0;
    teacher_places(t, p.top);
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (here(t.id[k])) {
            const double v = (double)widen(held[t.id[k] - from]), share = t.p[k];
            if (share != 0.0) entries += share * (t.z[k] - teacher.top_max - teacher.log_sum - v * p.inv_t);
            t.z[k] = v, top_max = fmax(top_max, v);
        }
    __syncthreads();                                          // all of them have been read
    if (with_entries) {
        top_max = distill_warp_max(top_max), entries = distill_warp_sum(entries);
        for (int k = threadIdx.x; k < p.top; k += blockDim.x)
            if (here(t.place[k])) {
                held[t.place[k] - from] = narrow<T>(distill_floor<A>());
                top_sum += exp((t.z[k] - top_max) * p.inv_t);
            }
        top_sum = distill_warp_sum(top_sum);
    }
    __syncthreads();

    // all the rest: every thread keeps the largest so far and the sum relative to it
    const A unit = distill_unit<T>(p.inv_t);
    A largest = distill_floor<A>(), sum = A(0);
    const Two<A> scale = both(unit);
    auto take = [&](auto many, const uint4 *from16, int step) {
        constexpr int M = many.value;
        Packed<T, E> v[M];
        A top = largest;
#pragma unroll
        for (int u = 0; u < M; ++u) {
            const uint4 w = from16[u * step];
            v[u].w[0] = w.x, v[u].w[1] = w.y, v[u].w[2] = w.z, v[u].w[3] = w.w;
            top = distill_largest<T>(v[u], top);
        }
        const A ref = top == distill_floor<A>() ? A(0) : top;
        Two<A> more = both(A(0));
        const Two<A> less = both(-ref);
#pragma unroll
        for (int u = 0; u < M; ++u)
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const Two<A> x = (v[u].get2(e) + less) * scale;
                more = more + two(distill_exp<T>(first(x)), distill_exp<T>(second(x)));
            }
        sum = fused_ma(sum, distill_exp<T>((largest - ref) * unit), joined(more));
        largest = top;
    };
    {
        const int step = blockDim.x;
        const uint4 *from16 = reinterpret_cast<const uint4 *>(held) + threadIdx.x;
        int i = threadIdx.x;
        for (; i + 3 * step < count; i += 4 * step, from16 += 4 * step) take(std::integral_constant<int, 4>(), from16, step);
        for (; i < count; i += step, from16 += step) take(std::integral_constant<int, 1>(), from16, step);
    }
    // the warp's, the CTA's
    A rest_max = largest;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) rest_max = larger(rest_max, __shfl_xor_sync(0xffffffffu, rest_max, o));
    A rest_sum = sum == A(0) ? A(0) : sum * distill_exp<T>((largest - rest_max) * unit);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) rest_sum += __shfl_xor_sync(0xffffffffu, rest_sum, o);
    if (lane == 0) warp_parts[warp] = {(double)rest_max, (double)rest_sum, top_max, top_sum, entries};
    __syncthreads();
    if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // every CTA has started
    const int half = lane & 15;
    if (warp == 0) {
        double m = -CUDART_INF, s = 0.0, en = 0.0;
        if (half < warps) {
            const DistillPart d = warp_parts[half];
            m = lane < 16 ? d.rest_max : d.top_max, s = lane < 16 ? d.rest_sum : d.top_sum, en = d.entries;
        }
        s = distill_halves(m, s, p.inv_t);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) en += __shfl_xor_sync(0xffffffffu, en, o);
        // lanes k and 16 + k tell CTA k
        if (cluster == 1) {
            if (lane == 0) parts[0].rest_max = m, parts[0].rest_sum = s, parts[0].entries = en;
            if (lane == 16) parts[0].top_max = m, parts[0].top_sum = s;
        } else if (half < (int)cluster) {
            unsigned to_peer;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to_peer) : "r"((unsigned)__cvta_generic_to_shared(&parts[rank])), "r"(half));
            to_peer += lane < 16 ? 0 : 16;
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to_peer), "d"(m) : "memory");
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to_peer + 8), "d"(s) : "memory");
            if (lane < 16) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to_peer + 32), "d"(en) : "memory");
        }
        __syncwarp();
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    // the row's
    double row_max = 0.0, total = 0.0, rest_of_row = 0.0, row_entries = 0.0;
    if (warp == 0) {
        double m = -CUDART_INF, s = 0.0;
        if (half < (int)cluster) m = lane < 16 ? parts[half].rest_max : parts[half].top_max, s = lane < 16 ? parts[half].rest_sum : parts[half].top_sum;
        const double own = m;
        row_max = distill_warp_max(m);
        if (s != 0.0) s *= exp((own - row_max) * p.inv_t);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        rest_of_row = __shfl_sync(0xffffffffu, s, 0);
        total = rest_of_row + __shfl_sync(0xffffffffu, s, 16);
        for (int k = 0; k < (int)cluster; ++k) row_entries += parts[k].entries;
        double factor = teacher.sum + teacher.rest;
        if (teacher.rest > 0.0) factor -= teacher.rest * total / rest_of_row;
        if (!(teacher.sum == teacher.sum)) factor = CUDART_NAN;           // an id outside the row
        if (lane == 0) result[0] = row_max, result[1] = total, result[2] = factor;
    }
    if constexpr (STEP) {
        __syncthreads();
        const A m = A(result[0]);
        const double factor = (double)weight * p.inv_t, s_all = teacher.sum + teacher.rest;
        const A coef = A(factor * result[2] / result[1]);
        const bool alike = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
        const Two<A> less = both(-m), coefs = both(coef);
        auto gradient = [&](int i) {
            Packed<T, E> v, out;
            if constexpr (sizeof(T) >= 4) out.clear();
            const uint4 w = reinterpret_cast<const uint4 *>(held)[i];
            v.w[0] = w.x, v.w[1] = w.y, v.w[2] = w.z, v.w[3] = w.w;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const Two<A> x = (v.get2(e) + less) * scale;
                out.put2(e, two(distill_exp<T>(first(x)), distill_exp<T>(second(x))) * coefs);
            }
            return out;
        };
        int i = threadIdx.x;
        if (alike) {
            T *out = dz - at.skip + (long long)(first_piece + begin + threadIdx.x) * E;
#pragma unroll 2
            for (i = begin + threadIdx.x; i < stop; i += blockDim.x, out += blockDim.x * E) store16(out, gradient(i).w);
            i = threadIdx.x < 2 ? (threadIdx.x ? stop : 0) : count;              // pieces that are not whole
            if (i >= begin && i < stop) i = count;
        }
        for (; i < count; i += alike ? count : blockDim.x) distill_put(at, first_piece + i, dz, alike, gradient(i));
        __syncthreads();                                      // the entries' places have been written with zeros
        for (int k = threadIdx.x; k < p.top; k += blockDim.x)
            if (here(t.place[k])) {
                const double q = exp((t.z[k] - result[0]) * p.inv_t) / result[1];
                dz[t.place[k]] = narrow<T>(A(factor * (q * s_all - t.share[k])));
            }
    }
    // what only the loss needs comes last
    if (rank == 0 && threadIdx.x == 0) {
        const double log_total = row_max * p.inv_t + log(total);
        double loss = teacher.sum != 0.0 ? row_entries + teacher.sum * log_total : 0.0;
        if (teacher.rest > 0.0) loss += teacher.rest * log(teacher.rest * total / rest_of_row);        // P (log P - log Q)
        if (!(teacher.sum == teacher.sum)) loss = CUDART_NAN;
        if (p.loss) static_cast<A *>(p.loss)[row] = A(loss);
        if (!STEP && p.stats) {
            A *const st = static_cast<A *>(p.stats);
            st[row] = A(row_max), st[p.rows + row] = A(total), st[2 * p.rows + row] = A(result[2]);
        }
    }
}

// dz from saved statistics: p.slice pieces of a row (blockIdx.x, blockIdx.y) a CTA.
template <class T>
__global__ void __launch_bounds__(256) distill_grad_kernel(const __grid_constant__ DistillParams p)
{
    using A = Acc<T>;
    constexpr int E = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char distill_memory[];
    __shared__ TeacherSums teacher;
    wait_for_earlier();
    const long long row = blockIdx.x;
    const int first = (int)blockIdx.y * p.slice;
    const T *z = static_cast<const T *>(p.logits) + row * p.ld_logits;
    T *dz = static_cast<T *>(p.dz) + row * p.ld_dz;
    const A weight = p.dloss ? static_cast<const A *>(p.dloss)[row] : A(1);
    if (weight == A(0)) {
        distill_zero(dz, p.vocab, first, blockIdx.y + 1 == gridDim.y ? p.slice + 1 : p.slice);
        return;
    }
    const RowPieces<T> at(z, p.vocab);
    const T *const base = z - at.skip;
    const int last = min(first + p.slice, at.pieces);
    const Teacher t = teacher_at(distill_memory, p.top);
    constexpr int kTogether = 4;
    Packed<T, E> v[kTogether];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int i = i0 + u * (int)blockDim.x;
            if (i >= last) continue;
            if (at.whole(i)) load16(v[u].w, base + (long long)i * E);
            else {
                v[u].clear();
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at.holds(i * E + e)) v[u].put(e, base[i * E + e]);
            }
        }
    };
    fetch(first + threadIdx.x);
    const A *const stats = static_cast<const A *>(p.stats);
    const A m = stats[row], total = stats[p.rows + row], factor = stats[2 * p.rows + row];
    if (threadIdx.x < 32) teacher_shares<T>(p, row, t, teacher);
    __syncthreads();
    teacher_places(t, p.top);
    const int from = first * E - at.skip, to = last * E - at.skip;
    const auto here = [&](int place) { return place >= 0 && place >= from && place < to; };
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (here(t.place[k])) t.z[k] = (double)widen(z[t.place[k]]);
    __syncthreads();                                          // before anything is written: dz may be the logits
    const double scale = (double)weight * p.inv_t, s_all = teacher.sum + teacher.rest;
    // an id outside the row is one in the statistics too, and makes them NaN
    const A unit = distill_unit<T>(p.inv_t), coef = A(scale * (double)factor / (double)total);
    const bool alike = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
    const Two<A> less = both(-m), units = both(unit), coefs = both(coef);
    for (int i0 = first + threadIdx.x; i0 < last; i0 += kTogether * blockDim.x) {
        if (i0 != first + (int)threadIdx.x) fetch(i0);
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int i = i0 + u * (int)blockDim.x;
            if (i >= last) continue;
            Packed<T, E> out;
            if constexpr (sizeof(T) >= 4) out.clear();
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const Two<A> x = (v[u].get2(e) + less) * units;
                out.put2(e, two(distill_exp<T>(fo::first(x)), distill_exp<T>(second(x))) * coefs);
            }
            distill_put(at, i, dz, alike, out);
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (here(t.place[k])) {
            const double q = exp((t.z[k] - (double)m) * p.inv_t) / (double)total;
            dz[t.place[k]] = narrow<T>(A(scale * (q * s_all - t.share[k])));
        }
}

// Host: the kernels of one element type; distill_*.cu instantiate them.
enum DistillWay { kDistillLoss, kDistillStep, kDistillGrad };
template <class T>
cudaError_t launch_distill(DistillParams p, DistillWay way, cudaStream_t st);

}  // namespace fo
