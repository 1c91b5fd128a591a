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

// Reductions of a CTA in a fixed order; `room`: 32 values, free again after the next barrier.
__device__ __forceinline__ double cta_sum(double v, double *room)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < (blockDim.x >> 5) ? room[threadIdx.x & 31] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double cta_max(double v, double *room)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < (blockDim.x >> 5) ? room[threadIdx.x & 31] : -CUDART_INF;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The teacher's entries of one row, in shared memory.
struct Teacher {
    int *id;                            // -1: no entry
    double *p, *z;                      // shares, and the student's logits
    double top_max, log_sum;            // log p = v / temperature - top_max - log_sum
    double sum, rest;                   // of p, and P
};

template <class T>
__device__ __forceinline__ double teacher_value(const DistillParams &p, long long row, int k)
{
    const long long at = row * p.ld_values + k;
    const double v = p.wide_values ? (double)static_cast<const float *>(p.values)[at] : (double)widen(static_cast<const T *>(p.values)[at]);
    return v * p.inv_t;
}

// Fills t (barriers inside; room: 3 x 32 values).  An id that is no place of the row makes the sum NaN, and with it everything.
template <class T>
__device__ __forceinline__ void teacher_shares(const DistillParams &p, long long row, double *room, Teacher &t)
{
    double most = -CUDART_INF, sum = 0.0;
    bool bad = false;
    for (int k = threadIdx.x; k < p.top; k += blockDim.x) {
        const long long at = row * p.ld_ids + k;
        const long long id = p.ids_long ? static_cast<const long long *>(p.ids)[at] : static_cast<const int *>(p.ids)[at];
        t.id[k] = id < 0 || id >= p.vocab ? -1 : (int)id;
        bad = bad || id >= p.vocab;
        if (id >= 0) most = fmax(most, teacher_value<T>(p, row, k));
    }
    if (p.tail) t.top_max = (double)static_cast<const Acc<T> *>(p.tail)[row];
    else t.top_max = cta_max(most, room);
    for (int k = threadIdx.x; k < p.top; k += blockDim.x) {
        const double e = t.id[k] >= 0 ? exp(teacher_value<T>(p, row, k) - t.top_max) : 0.0;
        t.p[k] = e, sum += e;
    }
    sum = cta_sum(bad ? CUDART_NAN : sum, room + 32);
    t.log_sum = 0.0, t.sum = sum, t.rest = 0.0;
    if (p.tail) {
        t.rest = sum < 1.0 ? 1.0 - sum : sum >= 1.0 ? 0.0 : sum;
    } else if (sum != 0.0) {                              // 0: no entries
        t.log_sum = log(sum);
        for (int k = threadIdx.x; k < p.top; k += blockDim.x) t.p[k] /= sum;
        t.sum = sum / sum;
    }
    __syncthreads();
}

// True for the first of the entries with this one's place; its share becomes that of all of them.
__device__ __forceinline__ bool first_of_place(const Teacher &t, int top, int k, double &share)
{
    const int id = t.id[k];
    for (int j = 0; j < k; ++j)
        if (t.id[j] == id) return false;
    share = t.p[k];
    for (int j = k + 1; j < top; ++j)
        if (t.id[j] == id) share += t.p[j];
    return true;
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

// What the CTAs of a cluster tell each other.
struct DistillPart {
    double rest_max, rest_sum, top_max, top_sum, entries;
};

template <class T, bool STEP>
__global__ void __launch_bounds__(512) distill_kernel(const __grid_constant__ DistillParams p)
{
    using A = Acc<T>;
    constexpr int E = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char distill_memory[];
    __shared__ double room[5][32];
    __shared__ DistillPart parts[8];
    __shared__ double result[5];
    unsigned rank, cluster;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
    if (cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    wait_for_earlier();
    const long long row = blockIdx.x / cluster;
    const T *z = static_cast<const T *>(p.logits) + row * p.ld_logits;
    T *dz = STEP ? static_cast<T *>(p.dz) + row * p.ld_dz : nullptr;
    const int first = (int)rank * p.slice;
    A weight = A(1);
    if (STEP) {
        if (p.dloss) weight = static_cast<const A *>(p.dloss)[row];
        if (weight == A(0)) {                                 // the row is not looked at
            if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            // one piece more than the logits' can be the gradient's, at another offset: the last CTA has it
            distill_zero(dz, p.vocab, first, rank + 1 == cluster ? p.slice + 1 : p.slice);
            if (rank == 0 && threadIdx.x == 0) static_cast<A *>(p.loss)[row] = A(0);
            return;
        }
    }
    const RowPieces<T> at(z, p.vocab);
    const int count = max(0, min(p.slice, at.pieces - first));
    T *const held = reinterpret_cast<T *>(distill_memory);
    Teacher t;
    t.p = reinterpret_cast<double *>(distill_memory + (size_t)p.slice * 16);
    t.z = t.p + p.top;
    t.id = reinterpret_cast<int *>(t.z + p.top);
    const T *const base = z - at.skip;
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        if (at.whole(first + i)) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(held + i * E)),
                         "l"(base + (long long)(first + i) * E) : "memory");
        } else {
            for (int e = 0; e < E; ++e) {
                const int j = (first + i) * E + e;
                held[i * E + e] = at.holds(j) ? base[j] : narrow<T>(distill_floor<A>());
            }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    teacher_shares<T>(p, row, &room[0][0], t);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();

    // the entries in this CTA's part: the largest, then out of the row
    const int from = first * E - at.skip, to = from + count * E;      // elements of the row
    double most = -CUDART_INF, entries = 0.0, top_sum = 0.0;
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (t.id[k] >= from && t.id[k] < to && t.id[k] >= 0) most = fmax(most, (double)widen(held[t.id[k] - from]));
    most = cta_max(most, room[2]);
    for (int k = threadIdx.x; k < p.top; k += blockDim.x) {
        if (t.id[k] < from || t.id[k] >= to || t.id[k] < 0) continue;
        const double v = (double)widen(held[t.id[k] - from]), share = t.p[k];
        t.z[k] = v;
        if (share != 0.0) entries += share * (teacher_value<T>(p, row, k) - t.top_max - t.log_sum - v * p.inv_t);
        double whole;
        if (first_of_place(t, p.top, k, whole)) top_sum += exp((v - most) * p.inv_t);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (t.id[k] >= from && t.id[k] < to && t.id[k] >= 0) held[t.id[k] - from] = narrow<T>(distill_floor<A>());
    __syncthreads();

    // all the rest: every thread keeps the largest so far and the sum relative to it
    const A unit = distill_unit<T>(p.inv_t);
    A largest = distill_floor<A>(), sum = A(0);
    constexpr int kTogether = 4;
    for (int i0 = threadIdx.x; i0 < count; i0 += kTogether * blockDim.x) {
        Packed<T, E> v[kTogether];
        A top = largest;
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int i = i0 + u * blockDim.x;
            if (i < count) {
                const uint4 w = *reinterpret_cast<const uint4 *>(held + i * E);
                v[u].w[0] = w.x, v[u].w[1] = w.y, v[u].w[2] = w.z, v[u].w[3] = w.w;
#pragma unroll
                for (int e = 0; e < E; ++e) top = larger(top, v[u].get(e));
            }
        }
        const A ref = top == distill_floor<A>() ? A(0) : top;
        A more = A(0);
#pragma unroll
        for (int u = 0; u < kTogether; ++u)
            if (i0 + u * (int)blockDim.x < count) {
#pragma unroll
                for (int e = 0; e < E; ++e) more += distill_exp<T>((v[u].get(e) - ref) * unit);
            }
        sum = fused_ma(sum, distill_exp<T>((largest - ref) * unit), more);
        largest = top;
    }
    // the CTA's
    double rest_max = (double)largest;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) rest_max = fmax(rest_max, __shfl_xor_sync(0xffffffffu, rest_max, o));
    double rest_sum = sum == A(0) ? 0.0 : (double)(sum * distill_exp<T>((largest - A(rest_max)) * unit));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        rest_sum += __shfl_xor_sync(0xffffffffu, rest_sum, o);
        top_sum += __shfl_xor_sync(0xffffffffu, top_sum, o);
        entries += __shfl_xor_sync(0xffffffffu, entries, o);
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (lane == 0) room[0][warp] = rest_max, room[1][warp] = rest_sum, room[3][warp] = top_sum, room[4][warp] = entries;
    __syncthreads();
    if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // every CTA has started
    if (warp == 0) {
        const bool in = lane < warps;
        double m = in ? room[0][lane] : -CUDART_INF, s = in ? room[1][lane] : 0.0, ts = in ? room[3][lane] : 0.0, en = in ? room[4][lane] : 0.0;
        double all = m;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all = fmax(all, __shfl_xor_sync(0xffffffffu, all, o));
        if (s != 0.0) s *= exp((m - all) * p.inv_t);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            ts += __shfl_xor_sync(0xffffffffu, ts, o);
            en += __shfl_xor_sync(0xffffffffu, en, o);
        }
        const double mine[5] = {all, s, most, ts, en};
        if (cluster == 1) {
            if (lane == 0) parts[0] = {all, s, most, ts, en};
        } else if (lane < (int)cluster) {                     // lane k tells CTA k
            unsigned to_peer;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to_peer) : "r"((unsigned)__cvta_generic_to_shared(&parts[rank])), "r"(lane));
#pragma unroll
            for (int k = 0; k < 5; ++k)
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to_peer + 8 * k), "d"(mine[k]) : "memory");
        }
        __syncwarp();
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    // the row's
    if (warp == 0) {
        const bool in = lane < (int)cluster;
        const DistillPart d = in ? parts[lane] : DistillPart{-CUDART_INF, 0.0, -CUDART_INF, 0.0, 0.0};
        double m = fmax(d.rest_max, d.top_max), en = d.entries;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
        double s = d.rest_sum != 0.0 ? d.rest_sum * exp((d.rest_max - m) * p.inv_t) : 0.0;
        double ts = d.top_sum != 0.0 ? d.top_sum * exp((d.top_max - m) * p.inv_t) : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            ts += __shfl_xor_sync(0xffffffffu, ts, o);
            en += __shfl_xor_sync(0xffffffffu, en, o);
        }
        const double total = s + ts, log_total = m * p.inv_t + log(total);
        double loss = t.sum != 0.0 ? en + t.sum * log_total : 0.0, factor = t.sum + t.rest;
        if (t.rest > 0.0) {                                   // P (log P - log Q), Q = s / total
            const double ratio = t.rest * total / s;
            loss += t.rest * log(ratio), factor -= ratio;
        }
        if (!(t.sum == t.sum)) loss = factor = CUDART_NAN;    // an id outside the row
        if (lane == 0) {
            result[0] = m, result[1] = total, result[2] = factor;
            if (rank == 0) {
                if (p.loss) static_cast<A *>(p.loss)[row] = A(loss);
                if (!STEP && p.stats) {
                    A *const st = static_cast<A *>(p.stats);
                    st[row] = A(m), st[p.rows + row] = A(total), st[2 * p.rows + row] = A(factor);
                }
            }
        }
    }
    if constexpr (STEP) {
        __syncthreads();
        const A m = A(result[0]);
        const double scale = (double)weight * p.inv_t, s_all = t.sum + t.rest;
        const A coef = A(scale * result[2] / result[1]);
        const bool alike = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
        for (int i = threadIdx.x; i < count; i += blockDim.x) {
            Packed<T, E> v, out;
            out.clear();
            const uint4 w = *reinterpret_cast<const uint4 *>(held + i * E);
            v.w[0] = w.x, v.w[1] = w.y, v.w[2] = w.z, v.w[3] = w.w;
#pragma unroll
            for (int e = 0; e < E; e += 2) out.put2(e, two(distill_exp<T>((v.get(e) - m) * unit) * coef, distill_exp<T>((v.get(e + 1) - m) * unit) * coef));
            distill_put(at, first + i, dz, alike, out);
        }
        __syncthreads();                                      // the entries' places have been written with zeros
        for (int k = threadIdx.x; k < p.top; k += blockDim.x) {
            double share;
            if (t.id[k] < from || t.id[k] >= to || t.id[k] < 0 || !first_of_place(t, p.top, k, share)) continue;
            const double q = exp((t.z[k] - result[0]) * p.inv_t) / result[1];
            dz[t.id[k]] = narrow<T>(A(scale * (q * s_all - share)));
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
    __shared__ double room[2][32];
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
    Teacher t;
    t.p = reinterpret_cast<double *>(distill_memory);
    t.z = t.p + p.top;
    t.id = reinterpret_cast<int *>(t.z + p.top);
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
    teacher_shares<T>(p, row, &room[0][0], t);
    const int from = first * E - at.skip, to = last * E - at.skip;
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (t.id[k] >= from && t.id[k] < to && t.id[k] >= 0) t.z[k] = (double)widen(z[t.id[k]]);
    __syncthreads();                                          // before anything is written: dz may be the logits
    const double scale = (double)weight * p.inv_t, s_all = t.sum + t.rest;
    // an id outside the row is one in the statistics too, and makes them NaN
    const A unit = distill_unit<T>(p.inv_t), coef = A(scale * (double)factor / (double)total);
    const bool alike = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
    for (int i0 = first + threadIdx.x; i0 < last; i0 += kTogether * blockDim.x) {
        if (i0 != first + (int)threadIdx.x) fetch(i0);
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int i = i0 + u * (int)blockDim.x;
            if (i >= last) continue;
            Packed<T, E> out;
            out.clear();
#pragma unroll
            for (int e = 0; e < E; e += 2)
                out.put2(e, two(distill_exp<T>((v[u].get(e) - m) * unit) * coef, distill_exp<T>((v[u].get(e + 1) - m) * unit) * coef));
            distill_put(at, i, dz, alike, out);
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < p.top; k += blockDim.x) {
        double share;
        if (t.id[k] < from || t.id[k] >= to || t.id[k] < 0 || !first_of_place(t, p.top, k, share)) continue;
        const double q = exp((t.z[k] - (double)m) * p.inv_t) / (double)total;
        dz[t.id[k]] = narrow<T>(A(scale * (q * s_all - share)));
    }
}

// Host: the kernels of one element type; distill_*.cu instantiate them.
enum DistillWay { kDistillLoss, kDistillStep, kDistillGrad };
template <class T>
cudaError_t launch_distill(DistillParams p, DistillWay way, cudaStream_t st);

}  // namespace fo
