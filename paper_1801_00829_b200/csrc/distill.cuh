// The distillation loss from a teacher's top logits and its gradient.
//
// Loss, or loss and gradient at once: a CTA, or of short rows a team of its warps, goes through a row once for the sums and a second
// time, backwards, for the gradient; the first time the row is marked to be kept in L2, the second time, and what is written, as not
// needed again (4096 x 128000 in bfloat16 494 us, without the marks 571: of the second reading 0.45 hit L2, without them none).  Rows
// kept in the shared memory of clusters are read once, but leave room for few CTAs, and what they do besides reading and writing is then
// not hidden (542 us).  The entries' places are marked in a map of bits and passed over in the sums: what the teacher's entries leave is
// added up by itself, not as 1 minus their sum, and the entries, which hold most of the probability, are summed in 64 bits.
// The gradient alone is elementwise from the saved statistics, a CTA to a part of a row; the entries' places are written over at the end, so
// that their shares are found meanwhile (4096 x 128000 in bfloat16 358 us, 5.9 TB/s).
#pragma once

#include <cfloat>

#include <math_constants.h>

#include "elem.cuh"
#include "../../include/fusedops_lm.h"

namespace fo {

// Threads of a CTA, of which three work on an SM; of a row where there are few rows; and the bound on threads that keeps registers
// for 3 x 256 of them.
constexpr int kDistillCta = 256, kDistillRow = 512, kDistillBound = 768;

struct DistillParams {
    long long rows;
    int vocab, top;
    int ids_long, wide_values;
    int slice;                          // pieces of a CTA (gradient)
    int team, shared;                   // threads of a row, and their shared memory
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
__device__ __forceinline__ constexpr double distill_unit_of()
{
    return sizeof(T) == 2 ? 1.4426950408889634074 : 1.0;
}
// 1 / temperature in these units, as a number of 32 bits neither zero nor infinite (times a masked logit's minus infinity or the largest
// logit's zero it would be NaN)
template <class T>
__device__ __forceinline__ Acc<T> distill_unit(double inv_t)
{
    const double unit = inv_t * distill_unit_of<T>();
    if constexpr (sizeof(T) == 8) return unit;
    else return (float)fmin(fmax(unit, 0x1p-149), (double)FLT_MAX);
}
// What exponentials are multiplied by, some of which are zero: finite if it is so in 64 bits
template <class T>
__device__ __forceinline__ Acc<T> distill_coef(double v)
{
    if constexpr (sizeof(T) == 8) return v;
    else return fabs(v) > (double)FLT_MAX && fabs(v) < CUDART_INF ? (v < 0.0 ? -FLT_MAX : FLT_MAX) : (float)v;
}
template <class A> __device__ __forceinline__ A distill_floor() { return -A(CUDART_INF); }

__device__ __forceinline__ float next_below(float v) { return nextafterf(v, -CUDART_INF_F); }
__device__ __forceinline__ double next_below(double v) { return nextafter(v, -CUDART_INF); }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }

// The threads of one row: a CTA's, or a part of them that has barriers of its own.
struct Team {
    int thread, threads, number;        // this thread, all of them, and the team's number in its CTA
    __device__ __forceinline__ void sync() const
    {
        if (threads == 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(number + 1), "r"(threads) : "memory");
    }
};

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
// The teacher's entries of one row, in shared memory.
struct Teacher {
    int *id;                            // -1: no entry; padded to a multiple of 4
    double *p, *share, *z, *v;          // shares, those of a place, the student's logits, and the teacher's over temperature
    int *place;                         // of an entry that is the first of its place; -1
};

constexpr int kTeacherBytes = 40;       // of an entry in shared memory
__device__ __forceinline__ Teacher teacher_at(void *memory, int top)
{
    const int room = (top + 3) / 4 * 4;
    Teacher t;
    t.p = static_cast<double *>(memory), t.share = t.p + room, t.z = t.share + room, t.v = t.z + room;
    t.id = reinterpret_cast<int *>(t.v + room), t.place = t.id + room;
    return t;
}

template <class T>
__device__ __forceinline__ double teacher_value(const DistillParams &p, long long row, int k)
{
    const long long at = row * p.ld_values + k;
    const double v = p.wide_values ? (double)static_cast<const float *>(p.values)[at] : (double)widen(static_cast<const T *>(p.values)[at]);
    return v * p.inv_t;
}

// P up to this is taken as zero where nothing of q lies outside the entries (they are the whole vocabulary, or the rest of it is
// masked): it is what the rounding of values and tail has left.  A value of 16 is off by 2^-5 in bfloat16, and so is its share then.
constexpr double kDistillNoise = 0.03125;
// A student is sure where P / Q is above this.  Q then comes near the smallest numbers of 32 bits, and P / Q near the largest: the gradient
// outside, q (S - P / Q), is formed as -exp((z - largest) / T + log(P / Q)) over the row's sum, and what is kept of the row is that
// logarithm (S is below its last bit), with a minus at the sum.
constexpr double kDistillSure = 0x1p60;

// What all threads need to know of the entries besides the arrays.
struct TeacherSums {
    double top_max, log_sum;            // log p = v / temperature - top_max - log_sum
    double sum, rest;                   // of p, and P
};
// All threads: the entries as they lie in memory.  An id that is no place of the row makes the sum of the shares NaN, and with it
// everything.  Z: the student's logits too.
template <class T, bool Z = false>
__device__ __forceinline__ void teacher_read(const DistillParams &p, long long row, const Teacher &t, const Team &team, const T *z = nullptr)
{
    for (int k = team.thread; k < p.top; k += team.threads) {
        const long long at = row * p.ld_ids + k;
        const long long id = p.ids_long ? static_cast<const long long *>(p.ids)[at] : static_cast<const int *>(p.ids)[at];
        t.v[k] = id >= p.vocab ? CUDART_NAN : teacher_value<T>(p, row, k);
        t.id[k] = id < 0 ? -1 : id >= p.vocab ? -2 : (int)id;
        if (Z) t.z[k] = id >= 0 && id < p.vocab ? (double)widen(z[id]) : 0.0;
    }
    if (team.thread < ((4 - p.top % 4) & 3)) t.id[p.top + team.thread] = -1;
}
// The first warp, after a barrier: shares and their sums.  tail: the row's.
__device__ __forceinline__ void teacher_shares(const DistillParams &p, const Teacher &t, double tail, TeacherSums &out)
{
    const int lane = threadIdx.x & 31;
    double reference = tail, sum = 0.0;
    if (!p.tail) {
        reference = -CUDART_INF;
        for (int k = lane; k < p.top; k += 32)
            if (t.id[k] >= 0) reference = fmax(reference, t.v[k]);
        reference = distill_warp_max(reference);
    }
    for (int k = lane; k < p.top; k += 32) {
        const double e = t.id[k] == -1 ? 0.0 : exp(t.v[k] - reference);
        t.p[k] = e, sum += e;
    }
    sum = distill_warp_sum(sum);
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
// Meanwhile, from the last thread on: of entries with the same place the first one (place; the others have none), and the student's
// logits (Z).
template <class T, bool Z = true>
__device__ __forceinline__ void teacher_places(const Teacher &t, int top, const T *z, const Team &team)
{
    for (int k = team.threads - 1 - team.thread; k < top; k += team.threads) {
        const int id = t.id[k];
        const double own = Z && id >= 0 ? (double)widen(z[id]) : 0.0;
        bool again = false;
        const int4 *const four = reinterpret_cast<const int4 *>(t.id);
#pragma unroll 4
        for (int j = 0; j < (k + 3) / 4; ++j) {
            const int4 v = four[j];
            again = again || (v.x == id && 4 * j < k) || (v.y == id && 4 * j + 1 < k) || (v.z == id && 4 * j + 2 < k) || (v.w == id && 4 * j + 3 < k);
        }
        t.place[k] = again || id < 0 ? -1 : id;
        if (Z) t.z[k] = own;
    }
}
// After another barrier: the share of the first entry of a place, which is that of all of them.
__device__ __forceinline__ double teacher_share(const Teacher &t, int top, int k)
{
    double all = t.p[k];
    const int id = t.id[k];
    const int4 *const four = reinterpret_cast<const int4 *>(t.id);
#pragma unroll 4
    for (int j = k / 4; j < (top + 3) / 4; ++j) {
        const int4 v = four[j];
        if (v.x == id || v.y == id || v.z == id || v.w == id)
            for (int q = max(k + 1, 4 * j); q < min(top, 4 * j + 4); ++q)
                if (t.id[q] == id) all += t.p[q];
    }
    return all;
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
__device__ __forceinline__ void distill_zero(T *dz, int vocab, int first, int count, const Team &team)
{
    const RowPieces<T> out(dz, vocab);
    T *const base = dz - out.skip;
    const uint32_t none[4] = {0, 0, 0, 0};
    for (int i = first + team.thread; i < min(first + count, out.pieces); i += team.threads) {
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

// Ways through L2: what is kept for the second reading, and what is not needed again.
__device__ __forceinline__ unsigned long long distill_keep()
{
    unsigned long long policy;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
__device__ __forceinline__ unsigned long long distill_drop()
{
    unsigned long long policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
__device__ __forceinline__ void distill_store(void *p, const uint32_t *w, unsigned long long policy)
{
    asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "l"(policy) : "memory");
}
// A whole piece of logits.
template <class T>
__device__ __forceinline__ Packed<T, 16 / sizeof(T)> distill_piece(const T *at, unsigned long long policy)
{
    Packed<T, 16 / sizeof(T)> v;
    asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "l"(at), "l"(policy) : "memory");
    return v;
}

struct DistillPart {
    double rest_max, rest_sum, top_max, top_sum, entries;
};
// A row's sums, in shared memory: its threads' registers are for the pieces of the second reading.
struct DistillResult {
    double largest, total, factor;      // factor: S - P / Q
    double log_share;                   // log(P / Q) of a student that is sure, else zero
    double coef;                        // of exp((z - largest) / T + log_share) outside the entries
    double all, rest, ratio, entries;   // S, P, P / Q, and what the entries add to the loss
};

// Loss, and with STEP the gradient.  Bound by DRAM and by what of the second reading misses L2 (about half): 4096 x 128000 in bfloat16
// with rows of padding 441 to 457 us, with all rows counting 490 (4.3 TB/s of one reading and one writing); short rows by what a row
// costs besides, which other rows on the SM hide (16384 x 1000 90 us).
template <class T, bool STEP>
__global__ void __launch_bounds__(kDistillBound, 1) distill_kernel(const __grid_constant__ DistillParams p)
{
    using A = Acc<T>;
    constexpr int E = 16 / (int)sizeof(T), kTogether = 4;
    extern __shared__ __align__(16) unsigned char distill_memory[];
    __shared__ DistillPart all_parts[kDistillRow / 32];
    __shared__ DistillResult results[kDistillCta / 32];
    __shared__ TeacherSums teachers[kDistillCta / 32];
    wait_for_earlier();
    const int number = threadIdx.x / p.team, lane = threadIdx.x & 31, step = p.team;
    const Team team = {(int)threadIdx.x - number * p.team, p.team, number};
    const int warp = team.thread >> 5, warps = p.team >> 5;
    DistillPart *const parts = all_parts + number * warps;
    DistillResult &result = results[number];
    TeacherSums &teacher = teachers[number];
    const long long row = (long long)blockIdx.x * (blockDim.x / p.team) + number;
    if (row >= p.rows) return;
    const T *z = static_cast<const T *>(p.logits) + row * p.ld_logits;
    T *dz = STEP ? static_cast<T *>(p.dz) + row * p.ld_dz : nullptr;
    unsigned char *const memory = distill_memory + (size_t)number * p.shared;
    const Teacher t = teacher_at(memory, p.top);
    uint32_t *const marks = reinterpret_cast<uint32_t *>(memory + (size_t)(p.top + 3) / 4 * 4 * kTeacherBytes);
    A weight = A(1);
    if (STEP && p.dloss) weight = static_cast<const A *>(p.dloss)[row];
    const double tail = p.tail ? (double)static_cast<const A *>(p.tail)[row] : 0.0;
    teacher_read<T>(p, row, t, team);
    const RowPieces<T> at(z, p.vocab);
    if (STEP && weight == A(0)) {                             // the row is not looked at
        distill_zero(dz, p.vocab, 0, at.pieces + 1, team);          // (the gradient's may be one piece more, at another offset)
        if (team.thread == 0) static_cast<A *>(p.loss)[row] = A(0);
        return;
    }
    // whole pieces of the row: [begin, stop); of the others there is at most one at each end
    const T *const base = z - at.skip;
    const int begin = at.skip ? 1 : 0, stop = max(begin, at.end / E), mine = begin + team.thread;
    const unsigned long long drop = distill_drop(), keep = STEP ? distill_keep() : drop;
    int i = mine;
    const T *from = base + (long long)i * E;
    Packed<T, E> next[kTogether];                             // the first pieces are on their way while the entries are seen to
    auto fetch = [&]() {
        if (i + (kTogether - 1) * step < stop)
#pragma unroll
            for (int u = 0; u < kTogether; ++u) next[u] = distill_piece(from + (long long)u * step * E, keep);
    };
    fetch();
    for (int k = team.thread; k < (at.end + 127) / 128; k += step) reinterpret_cast<uint4 *>(marks)[k] = make_uint4(0, 0, 0, 0);
    team.sync();

    // the entries: a mark at each place, and what they add
    if (warp == 0) teacher_shares(p, t, tail, teacher);
    teacher_places(t, p.top, z, team);
    for (int k = step - 1 - team.thread; k < p.top; k += step)
        if (t.place[k] >= 0) {
            const int place = at.skip + t.place[k];
            atomicOr(&marks[place >> 5], 1u << (place & 31));
        }
    team.sync();
    double entries = 0.0, top_max = -CUDART_INF, top_sum = 0.0;
    if ((warps - 1 - warp) * 32 < p.top) {
        for (int k = step - 1 - team.thread; k < p.top; k += step)
            if (t.id[k] >= 0) {
                const double share = t.p[k];
                if (share != 0.0) entries += share * (t.v[k] - teacher.top_max - teacher.log_sum - t.z[k] * p.inv_t);
                if (t.place[k] >= 0) top_max = fmax(top_max, t.z[k]);
            }
        top_max = distill_warp_max(top_max), entries = distill_warp_sum(entries);
        const double ref = top_max == -CUDART_INF ? 0.0 : top_max;        // the warp's entries may all be masked
        for (int k = step - 1 - team.thread; k < p.top; k += step)
            if (t.place[k] >= 0) {
                top_sum += exp((t.z[k] - ref) * p.inv_t);
                if (STEP) t.share[k] = teacher_share(t, p.top, k);
            }
        top_sum = distill_warp_sum(top_sum);
    }

    // all the rest: every thread keeps the largest so far and the sum relative to it
    const A unit = distill_unit<T>(p.inv_t);
    const Two<A> scale = both(unit);
    A largest = distill_floor<A>(), sum = A(0);
    auto marked = [&](int i) { return (marks[i * E >> 5] >> (i * E & 31)) & ((1u << E) - 1u); };
    auto without = [&](Packed<T, E> v, unsigned bits) {       // minus infinity at the marked places
        Packed<T, E> r;
        r.clear();
#pragma unroll
        for (int e = 0; e < E; ++e) r.put(e, (bits >> e) & 1u ? narrow<T>(distill_floor<A>()) : v.raw(e));
        return r;
    };
    auto take = [&](auto many, const Packed<T, E> *v) {
        constexpr int M = many.value;
        A top = largest;
#pragma unroll
        for (int u = 0; u < M; ++u) top = distill_largest<T>(v[u], top);
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
        while (i + (kTogether - 1) * step < stop) {
            Packed<T, E> v[kTogether];
            const int now = i;
#pragma unroll
            for (int u = 0; u < kTogether; ++u) v[u] = next[u];
            i += kTogether * step, from += (long long)kTogether * step * E;
            fetch();
#pragma unroll
            for (int u = 0; u < kTogether; ++u) {
                const unsigned bits = marked(now + u * step);
                if (bits) v[u] = without(v[u], bits);
            }
            take(std::integral_constant<int, kTogether>(), v);
        }
        for (; i < stop; i += step, from += (long long)step * E) {
            Packed<T, E> v = distill_piece(from, keep);
            const unsigned bits = marked(i);
            if (bits) v = without(v, bits);
            take(std::integral_constant<int, 1>(), &v);
        }
    }
    // pieces that are not whole: their elements outside the row are minus infinity
    auto ragged = [&](int i) {
        Packed<T, E> v;
        v.clear();
#pragma unroll
        for (int e = 0; e < E; ++e) v.put(e, at.holds(i * E + e) ? base[i * E + e] : narrow<T>(distill_floor<A>()));
        return v;
    };
    const int other = team.thread == 0 ? (begin ? 0 : at.pieces) : team.thread == 1 ? stop : at.pieces;
    const bool ends = other < at.pieces && (other < begin || other >= stop);
    if (ends) {
        const Packed<T, E> v = without(ragged(other), marked(other));
        take(std::integral_constant<int, 1>(), &v);
    }
    // the warp's
    A rest_max = largest;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) rest_max = larger(rest_max, __shfl_xor_sync(0xffffffffu, rest_max, o));
    A rest_sum = sum == A(0) ? A(0) : sum * distill_exp<T>((largest - rest_max) * unit);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) rest_sum += __shfl_xor_sync(0xffffffffu, rest_sum, o);
    if (lane == 0) parts[warp] = {(double)rest_max, (double)rest_sum, top_max, top_sum, entries};
    team.sync();
    // the row's
    if (warp == 0) {
        DistillPart d = {-CUDART_INF, 0.0, -CUDART_INF, 0.0, 0.0};
        if (lane < warps) d = parts[lane];
        const double row_max = distill_warp_max(fmax(d.rest_max, d.top_max));
        // in 64 bits: zero only if Q is as a number of 64 bits
        const double rest_of_row = distill_warp_sum(d.rest_sum != 0.0 ? d.rest_sum * exp((d.rest_max - row_max) * p.inv_t) : 0.0);
        const double total = rest_of_row + distill_warp_sum(d.top_sum != 0.0 ? d.top_sum * exp((d.top_max - row_max) * p.inv_t) : 0.0);
        const double row_entries = distill_warp_sum(d.entries);
        const double rest = rest_of_row == 0.0 && teacher.rest <= kDistillNoise ? 0.0 : teacher.rest;
        const double ratio = rest > 0.0 ? rest * total / rest_of_row : 0.0;
        const bool sure = rest_of_row > 0.0 && ratio > kDistillSure;
        double log_share = 0.0;
        if (sure) {                                           // by logarithms, from the largest outside
            const double rest_max = distill_warp_max(d.rest_max);
            const double outside = distill_warp_sum(d.rest_sum != 0.0 ? d.rest_sum * exp((d.rest_max - rest_max) * p.inv_t) : 0.0);
            log_share = log(rest) + log(total) - ((rest_max - row_max) * p.inv_t + log(outside));
        }
        double factor = teacher.sum + rest - ratio;
        if (!(teacher.sum == teacher.sum)) factor = CUDART_NAN;           // an id outside the row
        if (lane == 0) result = {row_max, total, factor, log_share, (double)weight * p.inv_t * (sure ? -1.0 : factor) / total, teacher.sum + rest, rest, ratio, row_entries};
    }
    if constexpr (STEP) {
        team.sync();
        const A m = A(result.largest), coef = distill_coef<T>(result.coef), shift = A(result.log_share * distill_unit_of<T>());
        const bool alike = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
        const Two<A> less = both(-m), coefs = both(coef), shifts = both(shift);
        auto gradient = [&](const Packed<T, E> &v) {
            Packed<T, E> out;
            if constexpr (sizeof(T) >= 4) out.clear();
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const Two<A> x = fused_ma(v.get2(e) + less, scale, shifts);
                out.put2(e, two(distill_exp<T>(first(x)), distill_exp<T>(second(x))) * coefs);
            }
            return out;
        };
        // what was read last is read first
        i = mine + (stop - 1 - mine) / step * step;
        if (stop - 1 < mine) i = -1;
        if (alike) {
            from = base + (long long)i * E;
            T *to = dz - at.skip + (long long)i * E;
            const long long back = (long long)step * E;
            auto fetch_back = [&]() {
                if (i - (kTogether - 1) * step >= begin)
#pragma unroll
                    for (int u = 0; u < kTogether; ++u) next[u] = distill_piece(from - u * back, drop);
            };
            fetch_back();
            while (i - (kTogether - 1) * step >= begin) {
                Packed<T, E> v[kTogether];
#pragma unroll
                for (int u = 0; u < kTogether; ++u) v[u] = next[u];
                i -= kTogether * step, from -= kTogether * back;
                fetch_back();
#pragma unroll
                for (int u = 0; u < kTogether; ++u) distill_store(to - u * back, gradient(v[u]).w, drop);
                to -= kTogether * back;
            }
            for (; i >= begin; i -= step, from -= back, to -= back) distill_store(to, gradient(distill_piece(from, drop)).w, drop);
        } else {
            for (; i >= begin; i -= step) distill_put(at, i, dz, false, gradient(distill_piece(base + (long long)i * E, drop)));
        }
        if (ends) distill_put(at, other, dz, false, gradient(ragged(other)));
        team.sync();                                      // the entries' places have been written like the others
        const double by = (double)weight * p.inv_t, s_all = result.all, inverse = 1.0 / result.total;
        for (int k = team.thread; k < p.top; k += step)
            if (t.place[k] >= 0) {
                const double q = exp((t.z[k] - result.largest) * p.inv_t) * inverse;
                dz[t.place[k]] = narrow<T>(A(by * (q * s_all - t.share[k])));
            }
    }
    // what only the loss needs comes last
    if (team.thread == 0) {
        const double log_total = result.largest * p.inv_t + log(result.total);
        double loss = teacher.sum != 0.0 ? result.entries + teacher.sum * log_total : 0.0;
        if (result.rest > 0.0) loss += result.rest * (result.log_share != 0.0 ? result.log_share : log(result.ratio));        // P (log P - log Q)
        if (!(teacher.sum == teacher.sum)) loss = CUDART_NAN;
        if (p.loss) static_cast<A *>(p.loss)[row] = A(loss);
        if (!STEP && p.stats) {
            const bool sure = result.log_share != 0.0;
            A *const st = static_cast<A *>(p.stats);
            st[row] = A(result.largest), st[p.rows + row] = A(sure ? -result.total : result.total);
            // a P that counts leaves it below sum p, by a bit at least, and so the gradient knows that P counted
            A factor = A(sure ? result.log_share : result.factor);
            if (result.rest > 0.0 && !sure && factor >= A(teacher.sum)) factor = next_below(A(teacher.sum));
            st[2 * p.rows + row] = factor;
        }
    }
}

// dz from saved statistics: p.slice pieces of a row (blockIdx.x, blockIdx.y) a CTA.
template <class T>
__global__ void __launch_bounds__(kDistillCta, 5) distill_grad_kernel(const __grid_constant__ DistillParams p)
{
    using A = Acc<T>;
    constexpr int E = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char distill_memory[];
    __shared__ TeacherSums teacher;
    wait_for_earlier();
    const Team team = {(int)threadIdx.x, (int)blockDim.x, 0};
    const long long row = blockIdx.x;
    const int first = (int)blockIdx.y * p.slice;
    const T *z = static_cast<const T *>(p.logits) + row * p.ld_logits;
    T *dz = static_cast<T *>(p.dz) + row * p.ld_dz;
    const A weight = p.dloss ? static_cast<const A *>(p.dloss)[row] : A(1);
    if (weight == A(0)) {
        distill_zero(dz, p.vocab, first, blockIdx.y + 1 == gridDim.y ? p.slice + 1 : p.slice, team);
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
    const A m = stats[row], kept = stats[p.rows + row], factor = stats[2 * p.rows + row];
    const bool sure = kept < A(0);
    const A total = sure ? -kept : kept;
    teacher_read<T, true>(p, row, t, team, z);
    const double tail = p.tail ? (double)static_cast<const A *>(p.tail)[row] : 0.0;
    __syncthreads();                                                // before anything is written: dz may be the logits
    if (threadIdx.x < 32) teacher_shares(p, t, tail, teacher);
    teacher_places<T, false>(t, p.top, z, team);
    const int from = first * E - at.skip, to = last * E - at.skip;
    const auto here = [&](int place) { return place >= 0 && place >= from && place < to; };
    const double scale = (double)weight * p.inv_t;
    // an id outside the row is one in the statistics too, and makes them NaN
    const A unit = distill_unit<T>(p.inv_t), coef = distill_coef<T>(scale * (sure ? -1.0 : (double)factor) / (double)total);
    const A shift = sure ? A((double)factor * distill_unit_of<T>()) : A(0);
    const bool alike = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
    const Two<A> less = both(-m), units = both(unit), coefs = both(coef), shifts = both(shift);
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
                const Two<A> x = fused_ma(v[u].get2(e) + less, units, shifts);
                out.put2(e, two(distill_exp<T>(fo::first(x)), distill_exp<T>(second(x))) * coefs);
            }
            distill_put(at, i, dz, alike, out);
        }
    }
    __syncthreads();
    // the statistics' S - P / Q is below sum p where P counted; P was zero, or taken as zero, where it is not
    const bool all = !sure && teacher.rest <= kDistillNoise && factor >= A(teacher.sum);
    const double s_all = all ? teacher.sum : teacher.sum + teacher.rest;
    for (int k = threadIdx.x; k < p.top; k += blockDim.x)
        if (here(t.place[k])) {
            const double q = exp((t.z[k] - (double)m) * p.inv_t) / (double)total;
            dz[t.place[k]] = narrow<T>(A(scale * (q * s_all - teacher_share(t, p.top, k))));
        }
}

// Host: the kernels of one element type; distill_*.cu instantiate them.
enum DistillWay { kDistillLoss, kDistillStep, kDistillGrad };
template <class T>
cudaError_t launch_distill(DistillParams p, DistillWay way, cudaStream_t st);

}  // namespace fo
