// Block norm and its gradient (see fusedops_train.h for the mathematics): one pass over the rows,
// each row held in registers between its sums.
//
// A row belongs to a group of threads that hold E of its elements each.  Up to 32 threads the group
// is a part of a warp and its sums are shuffles; above, the group is the CTA, and a sum is a shuffle, one
// exchange through shared memory and a shuffle; the longest rows are split over a cluster of C CTAs, which
// exchange through each other's shared memory.  Rows are read and written once; what bounds the kernels
// is DRAM bandwidth, so the shapes only have to keep enough 16-byte loads in flight and the sums short.
#pragma once

#include <type_traits>

#include "elem.cuh"

namespace fo {

constexpr int kGroupCta = 256;               // CTA size where a group is a warp or less
constexpr int kMostCta = 512;                // and at most where it is the CTA
constexpr int kGradSlots = 6;                // column sums of the gradient: see Slot
enum Slot { kPreW = 0, kPreB = 1, kPostW = 2, kPostB = 3, kColScale = 4, kGateCol = 5 };

struct NormSpec {
    int kind, pad;
    double eps;
    const void *weight, *bias;
};

struct BlockNormParams {
    long long rows;
    int cols;
    int aligned;                             // rows and vectors are whole pieces
    int vectors;                             // vectors begin on 16-byte boundaries
    double inv_cols;                         // 1 / cols
    int wide_vec;                            // vectors are float although the block has 16 bits
    int gate_access, gate_act;               // gate_access -1: none
    const void *x, *f, *gate, *col_scale;
    long long ld_x, ld_f, ld_gate;
    double scale;
    NormSpec post, pre;
    void *h, *y, *stats;
    long long ld_h, ld_y;
};

struct BlockNormGradParams {
    long long rows;
    int cols;
    int aligned, vectors, wide_vec;
    double inv_cols;
    int gate_access, gate_act;
    const void *dh, *dy, *h, *f, *gate, *col_scale, *stats;
    long long ld_dh, ld_dy, ld_h, ld_f, ld_gate;
    double scale;
    NormSpec post, pre;
    void *dx, *df, *dgate;
    long long ld_dx, ld_df, ld_dgate;
    int group;                               // threads of a row's group where that is more than a warp
    unsigned slots;                          // bit k: the sum of slot k is wanted
    void *partial;                           // [slot among the wanted][CTA or cluster][cols]
};

// Which columns a thread holds: pieces of V elements, 16 bytes of the block's type.  Piece v of thread t covers
// columns (v * threads + t) * V .. + V - 1.  ALIGNED: every row of every matrix begins where a piece may (a
// 16-byte boundary, 32 for a stream of wider elements) and is whole pieces long; else rows may begin and end
// anywhere, and 16 bytes that straddle a boundary are put together from the two aligned 16 bytes they lie in.
// Values outside the row are held as zeros.
template <int T, int V>                        // T: threads of the row, 0: the CTAs' threads
struct Columns {
    int t, cols, count;                        // count: threads of the row
    bool vectors;                              // vectors over the columns begin on 16-byte boundaries
    __device__ __forceinline__ int threads() const { return T > 0 ? T : count; }
    __device__ __forceinline__ int of(int k) const { return ((k / V) * threads() + t) * V + k % V; }
    // elements k and k + 1 (k even) with zeros outside the row
    template <bool ALIGNED, class A>
    __device__ __forceinline__ Two<A> inside(int k, Two<A> v) const
    {
        if constexpr (ALIGNED) return of(k / V * V) < cols ? v : both(A(0));
        else return two(of(k) < cols ? first(v) : A(0), of(k + 1) < cols ? second(v) : A(0));
    }
};

// A matrix of the call: rows x cols at base, rows ld apart.
template <bool ALIGNED, class TE, int E, int T, int V>
__device__ __forceinline__ void load_row(Packed<TE, E> &r, const void *base, long long rows, long long row, long long ld,
                                         const Columns<T, V> &c, bool row_ok)
{
    const TE *begin = static_cast<const TE *>(base), *p = begin + row * ld;
    constexpr int kStep = 16 / (int)sizeof(TE);
    if constexpr (ALIGNED && V == 2 * kStep) {               // a float stream beside a block of 16 bits
#pragma unroll
        for (int k = 0; k < E; k += V) {
            uint32_t *w = r.w + k * (int)sizeof(TE) / 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0u;
            if (row_ok && c.of(k) < c.cols) load32(w, p + c.of(k));
        }
        return;
    }
    // an unaligned row's pieces reach 15 bytes before it and 47 behind its last whole one
    const TE *end = begin + (rows - 1) * ld + c.cols;
    const bool inner = !ALIGNED && p - begin >= 16 / (int)sizeof(TE) && end - (p + c.cols) >= 48 / (int)sizeof(TE);
#pragma unroll
    for (int k = 0; k < E; k += kStep) {
        uint32_t *w = r.w + k * (int)sizeof(TE) / 4;
        const int j = c.of(k);
        w[0] = w[1] = w[2] = w[3] = 0u;
        if (!row_ok || j >= c.cols) continue;
        if constexpr (ALIGNED) {
            load16(w, p + j);
        } else {
            load16_any<true>(w, p + j, begin, end, inner);
            if (j + kStep > c.cols) {                        // the row ends inside: zeros from there
                Packed<TE, kStep> whole, part;
#pragma unroll
                for (int i = 0; i < 4; ++i) whole.w[i] = w[i];
                part.clear();
#pragma unroll
                for (int e = 0; e < kStep; ++e)
                    if (j + e < c.cols) part.put(e, whole.raw(e));
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = part.w[i];
            }
        }
    }
}

// The thread's elements, rounded once.
template <class TE, int E>
__device__ __forceinline__ Packed<TE, E> pack_row(const Two<Acc<TE>> (&v)[E / 2])
{
    Packed<TE, E> r;
#pragma unroll
    for (int k = 0; k < E; k += 2) r.put2(k, v[k / 2]);
    return r;
}

// Stores the thread's elements into its row (`ok`: there is one).
// Unaligned: the pieces of the row's threads in a warp are neighbours; they are exchanged through the warp's
// `stage` so that full aligned 16 bytes can be written, and the ends singly.  All threads of the warp call it.
// DIRECT: without that where a row begins aligned (the gradient, short of registers, was slower with it: 24 us against 22).
template <bool ALIGNED, class TE, int E, bool DIRECT = false, int T, int V>
__device__ __forceinline__ void store_row(void *base, long long row, long long ld, const Packed<TE, E> &v,
                                          const Columns<T, V> &c, bool ok, unsigned char *stage)
{
    TE *p = static_cast<TE *>(base) + row * ld;
    constexpr int kStep = 16 / (int)sizeof(TE), kWords = (int)sizeof(TE);      // kWords / 4 words per element
    if constexpr (ALIGNED && V == 2 * kStep) {
#pragma unroll
        for (int k = 0; k < E; k += V)
            if (ok && c.of(k) < c.cols) store32(p + c.of(k), v.w + k * kWords / 4);
    } else if constexpr (ALIGNED) {
#pragma unroll
        for (int k = 0; k < E; k += kStep)
            if (ok && c.of(k) < c.cols) store16(p + c.of(k), v.w + k * kWords / 4);
    } else {
        constexpr int kLanes = T > 0 ? T : 32;               // threads of the row in this warp
        constexpr int kChunks = V / kStep;                   // 16-byte chunks of a piece
        const int lane = (threadIdx.x & 31) % kLanes;
        if (DIRECT && ((uintptr_t)p & 15u) == 0) {           // the row begins aligned: only its end is singly
#pragma unroll
            for (int k = 0; k < E; k += kStep) {
                const int j = c.of(k);
                if (!ok || j >= c.cols) continue;
                if (j + kStep <= c.cols) {
                    store16(p + j, v.w + k * kWords / 4);
                } else {
                    Packed<TE, kStep> last;
#pragma unroll
                    for (int i = 0; i < 4; ++i) last.w[i] = v.w[k * kWords / 4 + i];
#pragma unroll
                    for (int e = 0; e < kStep; ++e)
                        if (j + e < c.cols) p[j + e] = last.raw(e);
                }
            }
            if (T == 0) return;                              // (the rows of a warp's other groups may not)
        }
        unsigned char *mine = stage + (threadIdx.x & 31) / kLanes * (kLanes * V * (int)sizeof(TE));
#pragma unroll
        for (int k = 0; k < E; k += V) {
            __syncwarp();
#pragma unroll
            for (int h = 0; h < V; h += kStep) {
                const uint32_t *w = v.w + (k + h) * kWords / 4;
                *reinterpret_cast<uint4 *>(mine + (lane * V + h) * (int)sizeof(TE)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            __syncwarp();
            const int first_col = c.of(k) - lane * V, left = c.cols - first_col;
            const bool written = DIRECT && T > 0 && ((uintptr_t)p & 15u) == 0;
            const int n = !ok || written ? 0 : left < kLanes * V ? left : kLanes * V;     // elements to write, may be negative
            TE *q = p + first_col;
            const int head = (int)(((16u - (unsigned)((uintptr_t)q & 15u)) & 15u) / sizeof(TE));
            const TE *held = reinterpret_cast<const TE *>(mine);
            if (lane < head && lane < n) q[lane] = held[lane];
            const int full = n > head ? (n - head) / kStep : 0;                  // aligned chunks
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int chunk = lane + i * kLanes;
                if (chunk >= full) continue;
                const uint4 *a = reinterpret_cast<const uint4 *>(held + chunk * kStep);
                const uint4 x = a[0], y = head ? a[1] : x;
                const uint32_t u[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                uint32_t r[4];
                straddle<(int)sizeof(TE)>(r, u, (unsigned)(head * (int)sizeof(TE)));
                store16(q + head + chunk * kStep, r);
            }
            const int last = head + full * kStep + lane;
            if (lane < kStep && last < n) q[last] = held[last];
        }
    }
}

// N elements, whole pieces or half ones, from k0 of a vector over the columns (weight, bias, scale, gate per
// column).  `wide`: the vector is float although the block has 16 bits.  Outside the row it gives zeros, or, ALIGNED, some
// value of the vector, so that no zeros have to be put where a load might not take place (the gradient of 8192 x 4096 bf16
// took 141 us with them, and takes 129): it meets a zero there, and the forward kernel does not add up what an infinite
// one or a bias makes of that.  Ordinary loads: a kernel that is launched while the one before it ends may be given that
// one's result as a vector, and the read-only path is for what no kernel writes meanwhile.
template <bool ALIGNED, class TE, int N, int T, int V>
__device__ __forceinline__ void load_vector(Two<Acc<TE>> (&o)[N / 2], const void *base, bool wide, int k0,
                                            const Columns<T, V> &c)
{
    using A = Acc<TE>;
    if (!ALIGNED && !(c.vectors && c.of((k0 + N - 1) / V * V) + V <= c.cols)) {      // not whole, or not aligned
        auto at = [&](int k) -> A {
            const int j = c.of(k);
            if (j >= c.cols) return A(0);
            if (sizeof(TE) == 2 && wide) return (A)static_cast<const float *>(base)[j];
            return widen<TE>(static_cast<const TE *>(base)[j]);
        };
#pragma unroll
        for (int k = 0; k < N; k += 2) o[k / 2] = two(at(k0 + k), at(k0 + k + 1));
    } else if (sizeof(TE) == 2 && wide) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const int j = min(c.of((k0 + k) / V * V), c.cols - V) + (k0 + k) % V;
            const float4 q = *reinterpret_cast<const float4 *>(static_cast<const float *>(base) + j);
            o[k / 2] = two((A)q.x, (A)q.y), o[k / 2 + 1] = two((A)q.z, (A)q.w);
        }
    } else {
        if constexpr (N < V) {
            static_assert(N * sizeof(TE) == 8, "half a piece");
            const int j = min(c.of(k0 / V * V), c.cols - V) + k0 % V;
            const uint2 q = *reinterpret_cast<const uint2 *>(static_cast<const TE *>(base) + j);
            Packed<TE, V> r;
            r.w[0] = q.x, r.w[1] = q.y;
            o[0] = r.get2(0), o[1] = r.get2(2);
        }
#pragma unroll
        for (int k = 0; k + V <= N; k += V) {
            const int j = min(c.of(k0 + k), c.cols - V);
            const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const TE *>(base) + j);
            Packed<TE, V> r;
            r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
#pragma unroll
            for (int e = 0; e < V; e += 2) o[(k + e) / 2] = r.get2(e);
        }
    }
}

// h = op(h, vector) over the thread's elements
template <bool ALIGNED, class TE, int E, class Cols, class Op>
__device__ __forceinline__ void with_vector(Two<Acc<TE>> (&h)[E / 2], const void *base, bool wide, const Cols &c, Op op)
{
    constexpr int P = 16 / (int)sizeof(TE);
#pragma unroll
    for (int k0 = 0; k0 < E; k0 += P) {
        Two<Acc<TE>> w[P / 2];
        load_vector<ALIGNED, TE, P>(w, base, wide, k0, c);
#pragma unroll
        for (int i = 0; i < P / 2; ++i) h[k0 / 2 + i] = op(h[k0 / 2 + i], w[i]);
    }
}

// Sums N values over the threads of a group; every thread gets the totals, added in a fixed order.
// `buf` alternates between two exchange areas, so one barrier per sum is enough: an area is written
// again only after the barrier of the sum between.
template <class A>
using Area = A[2][3][128];

__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
template <class A>
__device__ __forceinline__ void store_remote(A *local, unsigned rank, A v)      // the same variable of CTA `rank`
{
    unsigned at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(local)), "r"(rank));
    if constexpr (sizeof(A) == 4) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
    else asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(v) : "memory");
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A CTA's shared memory exists for the others of its cluster once it has started: each says so when it enters the kernel,
// and before its first sum waits until all have.  The arrival orders no memory; what stands between hides the wait.
template <int C>
__device__ __forceinline__ void say_started()
{
    if constexpr (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
template <int C>
__device__ __forceinline__ void wait_until_all_started()
{
    if constexpr (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The group a thread belongs to where groups are larger than a warp: `threads` threads (a multiple of 32) of its
// CTA, number `id` of that size, with C - 1 more CTAs.
struct Group {
    int id, threads;
};

template <int T, int C, int N, class A>
__device__ __forceinline__ void group_sum(A (&v)[N], const Group &g, Area<A> &area, int &buf)
{
    constexpr int kLanes = T > 0 ? T : 32;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
    if constexpr (T == 0) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = g.threads >> 5, first = g.id * warps;
        if constexpr (C == 1) {
            if (lane == 0) {
#pragma unroll
                for (int n = 0; n < N; ++n) area[buf][n][warp] = v[n];
            }
            asm volatile("bar.sync %0, %1;" ::"r"(g.id + 1), "r"(g.threads) : "memory");
        } else {
            if (lane < C) {
                const int at = (int)cluster_rank() * warps + warp;
#pragma unroll
                for (int n = 0; n < N; ++n) store_remote(&area[buf][n][at], (unsigned)lane, v[n]);
            }
            cluster_barrier();
        }
        constexpr int kSpan = C == 1 ? 16 : 32;              // at most 16 warps in a CTA
        const int mine = lane & (kSpan - 1);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = mine < warps * C ? area[buf][n][first + mine] : A(0);
#pragma unroll
            for (int more = 32; more < 16 * C; more += 32)
                v[n] += mine + more < warps * C ? area[buf][n][mine + more] : A(0);
        }
#pragma unroll
        for (int o = kSpan / 2; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
        buf ^= 1;
    }
}

template <int T>
constexpr int kDivisor = T > 0 ? T : 1;

template <int T, int C, int V>
__device__ __forceinline__ Columns<T, V> columns_of(int cols, bool vectors, const Group &g)
{
    if constexpr (T > 0) return {(int)(threadIdx.x % kDivisor<T>), cols, T, vectors};
    else if constexpr (C == 1) return {(int)threadIdx.x - g.id * g.threads, cols, g.threads, vectors};
    else return {(int)threadIdx.x + (int)cluster_rank() * g.threads, cols, g.threads * C, vectors};
}

// Where a warp exchanges the pieces of an unaligned store, and 16 bytes more.
template <class TS, int V, int T, bool ALIGNED>
struct Stage {
    static constexpr int kWarps = (T > 0 ? kGroupCta : kMostCta) / 32, kBytes = 32 * V * (int)sizeof(TS) + 16;
    uint4 room[kWarps * kBytes / 16];
    __device__ __forceinline__ unsigned char *of_warp()
    {
        return reinterpret_cast<unsigned char *>(room) + (threadIdx.x >> 5) * kBytes;
    }
};
template <class TS, int V, int T>
struct Stage<TS, V, T, true> {
    __device__ __forceinline__ unsigned char *of_warp() { return nullptr; }
};

// Mean (0 for the root-mean-square norm) and r = 1 / sqrt(mean((t - mean)^2) + eps) of a row, which is left
// centred.  The mean first and the centred squares after it, from registers: E[t^2] - mean^2 would
// cancel where a row's mean is large against its spread.
template <class A>
struct RowNorm {
    A mean, r;
};
// FACTORS: the row was multiplied by vectors, and an infinite one made NaN of the zeros outside the row (ALIGNED).  That is
// looked for only where a sum is not finite: the same test in all threads of the group.  (A layer norm of a row with
// an infinity is NaN anyway.)
template <bool ALIGNED, bool FACTORS, int T, int C, int E, class A, class Cols>
__device__ __forceinline__ RowNorm<A> row_norm(Two<A> (&t)[E], int kind, A eps, A inv, const Cols &c, const Group &g,
                                               Area<A> &area, int &buf)
{
    RowNorm<A> n = {A(0), A(0)};
    A s[1];
    if (kind == FO_NORM_LAYER) {
        Two<A> sum = t[0];
#pragma unroll
        for (int i = 1; i < E; ++i) sum = sum + t[i];
        s[0] = joined(sum);
        group_sum<T, C, 1, A>(s, g, area, buf);
        n.mean = s[0] * inv;
        const Two<A> minus = both(-n.mean);
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = c.template inside<ALIGNED>(2 * i, t[i] + minus);
    }
    auto squares = [&] {
        Two<A> sum = t[0] * t[0];
#pragma unroll
        for (int i = 1; i < E; ++i) sum = fused_ma(t[i], t[i], sum);
        s[0] = joined(sum);
        group_sum<T, C, 1, A>(s, g, area, buf);
    };
    squares();
    if constexpr (FACTORS && ALIGNED) {
        const bool finite = s[0] <= (sizeof(A) == 8 ? A(1.7976931348623157e308) : A(3.4028234e38f));
        if (T > 0 ? __any_sync(0xffffffffu, !finite) : !finite) {       // the groups of a warp shuffle together
#pragma unroll
            for (int i = 0; i < E; ++i) t[i] = c.template inside<ALIGNED>(2 * i, t[i]);
            squares();
        }
    }
    n.r = group_rsqrt(fused_ma(s[0], inv, eps));
    return n;
}

// What a kernel is compiled for besides types and shape; the rest it looks at at run time.
// GATE: none, one per element, or one per row or column.  LEAN: every matrix read and written, root-mean-square norms
// with weights and without biases, what transformer blocks mostly have.  Every test and every value that a form
// does not need is one less between a row's loads and its stores (8192 x 4096 bf16, gate per element: the gradient went
// from 172 us with everything at run time to 131; 8192 x 8192 with a stream of 32 bits forward from 146 to 133).
enum GateForm { kNoGate = 0, kCellGate = 1, kSharedGate = 2 };

// ------------------------------------------------------------------ forward
// BLK: there is a block output f (else the norm of the stream alone).  1024 threads share an SM with 64 registers, 1536
// with the 40 that the stream alone needs (8192 x 4096 bf16: 24 us, with 1024 threads 31).  A row's CTA does not stay for
// another row: a new one starts its loads while the others reduce.  8192 x 4096 bf16, gate per element: 61 to 65 us, 5.2
// to 5.5 TB/s; 8192 x 8192, stream of 32 bits, gate per row: 132 to 139 us, 5.8 to 6.1 TB/s (peak of a copy: 6.5).
template <class TS, class TB, int T, int C, int E, bool ALIGNED, bool BLK, int GATE, bool LEAN>
__global__ void __launch_bounds__(T > 0 ? kGroupCta : kMostCta,
                                  sizeof(Acc<TB>) == 8 ? 1 : T > 0 ? (BLK ? 4 : 6) : (BLK ? 2 : 3))
block_norm_kernel(const __grid_constant__ BlockNormParams p)
{
    using A = Acc<TB>;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int kHow = sizeof(TB) > 2 ? kExact : sizeof(TS) > 2 ? kClose : kRough;      // h has the stream's type
    constexpr bool kAny = !LEAN;
    __shared__ Area<A> area;
    __shared__ Stage<TS, V, T, ALIGNED> stages;
    unsigned char *const stage = stages.of_warp();
    int buf = 0;
    const long long row = T > 0 ? (long long)blockIdx.x * (kGroupCta / kDivisor<T>) + threadIdx.x / kDivisor<T>
                                : blockIdx.x / C;
    const bool ok = row < p.rows;
    const Group group = {0, (int)blockDim.x};
    const Columns<T, V> c = columns_of<T, C, V>(p.cols, p.vectors != 0, group);
    const bool wide = p.wide_vec != 0;
    const A inv = A(p.inv_cols);
    const auto times = [](Two<A> h, Two<A> w) { return h * w; };
    const auto plus = [](Two<A> h, Two<A> b) { return h + b; };

    say_started<C>();
    wait_for_earlier();
    let_later_start();
    Packed<TS, E> xr;
    Packed<TB, E> fr, gr;
    if (BLK) load_row<ALIGNED, TB, E>(fr, p.f, p.rows, row, p.ld_f, c, ok);
    if (!BLK || !kAny || p.x) load_row<ALIGNED, TS, E>(xr, p.x, p.rows, row, p.ld_x, c, ok);
    else xr.clear();
    if (BLK && GATE == kCellGate) load_row<ALIGNED, TB, E>(gr, p.gate, p.rows, row, p.ld_gate, c, ok);
    wait_until_all_started<C>();

    const int post_kind = kAny ? p.post.kind : FO_NORM_RMS, pre_kind = kAny ? p.pre.kind : FO_NORM_RMS;
    RowNorm<A> post = {A(0), A(0)}, pre = {A(0), A(0)};
    Two<A> h[E / 2];
    if constexpr (BLK) {
        A scale = A(p.scale);
#pragma unroll
        for (int k = 0; k < E; k += 2) h[k / 2] = fr.get2(k);
        if (post_kind != FO_NORM_NONE) {
            post = row_norm<ALIGNED, false, T, C>(h, post_kind, A(p.post.eps), inv, c, group, area, buf);
            const Two<A> r = both(post.r);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h[i] = h[i] * r;
            if (!kAny || p.post.weight) with_vector<ALIGNED, TB, E>(h, p.post.weight, wide, c, times);
            if (kAny && p.post.bias) with_vector<ALIGNED, TB, E>(h, p.post.bias, wide, c, plus);
        }
        if (GATE == kSharedGate && p.gate_access == FO_AT_ROW) {
            const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
            with_activation(p.gate_act, [&](auto kind) { scale *= first(activate<decltype(kind)::value, kHow, A>(both(g))); });
        } else if (GATE == kCellGate) {
            with_activation(p.gate_act, [&](auto kind) {
#pragma unroll
                for (int k = 0; k < E; k += 2) h[k / 2] = h[k / 2] * activate<decltype(kind)::value, kHow, A>(gr.get2(k));
            });
        } else if (GATE == kSharedGate) {
            with_activation(p.gate_act, [&](auto kind) {
                with_vector<ALIGNED, TB, E>(h, p.gate, false, c,
                                   [](Two<A> z, Two<A> g) { return z * activate<decltype(kind)::value, kHow, A>(g); });
            });
        }
        if (p.col_scale) with_vector<ALIGNED, TB, E>(h, p.col_scale, wide, c, times);
        const Two<A> k2 = both(scale);
#pragma unroll
        for (int k = 0; k < E; k += 2) h[k / 2] = fused_ma(h[k / 2], k2, xr.get2(k));
        if (kAny && ALIGNED && p.post.bias && p.cols != c.threads() * E) {  // a bias leaves no zeros outside the row
#pragma unroll
            for (int k = 0; k < E; k += 2) h[k / 2] = c.template inside<ALIGNED>(k, h[k / 2]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; k += 2) h[k / 2] = xr.get2(k);
    }
    if ((!kAny && BLK) || p.h) store_row<ALIGNED, TS, E, true>(p.h, row, p.ld_h, pack_row<TS, E>(h), c, ok, stage);
    if (pre_kind != FO_NORM_NONE) {
        // the short form has the weights on their way while the row is added up
        Packed<TB, E> early;
        const bool ready = LEAN && !wide;
        if (ready) {
#pragma unroll
            for (int k = 0; k < E; k += V) {
                const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const TB *>(p.pre.weight) + min(c.of(k), c.cols - V));
                uint32_t *w = early.w + k * (int)sizeof(TB) / 4;
                w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
            }
        }
        pre = row_norm<ALIGNED, BLK, T, C>(h, pre_kind, A(p.pre.eps), inv, c, group, area, buf);
        if (!kAny || p.y) {
            const Two<A> r = both(pre.r);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h[i] = h[i] * r;
            if (ready) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) h[i] = h[i] * early.get2(2 * i);
            } else if (!kAny || p.pre.weight) {
                with_vector<ALIGNED, TB, E>(h, p.pre.weight, wide, c, times);
            }
            if (kAny && p.pre.bias) with_vector<ALIGNED, TB, E>(h, p.pre.bias, wide, c, plus);
            store_row<ALIGNED, TB, E, true>(p.y, row, p.ld_y, pack_row<TB, E>(h), c, ok, stage);
        }
    }
    if (p.stats && ok && c.t == 0) {
        A *s = static_cast<A *>(p.stats) + row;
        s[0] = post.mean, s[p.rows] = post.r, s[2 * p.rows] = pre.mean, s[3 * p.rows] = pre.r;
    }
}

// ----------------------------------------------------------------- gradient
// The CTAs are persistent: each takes every gridDim-th row (or group of rows) and adds up what the rows give to the
// column sums.  A thread's part of those sums lies in shared memory, E values per sum in 16-byte pieces
// that neighbouring threads' pieces follow (no bank is hit twice): in registers, the two to six sums
// would leave room for so few threads that loads no longer cover their latency.
// At the end every CTA writes its line of partial sums, and column_sum_kernel adds the lines in order.
// 8192 x 4096 bf16 with a gate per element: 129 to 133 us, 4.0 to 4.2 TB/s; without a gate and with a stream of 32 bits 112
// us, 5.4 TB/s.  What bounds it is latency: warps wait for loads first (3.5 of the 12.9 cycles between a warp's instructions),
// then for shared memory, issue slots and barriers; 55 % of the issue slots are taken (75 instructions per
// element), DRAM is at 0.62 of a copy, and with two rows of 512 threads on an SM nothing is loaded during a row's sums.

constexpr int kGradE = 8;                    // elements of a row in a thread

// A thread's E values of one column sum: 16-byte pieces one behind the other, in an order that turns with the
// thread's number so that the 8 threads of one shared-memory access meet 32 different banks.
template <int E, class A>
struct SumPieces {
    static constexpr int kValues = 16 / (int)sizeof(A), kPieces = E / kValues;
    struct alignas(16) Piece {
        Two<A> v[kValues / 2];
    };
    static __device__ __forceinline__ int turned(int thread, int piece)
    {
        constexpr int kTurns = kPieces < 8 ? kPieces : 8;
        return piece ^ (thread / (8 / kTurns) % kTurns);
    }
    // elements k0 .. k0 + N - 1: v = body(pair, v)
    template <int N, class Body>
    static __device__ __forceinline__ void change(A *slot, int k0, Body body)
    {
        Piece *q = reinterpret_cast<Piece *>(slot) + threadIdx.x * kPieces;
#pragma unroll
        for (int k = 0; k < N; k += kValues) {
            Piece &at = q[turned(threadIdx.x, (k0 + k) / kValues)];
            Piece s = at;
#pragma unroll
            for (int i = 0; i < kValues / 2; ++i) s.v[i] = body(k / 2 + i, s.v[i]);
            at = s;
        }
    }
    static __device__ __forceinline__ Piece at(const A *slot, int thread, int piece)
    {
        return reinterpret_cast<const Piece *>(slot)[thread * kPieces + turned(thread, piece)];
    }
};

// 64 registers a thread, so that 1024 threads share an SM; for unaligned rows, too, although they spill (8192 x 4097: 392 us;
// with 128 registers and half the threads it took 881 when it took 405 with 64).
template <class TS, class TB, int T, int C, bool ALIGNED, bool BLK, int GATE, bool LEAN>
__global__ void __launch_bounds__(T > 0 ? kGroupCta : kMostCta,
                                  sizeof(Acc<TB>) == 8 ? 1 : T > 0 ? 4 : 2)
block_norm_grad_kernel(const __grid_constant__ BlockNormGradParams p)
{
    using A = Acc<TB>;
    constexpr int E = kGradE;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int P = 16 / (int)sizeof(A);                   // elements worked on at a time: what registers hold
    constexpr int kGroups = T > 0 ? kGroupCta / kDivisor<T> : 1;
    constexpr int kHow = sizeof(TB) > 2 ? kExact : kClose;   // sums have 32 bits or more
    constexpr int kSlope = kHow == kClose && GATE == kCellGate ? kRough : kHow;    // the gate's own gradient has the block's type
    __shared__ Area<A> area;
    __shared__ Stage<TS, V, T, ALIGNED> stages;
    unsigned char *const stage = stages.of_warp();
    extern __shared__ __align__(16) unsigned char dynamic[];
    int buf = 0;
    const Group group = {T > 0 ? 0 : (int)threadIdx.x / p.group, p.group};
    const int groups = T > 0 ? kGroups : (int)blockDim.x / p.group, cta = T > 0 ? kGroupCta : (int)blockDim.x;
    const Columns<T, V> c = columns_of<T, C, V>(p.cols, p.vectors != 0, group);
    const bool ragged = p.cols != c.threads() * E;
    const A inv = A(p.inv_cols);
    const A *stats = static_cast<const A *>(p.stats);
    const bool wide = p.wide_vec != 0;
    using Sums = SumPieces<E, A>;
    // lean: the mean is 0
    const auto centred = [](Two<A> v, Two<A> minus_mean) { return LEAN ? v : v + minus_mean; };
    constexpr bool kAny = !LEAN;
    const bool pre = !kAny || p.dy != nullptr, pre_layer = kAny && p.pre.kind == FO_NORM_LAYER;
    const bool pre_weight = !kAny || p.pre.weight != nullptr, post_weight = !kAny || p.post.weight != nullptr;
    const bool post_bias = kAny && p.post.bias != nullptr, post_layer = kAny && p.post.kind == FO_NORM_LAYER;
    const bool normed = !kAny || p.post.kind != FO_NORM_NONE;
    constexpr bool cell_gate = GATE == kCellGate;
    const bool row_gate = GATE == kSharedGate && p.gate_access == FO_AT_ROW;
    const bool col_gate = GATE == kSharedGate && p.gate_access == FO_AT_COL;
    const int n_slots = __popc(p.slots);
    A *const sums = reinterpret_cast<A *>(dynamic);
    // where each sum begins, -1: it is not wanted
    int slot_at[kGradSlots];
#pragma unroll
    for (int s = 0; s < kGradSlots; ++s)
        slot_at[s] = (s == kGateCol && GATE != kSharedGate) || (!kAny && (s == kPreB || s == kPostB)) ? -1
                     : !kAny && s == kPreW                                 ? 0
                     : !kAny && s == kPostW                                ? (BLK ? cta * E : -1)
                     : ((p.slots >> s) & 1u)                               ? __popc(p.slots & ((1u << s) - 1u)) * cta * E
                                                                           : -1;
    // adds term(i), for the pairs i of a piece from element k0, to a column sum that is wanted
    auto add = [&](int slot, int k0, auto term) {
        if (slot_at[slot] >= 0) Sums::template change<P>(sums + slot_at[slot], k0, term);
    };
    say_started<C>();
    for (int s = 0; s < n_slots; ++s)
        Sums::template change<E>(sums + s * cta * E, 0, [](int, Two<A>) { return both(A(0)); });

    wait_for_earlier();
    wait_until_all_started<C>();
    // all threads of a group, and all CTAs of a cluster, take the same number of turns: their sums meet at barriers
    for (long long row0 = (long long)(blockIdx.x / C) * groups; row0 < p.rows;
         row0 += (long long)(gridDim.x / C) * groups) {
        const long long row = row0 + (T > 0 ? (int)threadIdx.x / kDivisor<T> : group.id);
        const bool ok = row < p.rows;                        // past the end all values are zero
        Packed<TS, E> dhr, hr;
        Packed<TB, E> dyr, fr, gr;
        if (pre) {
            load_row<ALIGNED, TB, E>(dyr, p.dy, p.rows, row, p.ld_dy, c, ok);
            load_row<ALIGNED, TS, E>(hr, p.h, p.rows, row, p.ld_h, c, ok);
        }
        if (p.dh) load_row<ALIGNED, TS, E>(dhr, p.dh, p.rows, row, p.ld_dh, c, ok);
        else dhr.clear();
        if (BLK) load_row<ALIGNED, TB, E>(fr, p.f, p.rows, row, p.ld_f, c, ok);
        if (BLK && cell_gate) load_row<ALIGNED, TB, E>(gr, p.gate, p.rows, row, p.ld_gate, c, ok);

        Two<A> t[E / 2];
        if (pre) {
            const A r1 = ok ? stats[3 * p.rows + row] : A(0);
            const Two<A> minus = both(kAny && ok ? -stats[2 * p.rows + row] : A(0)), r = both(r1);
            Two<A> along = both(A(0)), level = both(A(0));
#pragma unroll
            for (int k0 = 0; k0 < E; k0 += P) {
                Two<A> n[P / 2], *a = t + k0 / 2;
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {
                    a[i] = dyr.get2(k0 + 2 * i);
                    n[i] = centred(hr.get2(k0 + 2 * i), minus) * r;
                }
                add(kPreW, k0, [&](int i, Two<A> s) { return fused_ma(a[i], n[i], s); });
                add(kPreB, k0, [&](int i, Two<A> s) { return s + a[i]; });
                if (pre_weight) {
                    Two<A> w[P / 2];
                    load_vector<ALIGNED, TB, P>(w, p.pre.weight, wide, k0, c);
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) a[i] = a[i] * w[i];
                }
#pragma unroll
                for (int i = 0; i < P / 2; ++i) along = fused_ma(a[i], n[i], along);
                if (pre_layer) {
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) level = level + a[i];
                }
            }
            A s[2] = {joined(along), A(0)};
            if (pre_layer) {
                s[1] = joined(level);
                group_sum<T, C, 2, A>(s, group, area, buf);
            } else {
                group_sum<T, C, 1, A>(*reinterpret_cast<A(*)[1]>(&s), group, area, buf);
            }
            // dh + r (a - n mean(a n) - mean(a))
            along = both(-s[0] * inv * r1 * r1), level = both(-s[1] * inv * r1);
#pragma unroll
            for (int k = 0; k < E; k += 2)
                t[k / 2] = fused_ma(t[k / 2], r, fused_ma(centred(hr.get2(k), minus), along,
                                                          LEAN ? dhr.get2(k) : dhr.get2(k) + level));
            if (ragged) {
#pragma unroll
                for (int k = 0; k < E; k += 2) t[k / 2] = c.template inside<ALIGNED>(k, t[k / 2]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < E; k += 2) t[k / 2] = dhr.get2(k);
        }
        if (!kAny || p.dx) store_row<ALIGNED, TS, E>(p.dx, row, p.ld_dx, pack_row<TS, E>(t), c, ok, stage);
        if constexpr (BLK) {
            const A r1 = ok && normed ? stats[p.rows + row] : A(1);
            const Two<A> minus = both(kAny && ok && normed ? -stats[row] : A(0)), r = both(r1), scale = both(A(p.scale));
            Two<A> row_act = both(A(1)), row_slope = both(A(0));
            if (row_gate) {
                const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
                with_activation(p.gate_act, [&](auto kind) {
                    row_act = activate_slope<decltype(kind)::value, kHow, kHow, A>(both(g), row_slope);
                });
            }
            Two<A> along = both(A(0)), level = both(A(0)), gate_sum = both(A(0));
#pragma unroll
            for (int k0 = 0; k0 < E; k0 += P) {
                Two<A> n[P / 2], z[P / 2], w[P / 2], a[P / 2], slope[P / 2], *d = t + k0 / 2;
                if (post_weight) load_vector<ALIGNED, TB, P>(w, p.post.weight, wide, k0, c);
                else
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) w[i] = both(A(1));
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {
                    n[i] = centred(fr.get2(k0 + 2 * i), minus) * r;
                    z[i] = n[i] * w[i];
                    d[i] = d[i] * scale;
                }
                if (post_bias) {
                    Two<A> b[P / 2];
                    load_vector<ALIGNED, TB, P>(b, p.post.bias, wide, k0, c);
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) z[i] = z[i] + b[i];
                }
                if (cell_gate || col_gate) {
                    Two<A> g[P / 2];
                    if (col_gate) load_vector<ALIGNED, TB, P>(g, p.gate, false, k0, c);
                    else
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) g[i] = gr.get2(k0 + 2 * i);
                    with_activation(p.gate_act, [&](auto kind) {
#pragma unroll
                        for (int i = 0; i < P / 2; ++i)
                            a[i] = activate_slope<decltype(kind)::value, kHow, kSlope, A>(g[i], slope[i]);
                    });
                } else if (row_gate) {
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) a[i] = row_act, slope[i] = row_slope;
                }
                add(kColScale, k0, [&](int i, Two<A> s) {    // without a col_scale it is the gradient at ones
                    return GATE == kNoGate ? fused_ma(d[i], z[i], s) : fused_ma(d[i] * z[i], a[i], s);
                });
                if (p.col_scale) {
                    Two<A> cs[P / 2];
                    load_vector<ALIGNED, TB, P>(cs, p.col_scale, wide, k0, c);
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) d[i] = d[i] * cs[i];
                }
                if constexpr (GATE != kNoGate) {
                    // z becomes the gate's gradient q' z act', d the normed output's q' act
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) {
                        z[i] = d[i] * z[i] * slope[i];
                        d[i] = d[i] * a[i];
                    }
                    if constexpr (cell_gate) {               // in the gate's place
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) gr.put2(k0 + 2 * i, z[i]);
                    }
                    add(kGateCol, k0, [&](int i, Two<A> s) { return s + z[i]; });
                    if (row_gate) {
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) gate_sum = gate_sum + z[i];
                    }
                }
                if (normed) {
                    add(kPostW, k0, [&](int i, Two<A> s) { return fused_ma(d[i], n[i], s); });
                    add(kPostB, k0, [&](int i, Two<A> s) { return s + d[i]; });
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) {
                        d[i] = d[i] * w[i];
                        along = fused_ma(d[i], n[i], along);
                    }
                    if (post_layer) {
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) level = level + d[i];
                    }
                }
            }
            if (cell_gate && p.dgate)
                store_row<ALIGNED, TB, E>(p.dgate, row, p.ld_dgate, gr, c, ok, stage);
            A s[3] = {joined(along), A(0), A(0)};
            if (row_gate || post_layer) {
                s[1] = joined(level), s[2] = joined(gate_sum);
                group_sum<T, C, 3, A>(s, group, area, buf);
                if (p.dgate && ok && row_gate && c.t == 0) static_cast<A *>(p.dgate)[row] = s[2];
            } else if (normed) {
                group_sum<T, C, 1, A>(*reinterpret_cast<A(*)[1]>(&s), group, area, buf);
            }
            if (normed) {
                along = both(-s[0] * inv * r1 * r1), level = both(-s[1] * inv * r1);
#pragma unroll
                for (int k = 0; k < E; k += 2)
                    t[k / 2] = fused_ma(t[k / 2], r, LEAN ? centred(fr.get2(k), minus) * along
                                                          : fused_ma(centred(fr.get2(k), minus), along, level));
            }
            if (!kAny || p.df) store_row<ALIGNED, TB, E>(p.df, row, p.ld_df, pack_row<TB, E>(t), c, ok, stage);
        }
    }

    let_later_start();                                       // the sum of the lines, which waits for this kernel's end
    // the CTA's line of every sum, its groups added in order: a thread takes the piece of one thread of all groups
    __syncthreads();
    const size_t plane = (size_t)(gridDim.x / C) * p.cols;
    A *const line = static_cast<A *>(p.partial) + (size_t)(blockIdx.x / C) * p.cols;
    const int threads = T > 0 ? T : p.group;
    for (int i = threadIdx.x; i < threads * n_slots * Sums::kPieces; i += cta) {
        const int t = i % threads, piece = i / threads % Sums::kPieces, s = i / threads / Sums::kPieces;
        typename Sums::Piece v = Sums::at(sums + s * cta * E, t, piece);
#pragma unroll 4
        for (int g = 1; g < groups; ++g) {
            const typename Sums::Piece more = Sums::at(sums + s * cta * E, g * threads + t, piece);
#pragma unroll
            for (int e = 0; e < Sums::kValues / 2; ++e) v.v[e] = v.v[e] + more.v[e];
        }
        const Columns<T, V> own = {t + (C > 1 ? (int)cluster_rank() * threads : 0), p.cols, c.count, c.vectors};
#pragma unroll
        for (int e = 0; e < Sums::kValues; ++e) {
            const int j = own.of(piece * Sums::kValues + e);
            if (j < p.cols) line[s * plane + j] = e & 1 ? second(v.v[e / 2]) : first(v.v[e / 2]);
        }
    }
}

// out[s][j] = sum over the lines of partial[s][line][j], in a fixed order: a CTA takes 32 columns of one
// sum, its 32 warps every 32nd line each (128-byte reads), then a warp adds the 32 sums of each column.
struct ColumnSumParams {
    const void *partial;
    void *out[kGradSlots];
    int lines, cols;
};

constexpr int kSumWarps = 32;

template <class A>
__global__ void __launch_bounds__(kSumWarps * 32) column_sum_kernel(const __grid_constant__ ColumnSumParams p)
{
    __shared__ A sum[kSumWarps][33];
    wait_for_earlier();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    const A *src = static_cast<const A *>(p.partial) + (size_t)blockIdx.y * p.lines * p.cols;
    A v = A(0);
    if (j < p.cols) {
#pragma unroll 8
        for (int g = warp; g < p.lines; g += kSumWarps) v += __ldcg(src + (size_t)g * p.cols + j);
    }
    sum[warp][lane] = v;
    __syncthreads();
    v = sum[lane][warp];                                     // warp w: column w
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0 && blockIdx.x * 32 + warp < (unsigned)p.cols) static_cast<A *>(p.out[blockIdx.y])[blockIdx.x * 32 + warp] = v;
}

}  // namespace fo
