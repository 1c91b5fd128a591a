// Block norm and its gradient (see fusedops_train.h for the mathematics): one pass over the rows,
// each row held in registers between its sums.
//
// A row belongs to a group of T threads that hold E of its elements each.  Up to 32 threads the group
// is a part of a warp and its sums are shuffles; above, the group is the CTA, and a sum is a shuffle, one
// exchange through shared memory and a shuffle; the longest rows are split over a cluster of C CTAs, which
// exchange through each other's shared memory.  Rows are read and written once; what bounds the kernels
// is DRAM bandwidth, so the shapes only have to keep enough 16-byte loads in flight and the sums short.
#pragma once

#include <type_traits>

#include "elem.cuh"

namespace fo {

constexpr int kGroupCta = 256;               // CTA size where a group is a warp or less
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
    int vec;                                 // rows move in 16-byte pieces
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
    int vec, wide_vec;
    double inv_cols;
    int gate_access, gate_act;
    const void *dh, *dy, *h, *f, *gate, *col_scale, *stats;
    long long ld_dh, ld_dy, ld_h, ld_f, ld_gate;
    double scale;
    NormSpec post, pre;
    void *dx, *df, *dgate;
    long long ld_dx, ld_df, ld_dgate;
    unsigned slots;                          // bit k: the sum of slot k is wanted
    void *sums;                              // where the CTAs hold their sums, NULL: in shared memory
    void *partial;                           // [slot among the wanted][CTA or cluster][cols]
};

// Which columns a thread holds.  VEC, 16-byte pieces of V elements: piece v of the thread covers columns
// (v * T + t) * V .. + V - 1 and lies inside the row or outside it.  Else element k is column k * T + t,
// so that the threads of a warp touch neighbouring elements.  Values outside the row are held as zeros.
template <int T, int V, bool VEC>              // T: threads of the row, over all its CTAs
struct Columns {
    int t, cols;
    __device__ __forceinline__ int of(int k) const { return VEC ? ((k / V) * T + t) * V + k % V : k * T + t; }
    __device__ __forceinline__ bool has(int k) const { return of(VEC ? k / V * V : k) < cols; }
    // elements k and k + 1 (k even) with zeros outside the row
    template <class A>
    __device__ __forceinline__ Two<A> inside(int k, Two<A> v) const
    {
        if constexpr (VEC) return has(k) ? v : both(A(0));
        else return two(has(k) ? first(v) : A(0), has(k + 1) ? second(v) : A(0));
    }
};

template <class TE, int E, int T, int V, bool VEC>
__device__ __forceinline__ void load_row(Packed<TE, E> &r, const void *base, long long at, const Columns<T, V, VEC> &c,
                                         bool row_ok)
{
    const TE *p = static_cast<const TE *>(base) + at;
    if constexpr (VEC) {
        constexpr int kStep = 16 / (int)sizeof(TE);
#pragma unroll
        for (int k = 0; k < E; k += kStep) {
            uint32_t *w = r.w + k * (int)sizeof(TE) / 4;
            w[0] = w[1] = w[2] = w[3] = 0u;
            if (row_ok && c.has(k)) load16(w, p + c.of(k));
        }
    } else {
        r.clear();
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (row_ok && c.has(k)) r.put(k, p[c.of(k)]);
    }
}

// Stores elements k0 .. k0 + N - 1 of the thread.
template <class TE, int N, int T, int V, bool VEC>
__device__ __forceinline__ void store_piece(TE *p, const Two<Acc<TE>> *v, int k0, const Columns<T, V, VEC> &c)
{
    if constexpr (VEC) {
        constexpr int kStep = 16 / (int)sizeof(TE);
#pragma unroll
        for (int k = 0; k < N; k += kStep) {
            if (!c.has(k0 + k)) continue;
            Packed<TE, kStep> r;
#pragma unroll
            for (int e = 0; e < kStep; e += 2) r.put2(e, v[(k + e) / 2]);
            store16(p + c.of(k0 + k), r.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (c.has(k0 + k)) p[c.of(k0 + k)] = narrow<TE>(k & 1 ? second(v[k / 2]) : first(v[k / 2]));
    }
}

// N elements from k0 of a vector over the columns (weight, bias, scale, gate per column).  `wide`: the
// vector is float although the block has 16 bits.  Outside the row it gives some value of the vector,
// which meets a zero there: no zeros have to be put where a load might not take place.
template <class TE, int N, int T, int V, bool VEC>
__device__ __forceinline__ void load_vector(Two<Acc<TE>> (&o)[N / 2], const void *base, bool wide, int k0,
                                            const Columns<T, V, VEC> &c)
{
    using A = Acc<TE>;
    if constexpr (!VEC) {
        auto at = [&](int k) -> A {
            const int j = min(c.of(k), c.cols - 1);
            if (sizeof(TE) == 2 && wide) return (A)__ldg(static_cast<const float *>(base) + j);
            return widen<TE>(static_cast<const TE *>(base)[j]);
        };
#pragma unroll
        for (int k = 0; k < N; k += 2) o[k / 2] = two(at(k0 + k), at(k0 + k + 1));
    } else if (sizeof(TE) == 2 && wide) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const int j = min(c.of((k0 + k) / V * V), c.cols - V) + (k0 + k) % V;
            const float4 q = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(base) + j));
            o[k / 2] = two((A)q.x, (A)q.y), o[k / 2 + 1] = two((A)q.z, (A)q.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; k += V) {
            const int j = min(c.of(k0 + k), c.cols - V);
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(static_cast<const TE *>(base) + j));
            Packed<TE, V> r;
            r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
#pragma unroll
            for (int e = 0; e < V; e += 2) o[(k + e) / 2] = r.get2(e);
        }
    }
}

// Elements that are worked on at a time where vectors over the columns are read.
template <class TB, bool VEC>
constexpr int kPieceOf = VEC ? 16 / (int)sizeof(TB) : 16 / (int)sizeof(Acc<TB>);

// h = op(h, vector) over the thread's elements
template <class TE, int E, class Cols, class Op>
__device__ __forceinline__ void with_vector(Two<Acc<TE>> (&h)[E / 2], const void *base, bool wide, const Cols &c, Op op)
{
    constexpr int P = 16 / (int)sizeof(TE);
#pragma unroll
    for (int k0 = 0; k0 < E; k0 += P) {
        Two<Acc<TE>> w[P / 2];
        load_vector<TE, P>(w, base, wide, k0, c);
#pragma unroll
        for (int i = 0; i < P / 2; ++i) h[k0 / 2 + i] = op(h[k0 / 2 + i], w[i]);
    }
}

// Sums N values over the threads of a group; every thread gets the totals, added in a fixed order.
// `buf` alternates between two exchange areas, so one barrier per sum is enough: an area is written
// again only after the barrier of the sum between.
template <class A>
using Area = A[2][3][64];

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

template <int T, int C, int N, class A>
__device__ __forceinline__ void group_sum(A (&v)[N], Area<A> &area, int &buf)
{
    constexpr int kLanes = T < 32 ? T : 32;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
    if constexpr (T > 32) {
        constexpr int kWarps = T / 32, kValues = kWarps * C;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if constexpr (C == 1) {
            if (lane == 0) {
#pragma unroll
                for (int n = 0; n < N; ++n) area[buf][n][warp] = v[n];
            }
            __syncthreads();
        } else {
            if (lane < C) {
                const int at = (int)cluster_rank() * kWarps + warp;
#pragma unroll
                for (int n = 0; n < N; ++n) store_remote(&area[buf][n][at], (unsigned)lane, v[n]);
            }
            cluster_barrier();
        }
        constexpr int kSpan = kValues < 32 ? kValues : 32;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = area[buf][n][lane & (kSpan - 1)];
            if constexpr (kValues > 32) v[n] += area[buf][n][lane + 32];
        }
#pragma unroll
        for (int o = kSpan / 2; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
        buf ^= 1;
    }
}

// Mean (0 for the root-mean-square norm) and r = 1 / sqrt(mean((t - mean)^2) + eps) of a row, which is left
// centred.  The mean first and the centred squares after it, from registers: E[t^2] - mean^2 would
// cancel where a row's mean is large against its spread.
template <class A>
struct RowNorm {
    A mean, r;
};
template <int T, int C, int E, class A, class Cols>
__device__ __forceinline__ RowNorm<A> row_norm(Two<A> (&t)[E], int kind, A eps, A inv, const Cols &c, Area<A> &area, int &buf)
{
    RowNorm<A> n = {A(0), A(0)};
    A s[1];
    if (kind == FO_NORM_LAYER) {
        Two<A> sum = t[0];
#pragma unroll
        for (int i = 1; i < E; ++i) sum = sum + t[i];
        s[0] = joined(sum);
        group_sum<T, C, 1, A>(s, area, buf);
        n.mean = s[0] * inv;
        const Two<A> minus = both(-n.mean);
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = c.inside(2 * i, t[i] + minus);
    }
    Two<A> sum = t[0] * t[0];
#pragma unroll
    for (int i = 1; i < E; ++i) sum = fused_ma(t[i], t[i], sum);
    s[0] = joined(sum);
    group_sum<T, C, 1, A>(s, area, buf);
    n.r = group_rsqrt(fused_ma(s[0], inv, eps));
    return n;
}

// ------------------------------------------------------------------ forward
// BLK: there is a block output f (else the norm of the stream alone).
template <class TS, class TB, int T, int C, int E, bool VEC, bool BLK>
__global__ void __launch_bounds__(T > 32 ? T : kGroupCta) block_norm_kernel(const __grid_constant__ BlockNormParams p)
{
    using A = Acc<TB>;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int kCta = T > 32 ? T : kGroupCta;
    constexpr bool kFast = sizeof(TB) == 2;
    __shared__ Area<A> area;
    int buf = 0;
    const long long row = (long long)(blockIdx.x / C) * (kCta / T) + threadIdx.x / T;
    const bool ok = row < p.rows;
    const Columns<T * C, V, VEC> c = {(int)(threadIdx.x % T + (C > 1 ? cluster_rank() * T : 0)), p.cols};
    const bool wide = p.wide_vec != 0;
    const A inv = A(p.inv_cols);
    const auto times = [](Two<A> h, Two<A> w) { return h * w; };
    const auto plus = [](Two<A> h, Two<A> b) { return h + b; };

    Packed<TS, E> xr;
    Packed<TB, E> fr, gr;
    if (BLK) load_row<TB, E>(fr, p.f, row * p.ld_f, c, ok);
    if (!BLK || p.x) load_row<TS, E>(xr, p.x, row * p.ld_x, c, ok);
    else xr.clear();
    if (BLK && p.gate_access == FO_AT_CELL) load_row<TB, E>(gr, p.gate, row * p.ld_gate, c, ok);

    RowNorm<A> post = {A(0), A(0)}, pre = {A(0), A(0)};
    Two<A> h[E / 2];
    if constexpr (BLK) {
        A scale = A(p.scale);
#pragma unroll
        for (int k = 0; k < E; k += 2) h[k / 2] = fr.get2(k);
        if (p.post.kind != FO_NORM_NONE) {
            post = row_norm<T, C>(h, p.post.kind, A(p.post.eps), inv, c, area, buf);
            const Two<A> r = both(post.r);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h[i] = h[i] * r;
            if (p.post.weight) with_vector<TB, E>(h, p.post.weight, wide, c, times);
            if (p.post.bias) with_vector<TB, E>(h, p.post.bias, wide, c, plus);
        }
        if (p.gate_access == FO_AT_ROW) {
            const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
            with_activation(p.gate_act, [&](auto kind) { scale *= first(activate<decltype(kind)::value, kFast, A>(both(g))); });
        } else if (p.gate_access == FO_AT_CELL) {
            with_activation(p.gate_act, [&](auto kind) {
#pragma unroll
                for (int k = 0; k < E; k += 2) h[k / 2] = h[k / 2] * activate<decltype(kind)::value, kFast, A>(gr.get2(k));
            });
        } else if (p.gate_access == FO_AT_COL) {
            with_activation(p.gate_act, [&](auto kind) {
                with_vector<TB, E>(h, p.gate, false, c,
                                   [](Two<A> z, Two<A> g) { return z * activate<decltype(kind)::value, kFast, A>(g); });
            });
        }
        if (p.col_scale) with_vector<TB, E>(h, p.col_scale, wide, c, times);
        const Two<A> k2 = both(scale);
#pragma unroll
        for (int k = 0; k < E; k += 2) h[k / 2] = fused_ma(h[k / 2], k2, xr.get2(k));
        if (p.post.bias && p.cols != T * C * E) {            // a bias leaves no zeros outside the row
#pragma unroll
            for (int k = 0; k < E; k += 2) h[k / 2] = c.inside(k, h[k / 2]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; k += 2) h[k / 2] = xr.get2(k);
    }
    if (p.h && ok) store_piece<TS, E>(static_cast<TS *>(p.h) + row * p.ld_h, h, 0, c);
    if (p.pre.kind != FO_NORM_NONE) {
        pre = row_norm<T, C>(h, p.pre.kind, A(p.pre.eps), inv, c, area, buf);
        if (p.y && ok) {
            const Two<A> r = both(pre.r);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h[i] = h[i] * r;
            if (p.pre.weight) with_vector<TB, E>(h, p.pre.weight, wide, c, times);
            if (p.pre.bias) with_vector<TB, E>(h, p.pre.bias, wide, c, plus);
            store_piece<TB, E>(static_cast<TB *>(p.y) + row * p.ld_y, h, 0, c);
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
// would leave room for so few threads that loads no longer cover their latency.  Where shared memory does not
// hold them (many sums of long rows, float64) they lie in the CTA's own part of the workspace instead.
// At the end every CTA writes its line of partial sums, and column_sum_kernel adds the lines in order.

// The thread's elements k0 .. k0 + N - 1 of the column sum at `place`.
template <int CTA, int E, int N, class A, class Body>
__device__ __forceinline__ void column_sums(A *sums, int place, int k0, Body body)
{
    constexpr int kPiece = 16 / (int)sizeof(A);
    struct alignas(16) Piece {
        Two<A> v[kPiece / 2];
    };
    Piece *q = reinterpret_cast<Piece *>(sums) + (place * (E / kPiece) + k0 / kPiece) * CTA + threadIdx.x;
#pragma unroll
    for (int k = 0; k < N; k += kPiece) {
        Piece s = q[k / kPiece * CTA];
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) s.v[i] = body(k / 2 + i, s.v[i]);
        q[k / kPiece * CTA] = s;
    }
}

// 128 registers a thread, so that 512 threads share an SM: with 140, which the compiler would take, it is half of that.
template <class TS, class TB, int T, int C, int E, bool VEC, bool BLK>
__global__ void __launch_bounds__(T > 32 ? T : kGroupCta, sizeof(Acc<TB>) == 8 ? 1 : 512 / (T > 32 ? T : kGroupCta))
block_norm_grad_kernel(const __grid_constant__ BlockNormGradParams p)
{
    using A = Acc<TB>;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int P = kPieceOf<TB, VEC>;
    constexpr int kCta = T > 32 ? T : kGroupCta;
    constexpr int kGroups = kCta / T;
    constexpr bool kFast = sizeof(TB) == 2;
    __shared__ Area<A> area;
    extern __shared__ __align__(16) unsigned char dynamic[];
    int buf = 0;
    const Columns<T * C, V, VEC> c = {(int)(threadIdx.x % T + (C > 1 ? cluster_rank() * T : 0)), p.cols};
    const bool ragged = p.cols != T * C * E;
    const A inv = A(p.inv_cols);
    const A *stats = static_cast<const A *>(p.stats);
    const bool wide = p.wide_vec != 0;
    const int n_slots = __popc(p.slots);
    A *const sums = p.sums ? static_cast<A *>(p.sums) + (size_t)blockIdx.x * n_slots * kCta * E
                           : reinterpret_cast<A *>(dynamic);
    // adds term(i), for the pairs i of a piece from element k0, to a column sum that is wanted
    auto add = [&](int slot, int k0, auto term) {
        if (!((p.slots >> slot) & 1u)) return;
        column_sums<kCta, E, P, A>(sums, __popc(p.slots & ((1u << slot) - 1u)), k0, term);
    };
    for (int s = 0; s < n_slots; ++s) column_sums<kCta, E, E, A>(sums, s, 0, [&](int, Two<A>) { return both(A(0)); });

    // all threads of a CTA, and all CTAs of a cluster, take the same number of turns: the sums meet at barriers
    for (long long row0 = (long long)(blockIdx.x / C) * kGroups; row0 < p.rows;
         row0 += (long long)(gridDim.x / C) * kGroups) {
        const long long row = row0 + threadIdx.x / T;
        const bool ok = row < p.rows;                        // past the end all values are zero
        Packed<TS, E> dhr, hr;
        Packed<TB, E> dyr, fr, gr;
        if (p.dy) {
            load_row<TB, E>(dyr, p.dy, row * p.ld_dy, c, ok);
            load_row<TS, E>(hr, p.h, row * p.ld_h, c, ok);
        }
        if (p.dh) load_row<TS, E>(dhr, p.dh, row * p.ld_dh, c, ok);
        else dhr.clear();
        if (BLK) load_row<TB, E>(fr, p.f, row * p.ld_f, c, ok);
        if (BLK && p.gate_access == FO_AT_CELL) load_row<TB, E>(gr, p.gate, row * p.ld_gate, c, ok);

        Two<A> t[E / 2];
        if (p.dy) {
            const A r1 = ok ? stats[3 * p.rows + row] : A(0);
            const Two<A> minus = both(ok ? -stats[2 * p.rows + row] : A(0)), r = both(r1);
            Two<A> along = both(A(0)), level = both(A(0));
#pragma unroll
            for (int k0 = 0; k0 < E; k0 += P) {
                Two<A> n[P / 2], *a = t + k0 / 2;
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {
                    a[i] = dyr.get2(k0 + 2 * i);
                    n[i] = (hr.get2(k0 + 2 * i) + minus) * r;
                }
                add(kPreW, k0, [&](int i, Two<A> s) { return fused_ma(a[i], n[i], s); });
                add(kPreB, k0, [&](int i, Two<A> s) { return s + a[i]; });
                if (p.pre.weight) {
                    Two<A> w[P / 2];
                    load_vector<TB, P>(w, p.pre.weight, wide, k0, c);
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) a[i] = a[i] * w[i];
                }
#pragma unroll
                for (int i = 0; i < P / 2; ++i) along = fused_ma(a[i], n[i], along);
                if (p.pre.kind == FO_NORM_LAYER) {
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) level = level + a[i];
                }
            }
            A s[2] = {joined(along), A(0)};
            if (p.pre.kind == FO_NORM_LAYER) {
                s[1] = joined(level);
                group_sum<T, C, 2, A>(s, area, buf);
            } else {
                group_sum<T, C, 1, A>(*reinterpret_cast<A(*)[1]>(&s), area, buf);
            }
            // dh + r (a - n mean(a n) - mean(a))
            along = both(-s[0] * inv * r1 * r1), level = both(-s[1] * inv * r1);
#pragma unroll
            for (int k = 0; k < E; k += 2)
                t[k / 2] = fused_ma(t[k / 2], r, fused_ma(hr.get2(k) + minus, along, dhr.get2(k) + level));
            if (ragged) {
#pragma unroll
                for (int k = 0; k < E; k += 2) t[k / 2] = c.inside(k, t[k / 2]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < E; k += 2) t[k / 2] = dhr.get2(k);
        }
        if (p.dx && ok) store_piece<TS, E>(static_cast<TS *>(p.dx) + row * p.ld_dx, t, 0, c);
        if constexpr (BLK) {
            const bool normed = p.post.kind != FO_NORM_NONE, row_gate = p.gate_access == FO_AT_ROW;
            const A r1 = ok && normed ? stats[p.rows + row] : A(1);
            const Two<A> minus = both(ok && normed ? -stats[row] : A(0)), r = both(r1), scale = both(A(p.scale));
            Two<A> row_act = both(A(1)), row_slope = both(A(0));
            if (row_gate) {
                const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
                with_activation(p.gate_act, [&](auto kind) {
                    row_act = activate_slope<decltype(kind)::value, kFast, A>(both(g), row_slope);
                });
            }
            Two<A> along = both(A(0)), level = both(A(0)), gate_sum = both(A(0));
#pragma unroll
            for (int k0 = 0; k0 < E; k0 += P) {
                Two<A> n[P / 2], z[P / 2], w[P / 2], a[P / 2], slope[P / 2], *d = t + k0 / 2;
                if (p.post.weight) load_vector<TB, P>(w, p.post.weight, wide, k0, c);
                else
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) w[i] = both(A(1));
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {
                    n[i] = (fr.get2(k0 + 2 * i) + minus) * r;
                    z[i] = n[i] * w[i];
                    d[i] = d[i] * scale;
                }
                if (p.post.bias) {
                    Two<A> b[P / 2];
                    load_vector<TB, P>(b, p.post.bias, wide, k0, c);
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) z[i] = z[i] + b[i];
                }
                if (p.gate_access == FO_AT_CELL || p.gate_access == FO_AT_COL) {
                    Two<A> g[P / 2];
                    if (p.gate_access == FO_AT_COL) load_vector<TB, P>(g, p.gate, false, k0, c);
                    else
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) g[i] = gr.get2(k0 + 2 * i);
                    with_activation(p.gate_act, [&](auto kind) {
#pragma unroll
                        for (int i = 0; i < P / 2; ++i)
                            a[i] = activate_slope<decltype(kind)::value, kFast, A>(g[i], slope[i]);
                    });
                } else {
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) a[i] = row_act, slope[i] = row_slope;
                }
                if (p.col_scale) {
                    add(kColScale, k0, [&](int i, Two<A> s) { return fused_ma(d[i] * z[i], a[i], s); });
                    Two<A> cs[P / 2];
                    load_vector<TB, P>(cs, p.col_scale, wide, k0, c);
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) d[i] = d[i] * cs[i];
                }
                // z becomes the gate's gradient q' z act', d the normed output's q' act
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {
                    z[i] = d[i] * z[i] * slope[i];
                    d[i] = d[i] * a[i];
                }
                if (p.dgate && ok && p.gate_access == FO_AT_CELL)
                    store_piece<TB, P>(static_cast<TB *>(p.dgate) + row * p.ld_dgate, z, k0, c);
                add(kGateCol, k0, [&](int i, Two<A> s) { return s + z[i]; });
                if (row_gate) {
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) gate_sum = gate_sum + z[i];
                }
                if (normed) {
                    add(kPostW, k0, [&](int i, Two<A> s) { return fused_ma(d[i], n[i], s); });
                    add(kPostB, k0, [&](int i, Two<A> s) { return s + d[i]; });
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) {
                        d[i] = d[i] * w[i];
                        along = fused_ma(d[i], n[i], along);
                    }
                    if (p.post.kind == FO_NORM_LAYER) {
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) level = level + d[i];
                    }
                }
            }
            A s[3] = {joined(along), A(0), A(0)};
            if (row_gate || p.post.kind == FO_NORM_LAYER) {
                s[1] = joined(level), s[2] = joined(gate_sum);
                group_sum<T, C, 3, A>(s, area, buf);
                if (p.dgate && ok && row_gate && c.t == 0) static_cast<A *>(p.dgate)[row] = s[2];
            } else if (normed) {
                group_sum<T, C, 1, A>(*reinterpret_cast<A(*)[1]>(&s), area, buf);
            }
            if (normed) {
                along = both(-s[0] * inv * r1 * r1), level = both(-s[1] * inv * r1);
#pragma unroll
                for (int k = 0; k < E; k += 2)
                    t[k / 2] = fused_ma(t[k / 2], r, fused_ma(fr.get2(k) + minus, along, level));
            }
            if (p.df && ok) store_piece<TB, E>(static_cast<TB *>(p.df) + row * p.ld_df, t, 0, c);
        }
    }

    // the CTA's line of every sum, its groups added in order
    const size_t plane = (size_t)(gridDim.x / C) * p.cols;
    A *line = static_cast<A *>(p.partial) + (size_t)(blockIdx.x / C) * p.cols;
    if constexpr (T > 32) {
        for (int s = 0; s < n_slots; ++s, line += plane)
            column_sums<kCta, E, E, A>(sums, s, 0, [&](int i, Two<A> sum) {
                if (c.has(2 * i)) line[c.of(2 * i)] = first(sum);
                if (c.has(2 * i + 1)) line[c.of(2 * i + 1)] = second(sum);
                return sum;
            });
    } else {
        constexpr int kPiece = 16 / (int)sizeof(A);
        __syncthreads();
        for (int i = threadIdx.x; i < n_slots * T * E; i += kCta) {
            const int s = i / (T * E), k = i / T % E, t = i % T;
            const Columns<T, V, VEC> own = {t, p.cols};
            if (!own.has(k)) continue;
            const A *q = sums + (size_t)(s * (E / kPiece) + k / kPiece) * kCta * kPiece + t * kPiece + k % kPiece;
            A v = q[0];
            for (int g = 1; g < kGroups; ++g) v += q[g * T * kPiece];
            line[s * plane + own.of(k)] = v;
        }
    }
}

// out[s][j] = sum over the lines of partial[s][line][j], in a fixed order: a CTA takes 32 columns of one
// sum, its 8 warps every 8th line each (128-byte reads), then the warps' sums are added in order.
struct ColumnSumParams {
    const void *partial;
    void *out[kGradSlots];
    int lines, cols;
};

template <class A>
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ ColumnSumParams p)
{
    __shared__ A sum[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    const A *src = static_cast<const A *>(p.partial) + (size_t)blockIdx.y * p.lines * p.cols;
    A v = A(0);
    if (j < p.cols) {
#pragma unroll 4
        for (int g = warp; g < p.lines; g += 8) v += __ldcg(src + (size_t)g * p.cols + j);
    }
    sum[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && j < p.cols) {
#pragma unroll
        for (int g = 1; g < 8; ++g) v += sum[g][lane];
        static_cast<A *>(p.out[blockIdx.y])[j] = v;
    }
}

}  // namespace fo
