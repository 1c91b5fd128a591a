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
// so that the threads of a warp touch neighbouring elements.  A "part" is what is inside or outside as a
// whole: a piece, or one element.
template <int T, int V, bool VEC>              // T: threads of the row, over all its CTAs
struct Columns {
    static constexpr int kPart = VEC ? V : 1;
    int t, cols;
    __device__ __forceinline__ int of(int k) const { return VEC ? ((k / V) * T + t) * V + k % V : k * T + t; }
    __device__ __forceinline__ bool has(int k) const { return of(k / kPart * kPart) < cols; }
};

// for (every element k that lies in the row) body(k)
template <int E, class Cols, class Body>
__device__ __forceinline__ void for_columns(const Cols &c, Body body)
{
#pragma unroll
    for (int k0 = 0; k0 < E; k0 += Cols::kPart) {
        if (!c.has(k0)) continue;
#pragma unroll
        for (int e = 0; e < Cols::kPart; ++e) body(k0 + e);
    }
}

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

template <class TE, int E, int T, int V, bool VEC>
__device__ __forceinline__ void store_row(void *base, long long at, const Acc<TE> (&v)[E], const Columns<T, V, VEC> &c)
{
    TE *p = static_cast<TE *>(base) + at;
    if constexpr (VEC) {
        constexpr int kStep = 16 / (int)sizeof(TE);
#pragma unroll
        for (int k = 0; k < E; k += kStep) {
            if (!c.has(k)) continue;
            Packed<TE, kStep> r;
#pragma unroll
            for (int e = 0; e < kStep; e += 2) r.round2(e, v[k + e], v[k + e + 1]);
            store16(p + c.of(k), r.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (c.has(k)) p[c.of(k)] = narrow<TE>(v[k]);
    }
}

// body(k, value) for the elements of a vector over the columns (weight, bias, scale, gate per column) that
// lie in the row.  `wide`: the vector is float although the block has 16 bits.
template <class TE, int E, int T, int V, bool VEC, class Body>
__device__ __forceinline__ void for_vector(const void *base, bool wide, const Columns<T, V, VEC> &c, Body body)
{
    if constexpr (!VEC) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (!c.has(k)) continue;
            if (sizeof(TE) == 2 && wide) body(k, (Acc<TE>)__ldg(static_cast<const float *>(base) + c.of(k)));
            else body(k, widen<TE>(static_cast<const TE *>(base)[c.of(k)]));
        }
    } else if (sizeof(TE) == 2 && wide) {
#pragma unroll
        for (int k = 0; k < E; k += 4) {
            if (!c.has(k)) continue;
            const float4 q = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(base) + c.of(k)));
            body(k, (Acc<TE>)q.x), body(k + 1, (Acc<TE>)q.y), body(k + 2, (Acc<TE>)q.z), body(k + 3, (Acc<TE>)q.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; k += V) {
            if (!c.has(k)) continue;
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(static_cast<const TE *>(base) + c.of(k)));
            Packed<TE, V> r;
            r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
#pragma unroll
            for (int e = 0; e < V; ++e) body(k + e, r.get(e));
        }
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
__device__ __forceinline__ RowNorm<A> row_norm(A (&t)[E], int kind, double eps, const Cols &c, Area<A> &area, int &buf)
{
    const A inv = A(1) / A(c.cols);
    RowNorm<A> n = {A(0), A(0)};
    A s[1] = {A(0)};
    if (kind == FO_NORM_LAYER) {
        for_columns<E>(c, [&](int k) { s[0] += t[k]; });
        group_sum<T, C, 1, A>(s, area, buf);
        n.mean = s[0] * inv;
        s[0] = A(0);
        for_columns<E>(c, [&](int k) { t[k] -= n.mean; });
    }
    for_columns<E>(c, [&](int k) { s[0] = fused_ma(t[k], t[k], s[0]); });
    group_sum<T, C, 1, A>(s, area, buf);
    n.r = group_rsqrt(fused_ma(s[0], inv, A(eps)));
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

    Packed<TS, E> xr;
    Packed<TB, E> fr, gr;
    if (BLK) load_row<TB, E>(fr, p.f, row * p.ld_f, c, ok);
    if (!BLK || p.x) load_row<TS, E>(xr, p.x, row * p.ld_x, c, ok);
    else xr.clear();
    if (BLK && p.gate_access == FO_AT_CELL) load_row<TB, E>(gr, p.gate, row * p.ld_gate, c, ok);

    RowNorm<A> post = {A(0), A(0)}, pre = {A(0), A(0)};
    A h[E];
    if constexpr (BLK) {
        A scale = A(p.scale);
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = fr.get(k);
        if (p.post.kind != FO_NORM_NONE) {
            post = row_norm<T, C, E>(h, p.post.kind, p.post.eps, c, area, buf);
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] *= post.r;
            if (p.post.weight) for_vector<TB, E>(p.post.weight, wide, c, [&](int k, A w) { h[k] *= w; });
            if (p.post.bias) for_vector<TB, E>(p.post.bias, wide, c, [&](int k, A b) { h[k] += b; });
        }
        if (p.gate_access == FO_AT_ROW) {
            const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
            with_activation(p.gate_act, [&](auto kind) { scale *= activate<decltype(kind)::value, kFast, A>(g); });
        } else if (p.gate_access == FO_AT_CELL) {
            with_activation(p.gate_act, [&](auto kind) {
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] *= activate<decltype(kind)::value, kFast, A>(gr.get(k));
            });
        } else if (p.gate_access == FO_AT_COL) {
            with_activation(p.gate_act, [&](auto kind) {
                for_vector<TB, E>(p.gate, false, c,
                                  [&](int k, A g) { h[k] *= activate<decltype(kind)::value, kFast, A>(g); });
            });
        }
        if (p.col_scale) for_vector<TB, E>(p.col_scale, wide, c, [&](int k, A w) { h[k] *= w; });
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = fused_ma(h[k], scale, A(xr.get(k)));
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = A(xr.get(k));
    }
    if (p.h && ok) store_row<TS, E>(p.h, row * p.ld_h, h, c);
    if (p.pre.kind != FO_NORM_NONE) {
        pre = row_norm<T, C, E>(h, p.pre.kind, p.pre.eps, c, area, buf);
        if (p.y && ok) {
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] *= pre.r;
            if (p.pre.weight) for_vector<TB, E>(p.pre.weight, wide, c, [&](int k, A w) { h[k] *= w; });
            if (p.pre.bias) for_vector<TB, E>(p.pre.bias, wide, c, [&](int k, A b) { h[k] += b; });
            store_row<TB, E>(p.y, row * p.ld_y, h, c);
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

// Calls body(k, sum) for the thread's elements of one column sum and stores `sum` back.
template <int CTA, int E, class A, class Body>
__device__ __forceinline__ void add_columns(A *sums, int place, Body body)
{
    constexpr int kPiece = 16 / (int)sizeof(A);
    struct alignas(16) Piece {
        A v[kPiece];
    };
    Piece *q = reinterpret_cast<Piece *>(sums) + place * (E / kPiece) * CTA + threadIdx.x;
#pragma unroll
    for (int k = 0; k < E; k += kPiece) {
        Piece s = q[k / kPiece * CTA];
#pragma unroll
        for (int e = 0; e < kPiece; ++e) body(k + e, s.v[e]);
        q[k / kPiece * CTA] = s;
    }
}

template <class TS, class TB, int T, int C, int E, bool VEC, bool BLK>
__global__ void __launch_bounds__(T > 32 ? T : kGroupCta)
block_norm_grad_kernel(const __grid_constant__ BlockNormGradParams p)
{
    using A = Acc<TB>;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int kCta = T > 32 ? T : kGroupCta;
    constexpr int kGroups = kCta / T;
    constexpr bool kFast = sizeof(TB) == 2;
    __shared__ Area<A> area;
    extern __shared__ __align__(16) unsigned char dynamic[];
    int buf = 0;
    const Columns<T * C, V, VEC> c = {(int)(threadIdx.x % T + (C > 1 ? cluster_rank() * T : 0)), p.cols};
    const A inv = A(1) / A(p.cols);
    const A *stats = static_cast<const A *>(p.stats);
    const bool wide = p.wide_vec != 0;
    const int n_slots = __popc(p.slots);
    A *const sums = p.sums ? static_cast<A *>(p.sums) + (size_t)blockIdx.x * n_slots * kCta * E
                           : reinterpret_cast<A *>(dynamic);
    auto wanted = [&](int slot) { return ((p.slots >> slot) & 1u) != 0; };
    auto place = [&](int slot) { return __popc(p.slots & ((1u << slot) - 1u)); };
    for (int s = 0; s < n_slots; ++s)
        add_columns<kCta, E, A>(sums, s, [&](int, A &sum) { sum = A(0); });

    // all threads of a CTA, and all CTAs of a cluster, take the same number of turns: the sums meet at barriers
    for (long long row0 = (long long)(blockIdx.x / C) * kGroups; row0 < p.rows;
         row0 += (long long)(gridDim.x / C) * kGroups) {
        const long long row = row0 + threadIdx.x / T;
        const bool ok = row < p.rows;
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

        A t[E];
        if (p.dy) {
            const A mean = ok ? stats[2 * p.rows + row] : A(0), r = ok ? stats[3 * p.rows + row] : A(0);
            const bool layer = p.pre.kind == FO_NORM_LAYER;
            A n[E];
#pragma unroll
            for (int k = 0; k < E; ++k) {
                t[k] = dyr.get(k);
                n[k] = (A(hr.get(k)) - mean) * r;
            }
            if (wanted(kPreW) && ok)
                add_columns<kCta, E, A>(sums, place(kPreW), [&](int k, A &sum) { sum = fused_ma(t[k], n[k], sum); });
            if (wanted(kPreB) && ok) add_columns<kCta, E, A>(sums, place(kPreB), [&](int k, A &sum) { sum += t[k]; });
            if (p.pre.weight) for_vector<TB, E>(p.pre.weight, wide, c, [&](int k, A w) { t[k] *= w; });
            A s[2] = {A(0), A(0)};
            for_columns<E>(c, [&](int k) { s[0] = fused_ma(t[k], n[k], s[0]); });
            if (layer) {
                for_columns<E>(c, [&](int k) { s[1] += t[k]; });
                group_sum<T, C, 2, A>(s, area, buf);
            } else {
                A s0[1] = {s[0]};
                group_sum<T, C, 1, A>(s0, area, buf);
                s[0] = s0[0];
            }
            // dh + r (a - n along - common)
            const A along = -s[0] * inv * r, common = -s[1] * inv * r;
#pragma unroll
            for (int k = 0; k < E; ++k) t[k] = fused_ma(t[k], r, fused_ma(n[k], along, A(dhr.get(k)) + common));
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) t[k] = A(dhr.get(k));
        }
        if (p.dx && ok) store_row<TS, E>(p.dx, row * p.ld_dx, t, c);
        if constexpr (BLK) {
            const bool normed = p.post.kind != FO_NORM_NONE, row_gate = p.gate_access == FO_AT_ROW;
            const A mean = ok && normed ? stats[row] : A(0), r = ok && normed ? stats[p.rows + row] : A(1);
            const A scale = A(p.scale);
            A z[E];
#pragma unroll
            for (int k = 0; k < E; ++k) {
                t[k] *= scale;
                z[k] = (fr.get(k) - mean) * r;
            }
            if (p.post.weight) for_vector<TB, E>(p.post.weight, wide, c, [&](int k, A w) { z[k] *= w; });
            if (p.post.bias) for_vector<TB, E>(p.post.bias, wide, c, [&](int k, A b) { z[k] += b; });
            A s[3] = {A(0), A(0), A(0)};
            // with q = t: col_scale's sum takes q act z; then, q' = q col_scale, z becomes dgate = q' z act' and
            // t becomes d = q' act
            auto through_gate = [&](auto gate_at) {
                if (p.col_scale) {
                    if (wanted(kColScale) && ok)
                        add_columns<kCta, E, A>(sums, place(kColScale), [&](int k, A &sum) {
                            A slope;
                            sum = fused_ma(t[k] * z[k], gate_at(k, slope), sum);
                        });
                    for_vector<TB, E>(p.col_scale, wide, c, [&](int k, A w) { t[k] *= w; });
                }
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    A slope;
                    const A a = gate_at(k, slope);
                    z[k] *= t[k] * slope;
                    t[k] *= a;
                }
            };
            if (p.gate_access == FO_AT_CELL || p.gate_access == FO_AT_COL) {
                A g[E];
                if (p.gate_access == FO_AT_CELL) {
#pragma unroll
                    for (int k = 0; k < E; ++k) g[k] = gr.get(k);
                } else {
#pragma unroll
                    for (int k = 0; k < E; ++k) g[k] = A(0);
                    for_vector<TB, E>(p.gate, false, c, [&](int k, A v) { g[k] = v; });
                }
                with_activation(p.gate_act, [&](auto kind) {
                    through_gate([&](int k, A &slope) { return activate_slope<decltype(kind)::value, kFast, A>(g[k], slope); });
                });
                if (p.dgate && ok && p.gate_access == FO_AT_CELL) store_row<TB, E>(p.dgate, row * p.ld_dgate, z, c);
                if (wanted(kGateCol) && ok)
                    add_columns<kCta, E, A>(sums, place(kGateCol), [&](int k, A &sum) { sum += z[k]; });
            } else {
                A a = A(1), da = A(0);
                if (row_gate) {
                    const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
                    with_activation(p.gate_act, [&](auto kind) { a = activate_slope<decltype(kind)::value, kFast, A>(g, da); });
                }
                through_gate([&](int, A &slope) {
                    slope = da;
                    return a;
                });
                if (row_gate) for_columns<E>(c, [&](int k) { s[2] += z[k]; });
            }
            if (normed) {
#pragma unroll
                for (int k = 0; k < E; ++k) z[k] = (fr.get(k) - mean) * r;
                if (wanted(kPostW) && ok)
                    add_columns<kCta, E, A>(sums, place(kPostW), [&](int k, A &sum) { sum = fused_ma(t[k], z[k], sum); });
                if (wanted(kPostB) && ok) add_columns<kCta, E, A>(sums, place(kPostB), [&](int k, A &sum) { sum += t[k]; });
                if (p.post.weight) for_vector<TB, E>(p.post.weight, wide, c, [&](int k, A w) { t[k] *= w; });
                for_columns<E>(c, [&](int k) { s[0] = fused_ma(t[k], z[k], s[0]); });
                if (p.post.kind == FO_NORM_LAYER) for_columns<E>(c, [&](int k) { s[1] += t[k]; });
            }
            if (row_gate || p.post.kind == FO_NORM_LAYER) {
                group_sum<T, C, 3, A>(s, area, buf);
                if (p.dgate && ok && row_gate && c.t == 0) static_cast<A *>(p.dgate)[row] = s[2];
            } else if (normed) {
                A s0[1] = {s[0]};
                group_sum<T, C, 1, A>(s0, area, buf);
                s[0] = s0[0];
            }
            if (normed) {
                const A along = -s[0] * inv * r, common = -s[1] * inv * r;
#pragma unroll
                for (int k = 0; k < E; ++k) t[k] = fused_ma(t[k], r, fused_ma(z[k], along, common));
            }
            if (p.df && ok) store_row<TB, E>(p.df, row * p.ld_df, t, c);
        }
    }

    // the CTA's line of every sum, its groups added in order
    const size_t plane = (size_t)(gridDim.x / C) * p.cols;
    A *line = static_cast<A *>(p.partial) + (size_t)(blockIdx.x / C) * p.cols;
    if constexpr (T > 32) {
        for (int s = 0; s < n_slots; ++s, line += plane)
            add_columns<kCta, E, A>(sums, s, [&](int k, A &sum) {
                if (c.has(k)) line[c.of(k)] = sum;
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
