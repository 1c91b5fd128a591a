// Block norm and its gradient (see fusedops_train.h for the mathematics): one pass over the rows,
// each row held in registers between its sums.
//
// A row belongs to a group of T threads that hold E of its elements each.  Up to 32 threads the group
// is a part of a warp and its sums are shuffles; above, the group is the CTA and a sum is a shuffle,
// one exchange through shared memory and a shuffle.  Rows are read and written once; what
// bounds the kernels is DRAM bandwidth, so the shapes below only have to keep enough 16-byte loads in
// flight (T x E x matrices x bytes per CTA, several CTAs per SM) and the sums short.
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
    void *partial;                           // [slot among the wanted][CTA][cols]
};

// Which columns a thread holds.  VEC, 16-byte pieces of V elements: piece v of the thread covers columns
// (v * T + t) * V .. + V - 1 and lies inside the row or outside it.  Else element k is column k * T + t,
// so that the threads of a warp touch neighbouring elements.  A "part" is what is inside or outside as a
// whole: a piece, or one element.
template <int T, int V, bool VEC>
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
template <int T, int N, class A>
__device__ __forceinline__ void group_sum(A (&v)[N], A (*area)[3][32], int &buf)
{
    constexpr int kLanes = T < 32 ? T : 32;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
    if constexpr (T > 32) {
        constexpr int kWarps = T / 32;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) area[buf][n][warp] = v[n];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = area[buf][n][lane & (kWarps - 1)];
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1)
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
template <int E, class A, int T, int V, bool VEC>
__device__ __forceinline__ RowNorm<A> row_norm(A (&t)[E], int kind, double eps, const Columns<T, V, VEC> &c,
                                               A (*area)[3][32], int &buf)
{
    const A inv = A(1) / A(c.cols);
    RowNorm<A> n = {A(0), A(0)};
    A s[1] = {A(0)};
    if (kind == FO_NORM_LAYER) {
        for_columns<E>(c, [&](int k) { s[0] += t[k]; });
        group_sum<T, 1, A>(s, area, buf);
        n.mean = s[0] * inv;
        s[0] = A(0);
        for_columns<E>(c, [&](int k) { t[k] -= n.mean; });
    }
    for_columns<E>(c, [&](int k) { s[0] = fused_ma(t[k], t[k], s[0]); });
    group_sum<T, 1, A>(s, area, buf);
    n.r = group_rsqrt(fused_ma(s[0], inv, A(eps)));
    return n;
}

// ------------------------------------------------------------------ forward
// BLK: there is a block output f (else the norm of the stream alone).
template <class TS, class TB, int T, int E, bool VEC, bool BLK>
__global__ void __launch_bounds__(T > 32 ? T : kGroupCta) block_norm_kernel(const __grid_constant__ BlockNormParams p)
{
    using A = Acc<TB>;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int kCta = T > 32 ? T : kGroupCta;
    constexpr bool kFast = sizeof(TB) == 2;
    __shared__ A area[2][3][32];
    int buf = 0;
    const long long row = (long long)blockIdx.x * (kCta / T) + threadIdx.x / T;
    const bool ok = row < p.rows;
    const Columns<T, V, VEC> c = {(int)(threadIdx.x % T), p.cols};
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
            post = row_norm<E>(h, p.post.kind, p.post.eps, c, area, buf);
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
        pre = row_norm<E>(h, p.pre.kind, p.pre.eps, c, area, buf);
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
// FORM says which column sums a kernel can hold (E accumulators per sum and thread): the norm of
// the stream alone; a block whose norms have no bias and whose gate is not per column; everything.
enum GradForm { kGradStream = 0, kGradLean = 1, kGradAll = 2 };

template <int FORM>
__device__ __forceinline__ constexpr int slot_place(int slot)     // accumulator of a slot, -1: not held
{
    if (FORM == kGradStream) return slot == kPreW ? 0 : slot == kPreB ? 1 : -1;
    if (FORM == kGradLean) return slot == kPreW ? 0 : slot == kPostW ? 1 : slot == kColScale ? 2 : -1;
    return slot;
}
template <int FORM>
__host__ __device__ constexpr int slots_held()
{
    return FORM == kGradStream ? 2 : FORM == kGradLean ? 3 : kGradSlots;
}

template <class TS, class TB, int T, int E, bool VEC, int FORM>
__global__ void __launch_bounds__(T > 32 ? T : kGroupCta)
block_norm_grad_kernel(const __grid_constant__ BlockNormGradParams p)
{
    using A = Acc<TB>;
    constexpr int V = 16 / (int)sizeof(TB);
    constexpr int kCta = T > 32 ? T : kGroupCta;
    constexpr int kGroups = kCta / T;
    constexpr bool kFast = sizeof(TB) == 2;
    constexpr bool BLK = FORM != kGradStream;
    constexpr int NS = slots_held<FORM>();
    __shared__ A area[2][3][32];
    int buf = 0;
    const Columns<T, V, VEC> c = {(int)(threadIdx.x % T), p.cols};
    const A inv = A(1) / A(p.cols);
    const A *stats = static_cast<const A *>(p.stats);
    const bool wide = p.wide_vec != 0;

    A acc[NS][E];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int k = 0; k < E; ++k) acc[s][k] = A(0);
    auto add = [&](auto slot, int k, A v) {
        constexpr int at = slot_place<FORM>(decltype(slot)::value);
        if constexpr (at >= 0) acc[at][k] += v;
    };
    auto add_product = [&](auto slot, int k, A a, A b) {
        constexpr int at = slot_place<FORM>(decltype(slot)::value);
        if constexpr (at >= 0) acc[at][k] = fused_ma(a, b, acc[at][k]);
    };

    // all threads of a CTA take the same number of turns: the sums meet at barriers
    for (long long row0 = (long long)blockIdx.x * kGroups; row0 < p.rows; row0 += (long long)gridDim.x * kGroups) {
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
#pragma unroll
            for (int k = 0; k < E; ++k) t[k] = dyr.get(k);
            if (p.pre.weight) for_vector<TB, E>(p.pre.weight, wide, c, [&](int k, A w) { t[k] *= w; });
            A s[2] = {A(0), A(0)};
            for_columns<E>(c, [&](int k) {
                const A dy = dyr.get(k), n = (A(hr.get(k)) - mean) * r;
                s[0] = fused_ma(t[k], n, s[0]);
                s[1] += t[k];
                add_product(std::integral_constant<int, kPreW>(), k, dy, n);
                add(std::integral_constant<int, kPreB>(), k, dy);
            });
            group_sum<T, 2, A>(s, area, buf);
            // dh + r (a - n along - common)
            const A slope = -s[0] * inv * r * r, level = p.pre.kind == FO_NORM_LAYER ? -s[1] * inv * r : A(0);
#pragma unroll
            for (int k = 0; k < E; ++k)
                t[k] = fused_ma(t[k], r, fused_ma(A(hr.get(k)) - mean, slope, A(dhr.get(k)) + level));
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) t[k] = A(dhr.get(k));
        }
        if (p.dx && ok) store_row<TS, E>(p.dx, row * p.ld_dx, t, c);
        if constexpr (BLK) {
            const bool normed = p.post.kind != FO_NORM_NONE;
            const A mean = ok && normed ? stats[row] : A(0), r = ok && normed ? stats[p.rows + row] : A(1);
            const A scale = A(p.scale);
            A z[E];                                          // act(gate) z, then what of it reaches the sums
#pragma unroll
            for (int k = 0; k < E; ++k) {
                t[k] *= scale;
                z[k] = (fr.get(k) - mean) * r;
            }
            if (p.post.weight) for_vector<TB, E>(p.post.weight, wide, c, [&](int k, A w) { z[k] *= w; });
            if (p.post.bias) for_vector<TB, E>(p.post.bias, wide, c, [&](int k, A b) { z[k] += b; });
            A s[3] = {A(0), A(0), A(0)};
            // q = t; col_scale's sum takes q act z; then q' = q col_scale, dgate = q' z act', d = q' act
            auto through_gate = [&](auto gate_at) {
                if (p.col_scale) {
                    for_vector<TB, E>(p.col_scale, wide, c, [&](int k, A w) {
                        A slope;
                        const A a = gate_at(k, slope);
                        add_product(std::integral_constant<int, kColScale>(), k, t[k], a * z[k]);
                        const A q = t[k] * w;
                        z[k] *= q * slope;
                        t[k] = q * a;
                    });
                } else {
                    for_columns<E>(c, [&](int k) {
                        A slope;
                        const A a = gate_at(k, slope);
                        z[k] *= t[k] * slope;
                        t[k] *= a;
                    });
                }
            };
            if (p.gate_access < 0) {
                through_gate([&](int, A &slope) {
                    slope = A(0);
                    return A(1);
                });
            } else if (p.gate_access == FO_AT_ROW) {
                const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
                A a = A(0), da = A(0);
                with_activation(p.gate_act, [&](auto kind) { a = activate_slope<decltype(kind)::value, kFast, A>(g, da); });
                through_gate([&](int, A &slope) {
                    slope = da;
                    return a;
                });
                for_columns<E>(c, [&](int k) { s[2] += z[k]; });
            } else if (p.gate_access == FO_AT_CELL) {
                with_activation(p.gate_act, [&](auto kind) {
                    through_gate(
                        [&](int k, A &slope) { return activate_slope<decltype(kind)::value, kFast, A>(gr.get(k), slope); });
                });
                if (p.dgate && ok) store_row<TB, E>(p.dgate, row * p.ld_dgate, z, c);
            } else {
                A g[E];
                for_vector<TB, E>(p.gate, false, c, [&](int k, A v) { g[k] = v; });
                with_activation(p.gate_act, [&](auto kind) {
                    through_gate([&](int k, A &slope) { return activate_slope<decltype(kind)::value, kFast, A>(g[k], slope); });
                });
                for_columns<E>(c, [&](int k) { add(std::integral_constant<int, kGateCol>(), k, z[k]); });
            }
            if (normed) {
                for_columns<E>(c, [&](int k) {
                    add_product(std::integral_constant<int, kPostW>(), k, t[k], (fr.get(k) - mean) * r);
                    add(std::integral_constant<int, kPostB>(), k, t[k]);
                });
                if (p.post.weight) for_vector<TB, E>(p.post.weight, wide, c, [&](int k, A w) { t[k] *= w; });
                for_columns<E>(c, [&](int k) {
                    s[0] = fused_ma(t[k], (fr.get(k) - mean) * r, s[0]);
                    s[1] += t[k];
                });
            }
            if (normed || (p.dgate && p.gate_access == FO_AT_ROW)) group_sum<T, 3, A>(s, area, buf);
            if (p.dgate && ok && p.gate_access == FO_AT_ROW && c.t == 0) static_cast<A *>(p.dgate)[row] = s[2];
            if (normed) {
                const A slope = -s[0] * inv * r * r, level = p.post.kind == FO_NORM_LAYER ? -s[1] * inv * r : A(0);
#pragma unroll
                for (int k = 0; k < E; ++k) t[k] = fused_ma(t[k], r, fused_ma(fr.get(k) - mean, slope, level));
            }
            if (p.df && ok) store_row<TB, E>(p.df, row * p.ld_df, t, c);
        }
    }

    // the CTA's column sums: over its groups in a fixed order, then to its line of the partial sums
    if (!p.slots) return;
    const size_t line = (size_t)blockIdx.x * p.cols, plane = (size_t)gridDim.x * p.cols;
    A *partial = static_cast<A *>(p.partial);
    __shared__ A sum[T > 32 ? 1 : kCta / 32 * T * E];
    int wanted = 0;
    auto flush = [&](auto slot) {
        constexpr int s = decltype(slot)::value;
        constexpr int at = slot_place<FORM>(s);
        if (!((p.slots >> s) & 1u)) return;
        A *out = partial + (size_t)wanted * plane + line;
        ++wanted;
        if constexpr (at >= 0) {
            if constexpr (T > 32) {
#pragma unroll
                for (int k = 0; k < E; ++k)
                    if (c.has(k)) out[c.of(k)] = acc[at][k];
            } else {
#pragma unroll
                for (int k = 0; k < E; ++k) {
#pragma unroll
                    for (int o = T; o < 32; o <<= 1) acc[at][k] += __shfl_xor_sync(0xffffffffu, acc[at][k], o);
                }
                __syncthreads();
                if ((threadIdx.x & 31) < T) {
#pragma unroll
                    for (int k = 0; k < E; ++k)
                        if (c.has(k)) sum[(threadIdx.x >> 5) * T * E + c.of(k)] = acc[at][k];
                }
                __syncthreads();
                for (int j = threadIdx.x; j < p.cols; j += kCta) {
                    A v = A(0);
#pragma unroll
                    for (int g = 0; g < kCta / 32; ++g) v += sum[g * T * E + j];
                    out[j] = v;
                }
            }
        }
    };
    flush(std::integral_constant<int, kPreW>());
    flush(std::integral_constant<int, kPreB>());
    flush(std::integral_constant<int, kPostW>());
    flush(std::integral_constant<int, kPostB>());
    flush(std::integral_constant<int, kColScale>());
    flush(std::integral_constant<int, kGateCol>());
}

// out[s][j] = sum over the CTAs of partial[s][cta][j], in a fixed order: a CTA takes 32 columns of one
// sum, its 8 warps every 8th line each (128-byte reads), then the warps' sums are added in order.
struct ColumnSumParams {
    const void *partial;
    void *out[kGradSlots];
    int ctas, cols;
};

template <class A>
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ ColumnSumParams p)
{
    __shared__ A sum[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    const A *src = static_cast<const A *>(p.partial) + (size_t)blockIdx.y * p.ctas * p.cols;
    A v = A(0);
    if (j < p.cols) {
#pragma unroll 4
        for (int g = warp; g < p.ctas; g += 8) v += __ldcg(src + (size_t)g * p.cols + j);
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
