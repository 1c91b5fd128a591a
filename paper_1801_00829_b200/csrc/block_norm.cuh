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

// Which columns a thread holds.  16-byte pieces: piece v of the thread covers columns
// (v * T + t) * V .. + V - 1.  Single elements: element k is column k * T + t, so that the threads of a
// warp touch neighbouring elements.
template <int T, int V>
struct Columns {
    int t, cols;
    bool vec;
    __device__ __forceinline__ int of(int k) const
    {
        return vec ? ((k / V) * T + t) * V + k % V : k * T + t;
    }
    __device__ __forceinline__ bool has(int k) const     // a piece lies inside the row or outside it
    {
        return vec ? ((k / V) * T + t) * V < cols : k * T + t < cols;
    }
};

template <class TE, int T, int V, int E>
__device__ __forceinline__ void load_row(Packed<TE, E> &r, const void *base, long long at, const Columns<T, V> &c,
                                         bool row_ok)
{
    const TE *p = static_cast<const TE *>(base) + at;
    constexpr int kStep = 16 / (int)sizeof(TE);
    if (c.vec) {
#pragma unroll
        for (int k = 0; k < E; k += kStep) {
            if (row_ok && c.has(k)) load16(r.w + k * (int)sizeof(TE) / 4, p + c.of(k));
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[k * (int)sizeof(TE) / 4 + i] = 0u;
        }
    } else {
        r.clear();
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (row_ok && c.has(k)) r.put(k, p[c.of(k)]);
    }
}

template <class TE, int T, int V, int E>
__device__ __forceinline__ void store_row(void *base, long long at, const Acc<TE> (&v)[E], const Columns<T, V> &c)
{
    TE *p = static_cast<TE *>(base) + at;
    constexpr int kStep = 16 / (int)sizeof(TE);
    if (c.vec) {
#pragma unroll
        for (int k = 0; k < E; k += kStep) {
            if (!c.has(k)) continue;
            Packed<TE, kStep> r;
            r.clear();
#pragma unroll
            for (int e = 0; e < kStep; ++e) r.put(e, narrow<TE>(v[k + e]));
            store16(p + c.of(k), r.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (c.has(k)) p[c.of(k)] = narrow<TE>(v[k]);
    }
}

// A vector over the columns (weight, bias, scale, gate per column), `none` where there is none.
template <class TE, int T, int V, int E>
__device__ __forceinline__ void load_cols(Acc<TE> (&o)[E], const void *base, bool wide, const Columns<T, V> &c,
                                          Acc<TE> none)
{
    if (!base) {
#pragma unroll
        for (int k = 0; k < E; ++k) o[k] = none;
        return;
    }
    if (sizeof(TE) == 2 && wide) {
        const float *p = static_cast<const float *>(base);
#pragma unroll
        for (int k = 0; k < E; k += V) {
            if (c.vec) {
                if (!c.has(k)) continue;
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const float4 q = __ldg(reinterpret_cast<const float4 *>(p + c.of(k) + e));
                    o[k + e] = q.x, o[k + e + 1] = q.y, o[k + e + 2] = q.z, o[k + e + 3] = q.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (c.has(k + e)) o[k + e] = __ldg(p + c.of(k + e));
            }
        }
        return;
    }
    const TE *p = static_cast<const TE *>(base);
#pragma unroll
    for (int k = 0; k < E; k += V) {
        if (c.vec) {
            if (!c.has(k)) continue;
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(p + c.of(k)));
            Packed<TE, V> r;
            r.w[0] = q.x, r.w[1] = q.y, r.w[2] = q.z, r.w[3] = q.w;
#pragma unroll
            for (int e = 0; e < V; ++e) o[k + e] = r.get(e);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c.has(k + e)) o[k + e] = widen<TE>(p[c.of(k + e)]);
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

// Mean (0 for the root-mean-square norm) and 1 / sqrt(mean((t - mean)^2) + eps) of a row.  The mean
// first and the centred squares after it, from registers: E[t^2] - mean^2 would cancel where a row's
// mean is large against its spread.
template <int T, int V, int E, class A>
__device__ __forceinline__ void row_stats(const A (&t)[E], int kind, double eps, const Columns<T, V> &c,
                                          A (*area)[3][32], int &buf, A &mean, A &r)
{
    const A inv = A(1) / A(c.cols);
    A s[1] = {A(0)};
    mean = A(0);
    if (kind == FO_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < E; ++k) s[0] += c.has(k) ? t[k] : A(0);
        group_sum<T, 1, A>(s, area, buf);
        mean = s[0] * inv;
        s[0] = A(0);
    }
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const A d = c.has(k) ? t[k] - mean : A(0);
        s[0] = fused_ma(d, d, s[0]);
    }
    group_sum<T, 1, A>(s, area, buf);
    r = group_rsqrt(fused_ma(s[0], inv, A(eps)));
}

// ------------------------------------------------------------------ forward
// BLK: there is a block output f (else the norm of the stream alone).
template <class TS, class TB, int T, int E, bool BLK>
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
    const Columns<T, V> c = {(int)(threadIdx.x % T), p.cols, p.vec != 0};

    Packed<TS, E> xr;
    Packed<TB, E> fr, gr;
    if (BLK) load_row<TB, T, V, E>(fr, p.f, row * p.ld_f, c, ok);
    if (p.x) load_row<TS, T, V, E>(xr, p.x, row * p.ld_x, c, ok);
    else xr.clear();
    if (BLK && p.gate_access == FO_AT_CELL) load_row<TB, T, V, E>(gr, p.gate, row * p.ld_gate, c, ok);

    A stat[4] = {A(0), A(0), A(0), A(0)};
    A h[E];
    if constexpr (BLK) {
        A w[E];
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = fr.get(k);
        if (p.post.kind != FO_NORM_NONE) {
            row_stats<T, V, E, A>(h, p.post.kind, p.post.eps, c, area, buf, stat[0], stat[1]);
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] = (h[k] - stat[0]) * stat[1];
            if (p.post.weight) {
                load_cols<TB, T, V, E>(w, p.post.weight, p.wide_vec, c, A(1));
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] *= w[k];
            }
            if (p.post.bias) {
                load_cols<TB, T, V, E>(w, p.post.bias, p.wide_vec, c, A(0));
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] += w[k];
            }
        }
        if (p.gate_access == FO_AT_CELL) {
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] *= activate<kFast, A>(p.gate_act, gr.get(k));
        } else if (p.gate_access == FO_AT_COL) {
            load_cols<TB, T, V, E>(w, p.gate, false, c, A(0));
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] *= activate<kFast, A>(p.gate_act, w[k]);
        } else if (p.gate_access == FO_AT_ROW) {
            const A g = ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate]) : A(0);
            const A a = activate<kFast, A>(p.gate_act, g);
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] *= a;
        }
        if (p.col_scale) {
            load_cols<TB, T, V, E>(w, p.col_scale, p.wide_vec, c, A(1));
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] *= w[k];
        }
        const A scale = A(p.scale);
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = fused_ma(h[k], scale, A(xr.get(k)));
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = A(xr.get(k));
    }
    if (p.h && ok) store_row<TS, T, V, E>(p.h, row * p.ld_h, h, c);
    if (p.pre.kind != FO_NORM_NONE) {
        A w[E];
        row_stats<T, V, E, A>(h, p.pre.kind, p.pre.eps, c, area, buf, stat[2], stat[3]);
        if (p.y) {
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] = (h[k] - stat[2]) * stat[3];
            if (p.pre.weight) {
                load_cols<TB, T, V, E>(w, p.pre.weight, p.wide_vec, c, A(1));
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] *= w[k];
            }
            if (p.pre.bias) {
                load_cols<TB, T, V, E>(w, p.pre.bias, p.wide_vec, c, A(0));
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] += w[k];
            }
            if (ok) store_row<TB, T, V, E>(p.y, row * p.ld_y, h, c);
        }
    }
    if (p.stats && ok && c.t == 0) {
        A *s = static_cast<A *>(p.stats);
#pragma unroll
        for (int k = 0; k < 4; ++k) s[(long long)k * p.rows + row] = stat[k];
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

template <class TS, class TB, int T, int E, int FORM>
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
    const Columns<T, V> c = {(int)(threadIdx.x % T), p.cols, p.vec != 0};
    const A inv = A(1) / A(p.cols);
    const A *stats = static_cast<const A *>(p.stats);

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
            load_row<TB, T, V, E>(dyr, p.dy, row * p.ld_dy, c, ok);
            load_row<TS, T, V, E>(hr, p.h, row * p.ld_h, c, ok);
        }
        if (p.dh) load_row<TS, T, V, E>(dhr, p.dh, row * p.ld_dh, c, ok);
        else dhr.clear();
        if (BLK) load_row<TB, T, V, E>(fr, p.f, row * p.ld_f, c, ok);
        if (BLK && p.gate_access == FO_AT_CELL) load_row<TB, T, V, E>(gr, p.gate, row * p.ld_gate, c, ok);

        A t[E], w[E];
#pragma unroll
        for (int k = 0; k < E; ++k) t[k] = A(dhr.get(k));
        if (p.dy) {
            const A mean = ok ? stats[2 * p.rows + row] : A(0), r = ok ? stats[3 * p.rows + row] : A(0);
            load_cols<TB, T, V, E>(w, p.pre.weight, p.wide_vec, c, A(1));
            A s[2] = {A(0), A(0)};
#pragma unroll
            for (int k = 0; k < E; ++k) {
                if (!c.has(k)) continue;
                const A dy = dyr.get(k), n = (A(hr.get(k)) - mean) * r, a = dy * w[k];
                s[0] = fused_ma(a, n, s[0]);
                s[1] += a;
                add_product(std::integral_constant<int, kPreW>(), k, dy, n);
                add(std::integral_constant<int, kPreB>(), k, dy);
            }
            group_sum<T, 2, A>(s, area, buf);
            const A along = s[0] * inv, common = p.pre.kind == FO_NORM_LAYER ? s[1] * inv : A(0);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const A n = (A(hr.get(k)) - mean) * r;
                t[k] = fused_ma(r, fused_ma(-n, along, A(dyr.get(k)) * w[k] - common), t[k]);
            }
        }
        if (p.dx && ok) store_row<TS, T, V, E>(p.dx, row * p.ld_dx, t, c);
        if constexpr (BLK) {
            const bool normed = p.post.kind != FO_NORM_NONE;
            const A mean = ok && normed ? stats[row] : A(0), r = ok ? (normed ? stats[p.rows + row] : A(1)) : A(0);
            A gate = A(1), slope = A(0);
            if (p.gate_access == FO_AT_ROW)
                gate = activate_slope<kFast, A>(p.gate_act, ok ? widen<TB>(static_cast<const TB *>(p.gate)[row * p.ld_gate])
                                                              : A(0), slope);
            A cs[E], g[E], b[E];
            load_cols<TB, T, V, E>(w, p.post.weight, p.wide_vec, c, A(1));
            load_cols<TB, T, V, E>(b, p.post.bias, p.wide_vec, c, A(0));
            load_cols<TB, T, V, E>(cs, p.col_scale, p.wide_vec, c, A(1));
            if (p.gate_access == FO_AT_COL) load_cols<TB, T, V, E>(g, p.gate, false, c, A(0));
            if (p.gate_access == FO_AT_CELL) {
#pragma unroll
                for (int k = 0; k < E; ++k) g[k] = gr.get(k);
            }
            A s[3] = {A(0), A(0), A(0)};
            const A scale = A(p.scale);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                if (!c.has(k)) continue;
                const A n = (fr.get(k) - mean) * r;
                const A z = fused_ma(n, w[k], b[k]);
                A a = gate, da = slope;
                if (p.gate_access == FO_AT_CELL || p.gate_access == FO_AT_COL)
                    a = activate_slope<kFast, A>(p.gate_act, g[k], da);
                const A q = t[k] * scale;
                add_product(std::integral_constant<int, kColScale>(), k, q, a * z);
                const A qc = q * cs[k];
                const A dg = qc * z * da;
                add(std::integral_constant<int, kGateCol>(), k, dg);
                s[2] += dg;
                g[k] = dg;
                const A d = qc * a;
                add_product(std::integral_constant<int, kPostW>(), k, d, n);
                add(std::integral_constant<int, kPostB>(), k, d);
                t[k] = d;
                const A aw = d * w[k];
                s[0] = fused_ma(aw, n, s[0]);
                s[1] += aw;
            }
            if (p.dgate && ok && p.gate_access == FO_AT_CELL)
                store_row<TB, T, V, E>(p.dgate, row * p.ld_dgate, g, c);
            if (normed || (p.dgate && p.gate_access == FO_AT_ROW)) group_sum<T, 3, A>(s, area, buf);
            if (p.dgate && ok && p.gate_access == FO_AT_ROW && c.t == 0) static_cast<A *>(p.dgate)[row] = s[2];
            if (normed) {
                const A along = s[0] * inv, common = p.post.kind == FO_NORM_LAYER ? s[1] * inv : A(0);
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    const A n = (fr.get(k) - mean) * r;
                    t[k] = r * fused_ma(-n, along, t[k] * w[k] - common);
                }
            }
            if (p.df && ok) store_row<TB, T, V, E>(p.df, row * p.ld_df, t, c);
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
