// Head norms with rotation: y = R(position) norm(x) for every head's vector of queries and keys, and the gradient.
//
// A vector belongs to L lanes (a power of two up to 32), so that a warp works on 32 / L heads of one token at a time; a lane
// holds I items of two pieces of V elements each: with halves the two pieces that are turned against each other, else two
// neighbouring ones.  Everything of a vector stays in registers between its one load and its one store, and what a token's heads
// share (cosines, sines, weights) is loaded once per token or once per CTA.
#pragma once

#include "elem.cuh"
#include "../../include/fusedops_lm.h"

namespace fo {

constexpr int kHeadCta = 256;
constexpr int kHeadWarps = kHeadCta / 32;

struct HeadTensor {
    const void *x, *dy;
    void *y;                            // the gradient's dx
    fo_strides x_at, dy_at, y_at;
    int heads, kind, chunks, per_chunk; // a task: per_chunk heads of one token
    const void *weight, *bias;
    double eps;
    void *partial_w, *partial_b;        // gradient: ctas lines of dim values each, or NULL
};

struct HeadParams {
    HeadTensor t[2];
    int ctas0;                          // CTAs [0, ctas0) work on tensor 0, the rest on tensor 1
    int tokens, all_tokens;             // of a sequence, and of all of them
    int dim, lanes, pairs, axes;
    int wide_vec, table_pieces, long_positions;
    int section_end[FO_MAX_AXES];
    long long rows, ld_cos, ld_sin;
    const void *cos_table, *sin_table, *positions;
    long long position_axis, position_batch, position_token;
    double inv_dim;
};

template <class T, int V>
struct HeadPiece {
    alignas(V * sizeof(T)) T v[V];
};

template <class T, int V>
__device__ __forceinline__ HeadPiece<T, V> head_load(const T *p)
{
    HeadPiece<T, V> r;
    if constexpr (V * sizeof(T) == 16) load16(reinterpret_cast<uint32_t *>(&r), p);
    else if constexpr (V * sizeof(T) == 8 && V > 1) *reinterpret_cast<uint2 *>(&r) = *reinterpret_cast<const uint2 *>(p);
    else
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = p[j];
    return r;
}
template <class T, int V>
__device__ __forceinline__ void head_store(T *p, const Acc<T> (&f)[V])
{
    HeadPiece<T, V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = narrow<T>(f[j]);
    if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(&r);
    else if constexpr (V * sizeof(T) == 8 && V > 1) *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(&r);
    else
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = r.v[j];
}

// What a lane holds of a vector: item i is the pieces at a[i] and b[i] (-1: none), of which ta and tb are turned; its first pair.
template <int V, int I, int PAIRING>
struct HeadItems {
    int a[I], b[I], pair[I];
    bool ta[I], tb[I];
    __device__ __forceinline__ HeadItems(int lane, int lanes, int dim, int pairs)
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int u = lane + i * lanes;
            if (PAIRING == FO_PAIR_HALVES || V == 1) {
                if (u * V < pairs) {
                    a[i] = PAIRING == FO_PAIR_HALVES ? u * V : 2 * u;
                    b[i] = PAIRING == FO_PAIR_HALVES ? pairs + u * V : 2 * u + 1;
                    ta[i] = tb[i] = true;
                } else {
                    a[i] = 2 * pairs + (u * V - pairs) * 2;
                    b[i] = a[i] + V;
                    ta[i] = tb[i] = false;
                }
            } else {
                a[i] = u * 2 * V, b[i] = a[i] + V;
                ta[i] = a[i] < 2 * pairs, tb[i] = b[i] < 2 * pairs;
            }
            pair[i] = u * V;
            if (a[i] >= dim) a[i] = -1;
            if (a[i] < 0 || b[i] >= dim) b[i] = -1;
        }
    }
};

// Cosines and sines of a lane's pairs for token (b, t).
template <class A, int V, int I, int PAIRING>
__device__ __forceinline__ void head_angles(const HeadParams &p, const HeadItems<V, I, PAIRING> &at, long long b, long long t,
                                            A (&c)[I][V], A (&s)[I][V])
{
    long long row[FO_MAX_AXES];
    const long long place = b * p.position_batch + t * p.position_token;
#pragma unroll
    for (int k = 0; k < FO_MAX_AXES; ++k) {
        row[k] = -1;
        if (k < p.axes) {
            const long long at_k = place + k * p.position_axis;
            row[k] = p.long_positions ? static_cast<const long long *>(p.positions)[at_k] : static_cast<const int *>(p.positions)[at_k];
            if (row[k] >= p.rows) row[k] = -1;
        }
    }
    const A *const ct = static_cast<const A *>(p.cos_table), *const st = static_cast<const A *>(p.sin_table);
    auto row_of = [&](int pair) {
        long long r = row[0];
#pragma unroll
        for (int k = 1; k < FO_MAX_AXES; ++k)
            if (k < p.axes && pair >= p.section_end[k - 1]) r = row[k];
        return r;
    };
    constexpr int W = 16 / (int)sizeof(A) < V ? 16 / (int)sizeof(A) : V;         // table values in one load
#pragma unroll
    for (int i = 0; i < I; ++i) {
#pragma unroll
        for (int j0 = 0; j0 < V; j0 += W) {
            const int pair = at.pair[i] + j0;
            const bool on = at.a[i] >= 0 && at.ta[i] && pair < p.pairs;
            const long long r = on ? row_of(pair) : -1;
#pragma unroll
            for (int j = 0; j < W; ++j) c[i][j0 + j] = s[i][j0 + j] = A(NAN);    // a position outside the table
            if (W > 1 && p.table_pieces) {
                if (r >= 0) {
                    const HeadPiece<A, W> u = *reinterpret_cast<const HeadPiece<A, W> *>(ct + r * p.ld_cos + pair);
                    const HeadPiece<A, W> v = *reinterpret_cast<const HeadPiece<A, W> *>(st + r * p.ld_sin + pair);
#pragma unroll
                    for (int j = 0; j < W; ++j) c[i][j0 + j] = u.v[j], s[i][j0 + j] = v.v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const long long q = on && pair + j < p.pairs ? row_of(pair + j) : -1;
                    if (q >= 0) c[i][j0 + j] = ct[q * p.ld_cos + pair + j], s[i][j0 + j] = st[q * p.ld_sin + pair + j];
                }
            }
        }
    }
}

// Turns an item's pieces; SIGN -1: back.
template <int V, int PAIRING, int SIGN, class A>
__device__ __forceinline__ void head_turn(A (&a)[V], A (&b)[V], bool ta, bool tb, const A (&c)[V], const A (&s)[V])
{
    if constexpr (PAIRING == FO_PAIR_HALVES || V == 1) {
        if (!ta) return;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const A sn = SIGN < 0 ? -s[j] : s[j], x = a[j], y = b[j];
            a[j] = fused_ma(x, c[j], -(y * sn));
            b[j] = fused_ma(x, sn, y * c[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const A sa = SIGN < 0 ? -s[j / 2] : s[j / 2], sb = SIGN < 0 ? -s[(V + j) / 2] : s[(V + j) / 2];
            A x = a[j], y = a[j + 1];
            if (ta) a[j] = fused_ma(x, c[j / 2], -(y * sa)), a[j + 1] = fused_ma(x, sa, y * c[j / 2]);
            x = b[j], y = b[j + 1];
            if (tb) b[j] = fused_ma(x, c[(V + j) / 2], -(y * sb)), b[j + 1] = fused_ma(x, sb, y * c[(V + j) / 2]);
        }
    }
}

template <class A>
__device__ __forceinline__ A head_sum(A v, int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// V values of a weight or bias vector.
template <class T, int V>
__device__ __forceinline__ void head_vector(const void *p, int wide, int at, Acc<T> (&f)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j)
        f[j] = wide ? (Acc<T>)static_cast<const float *>(p)[at + j] : widen(static_cast<const T *>(p)[at + j]);
}

template <class T, int V, int I, int PAIRING>
struct HeadWork {
    using A = Acc<T>;
    using Piece = HeadPiece<T, V>;

    // n = (x - mu) r of a vector, in place; returns r
    static __device__ __forceinline__ A normalise(const HeadParams &p, const HeadItems<V, I, PAIRING> &at, int kind, A eps,
                                                  A (&a)[I][V], A (&b)[I][V])
    {
        if (kind == FO_NORM_LAYER) {
            A sum = A(0);
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) sum += a[i][j] + b[i][j];            // absent pieces are zeros
            const A mean = head_sum(sum, p.lanes) * A(p.inv_dim);
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a[i][j] = at.a[i] >= 0 ? a[i][j] - mean : A(0);
                    b[i][j] = at.b[i] >= 0 ? b[i][j] - mean : A(0);
                }
        }
        A sq = A(0);
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) sq = fused_ma(a[i][j], a[i][j], fused_ma(b[i][j], b[i][j], sq));
        const A r = group_rsqrt(fused_ma(head_sum(sq, p.lanes), A(p.inv_dim), eps));
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) a[i][j] *= r, b[i][j] *= r;
        return r;
    }
    static __device__ __forceinline__ void fetch(const T *row, const HeadItems<V, I, PAIRING> &at, Piece (&a)[I], Piece (&b)[I], bool on)
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            a[i] = b[i] = Piece{};
            if (on && at.a[i] >= 0) a[i] = head_load<T, V>(row + at.a[i]);
            if (on && at.b[i] >= 0) b[i] = head_load<T, V>(row + at.b[i]);
        }
    }
    static __device__ __forceinline__ void widen_all(const Piece (&p)[I], A (&f)[I][V])
    {
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) f[i][j] = widen(p[i].v[j]);
    }
    static __device__ __forceinline__ void store(T *row, const HeadItems<V, I, PAIRING> &at, const A (&a)[I][V], const A (&b)[I][V])
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (at.a[i] >= 0) head_store<T, V>(row + at.a[i], a[i]);
            if (at.b[i] >= 0) head_store<T, V>(row + at.b[i], b[i]);
        }
    }
    static __device__ __forceinline__ void weights(const HeadParams &p, const HeadTensor &t, const HeadItems<V, I, PAIRING> &at,
                                                   A (&a)[I][V], A (&b)[I][V])
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
#pragma unroll
            for (int j = 0; j < V; ++j) a[i][j] = b[i][j] = A(1);
            if (t.weight && at.a[i] >= 0) head_vector<T, V>(t.weight, p.wide_vec, at.a[i], a[i]);
            if (t.weight && at.b[i] >= 0) head_vector<T, V>(t.weight, p.wide_vec, at.b[i], b[i]);
        }
    }
};

template <class T, int V, int I, int PAIRING>
__global__ void __launch_bounds__(kHeadCta) head_norm_kernel(const __grid_constant__ HeadParams p)
{
    using W = HeadWork<T, V, I, PAIRING>;
    using A = Acc<T>;
    wait_for_earlier();
    const int which = blockIdx.x >= (unsigned)p.ctas0;
    const HeadTensor &t = p.t[which];
    const int lane = threadIdx.x & (p.lanes - 1), group = (threadIdx.x & 31) / p.lanes, groups = 32 / p.lanes;
    const int cta = which ? blockIdx.x - p.ctas0 : blockIdx.x, ctas = which ? gridDim.x - p.ctas0 : p.ctas0;
    const HeadItems<V, I, PAIRING> at(lane, p.lanes, p.dim, p.pairs);
    A wa[I][V], wb[I][V], c[I][V], s[I][V];
    W::weights(p, t, at, wa, wb);
    const unsigned tasks = (unsigned)p.all_tokens * (unsigned)t.chunks;
    for (unsigned task = cta * kHeadWarps + threadIdx.x / 32; task < tasks; task += ctas * kHeadWarps) {
        const unsigned token = task / (unsigned)t.chunks, h0 = (task - token * (unsigned)t.chunks) * (unsigned)t.per_chunk;
        const long long bt = token / (unsigned)p.tokens, tt = token - bt * p.tokens;
        const int h1 = min(t.heads, (int)h0 + t.per_chunk);
        const T *x = static_cast<const T *>(t.x) + bt * t.x_at.batch + tt * t.x_at.token;
        T *y = static_cast<T *>(t.y) + bt * t.y_at.batch + tt * t.y_at.token;
        typename W::Piece na[I], nb[I];
        int h = (int)h0 + group;
        W::fetch(x + h * t.x_at.head, at, na, nb, h < h1);
        if (p.pairs) head_angles<A>(p, at, bt, tt, c, s);
        for (int first = (int)h0; first < h1; first += groups, h += groups) {
            A a[I][V], b[I][V];
            W::widen_all(na, a), W::widen_all(nb, b);
            W::fetch(x + (h + groups) * t.x_at.head, at, na, nb, h + groups < h1);
            if (t.kind != FO_NORM_NONE) {
                W::normalise(p, at, t.kind, A(t.eps), a, b);
#pragma unroll
                for (int i = 0; i < I; ++i) {
#pragma unroll
                    for (int j = 0; j < V; ++j) a[i][j] *= wa[i][j], b[i][j] *= wb[i][j];
                    if (t.bias) {
                        A ba[V], bb[V];
                        if (at.a[i] >= 0) {
                            head_vector<T, V>(t.bias, p.wide_vec, at.a[i], ba);
#pragma unroll
                            for (int j = 0; j < V; ++j) a[i][j] += ba[j];
                        }
                        if (at.b[i] >= 0) {
                            head_vector<T, V>(t.bias, p.wide_vec, at.b[i], bb);
#pragma unroll
                            for (int j = 0; j < V; ++j) b[i][j] += bb[j];
                        }
                    }
                }
            }
            if (p.pairs)
#pragma unroll
                for (int i = 0; i < I; ++i) head_turn<V, PAIRING, 1>(a[i], b[i], at.ta[i], at.tb[i], c[i], s[i]);
            if (h < h1) W::store(y + h * t.y_at.head, at, a, b);
        }
    }
}

// The gradient.  Every lane keeps the sums of its own elements of dweight and dbias; at the end a CTA writes a line of
// them, and head_sum_kernel adds the lines in order.
template <class T, int V, int I, int PAIRING, bool BIAS>
__global__ void __launch_bounds__(kHeadCta) head_norm_grad_kernel(const __grid_constant__ HeadParams p)
{
    using W = HeadWork<T, V, I, PAIRING>;
    using A = Acc<T>;
    __shared__ A line[2][FO_HEAD_MAX_DIM];
    wait_for_earlier();
    const int which = blockIdx.x >= (unsigned)p.ctas0;
    const HeadTensor &t = p.t[which];
    const int lane = threadIdx.x & (p.lanes - 1), group = (threadIdx.x & 31) / p.lanes, groups = 32 / p.lanes;
    const int cta = which ? blockIdx.x - p.ctas0 : blockIdx.x, ctas = which ? gridDim.x - p.ctas0 : p.ctas0;
    const HeadItems<V, I, PAIRING> at(lane, p.lanes, p.dim, p.pairs);
    A wa[I][V], wb[I][V], c[I][V], s[I][V], da[I][V], db[I][V], ea[BIAS ? I : 1][V], eb[BIAS ? I : 1][V];
    W::weights(p, t, at, wa, wb);
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            da[i][j] = db[i][j] = A(0);
            if (BIAS) ea[i][j] = eb[i][j] = A(0);
        }
    const bool normed = t.kind != FO_NORM_NONE;
    const unsigned tasks = (unsigned)p.all_tokens * (unsigned)t.chunks;
    for (unsigned task = cta * kHeadWarps + threadIdx.x / 32; task < tasks; task += ctas * kHeadWarps) {
        const unsigned token = task / (unsigned)t.chunks, h0 = (task - token * (unsigned)t.chunks) * (unsigned)t.per_chunk;
        const long long bt = token / (unsigned)p.tokens, tt = token - bt * p.tokens;
        const int h1 = min(t.heads, (int)h0 + t.per_chunk);
        const T *x = static_cast<const T *>(t.x) + bt * t.x_at.batch + tt * t.x_at.token;
        const T *dy = static_cast<const T *>(t.dy) + bt * t.dy_at.batch + tt * t.dy_at.token;
        T *dx = static_cast<T *>(t.y) + bt * t.y_at.batch + tt * t.y_at.token;
        typename W::Piece na[I], nb[I], ga[I], gb[I];
        int h = (int)h0 + group;
        W::fetch(x + h * t.x_at.head, at, na, nb, normed && h < h1);
        W::fetch(dy + h * t.dy_at.head, at, ga, gb, h < h1);
        if (p.pairs) head_angles<A>(p, at, bt, tt, c, s);
        for (int first = (int)h0; first < h1; first += groups, h += groups) {
            A a[I][V], b[I][V], u[I][V], v[I][V];
            W::widen_all(na, a), W::widen_all(nb, b), W::widen_all(ga, u), W::widen_all(gb, v);
            const bool more = h + groups < h1;
            W::fetch(x + (h + groups) * t.x_at.head, at, na, nb, normed && more);
            W::fetch(dy + (h + groups) * t.dy_at.head, at, ga, gb, more);
            if (p.pairs)
#pragma unroll
                for (int i = 0; i < I; ++i) head_turn<V, PAIRING, -1>(u[i], v[i], at.ta[i], at.tb[i], c[i], s[i]);
            if (normed) {
                // a lane without a head has zeros throughout; its r is finite only with eps > 0, so it must not be multiplied in
                const A r = W::normalise(p, at, t.kind, h < h1 ? A(t.eps) : A(1), a, b);
                A with_n = A(0), alone = A(0);
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        da[i][j] = fused_ma(u[i][j], a[i][j], da[i][j]);
                        db[i][j] = fused_ma(v[i][j], b[i][j], db[i][j]);
                        if (BIAS) ea[i][j] += u[i][j], eb[i][j] += v[i][j];
                        u[i][j] *= wa[i][j], v[i][j] *= wb[i][j];
                        with_n = fused_ma(u[i][j], a[i][j], fused_ma(v[i][j], b[i][j], with_n));
                        alone += u[i][j] + v[i][j];
                    }
                with_n = head_sum(with_n, p.lanes) * A(p.inv_dim);
                alone = t.kind == FO_NORM_LAYER ? head_sum(alone, p.lanes) * A(p.inv_dim) : A(0);
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        u[i][j] = r * (fused_ma(-with_n, a[i][j], u[i][j]) - alone);
                        v[i][j] = r * (fused_ma(-with_n, b[i][j], v[i][j]) - alone);
                    }
            }
            if (h < h1) W::store(dx + h * t.y_at.head, at, u, v);
        }
    }
    if (!t.partial_w && !t.partial_b) return;
    // the warp's groups, then the CTA's warps one after the other
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j)
            for (int o = p.lanes; o < 32; o <<= 1) {
                da[i][j] += __shfl_xor_sync(0xffffffffu, da[i][j], o);
                db[i][j] += __shfl_xor_sync(0xffffffffu, db[i][j], o);
                if (BIAS) {
                    ea[i][j] += __shfl_xor_sync(0xffffffffu, ea[i][j], o);
                    eb[i][j] += __shfl_xor_sync(0xffffffffu, eb[i][j], o);
                }
            }
    for (int w = 0; w < kHeadWarps; ++w) {
        if ((int)threadIdx.x / 32 == w && group == 0) {
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (at.a[i] >= 0) {
                        line[0][at.a[i] + j] = (w ? line[0][at.a[i] + j] : A(0)) + da[i][j];
                        if (BIAS) line[1][at.a[i] + j] = (w ? line[1][at.a[i] + j] : A(0)) + ea[i][j];
                    }
                    if (at.b[i] >= 0) {
                        line[0][at.b[i] + j] = (w ? line[0][at.b[i] + j] : A(0)) + db[i][j];
                        if (BIAS) line[1][at.b[i] + j] = (w ? line[1][at.b[i] + j] : A(0)) + eb[i][j];
                    }
                }
        }
        __syncthreads();
    }
    for (int j = threadIdx.x; j < p.dim; j += kHeadCta) {
        if (t.partial_w) static_cast<A *>(t.partial_w)[(size_t)cta * p.dim + j] = line[0][j];
        if (BIAS && t.partial_b) static_cast<A *>(t.partial_b)[(size_t)cta * p.dim + j] = line[1][j];
    }
}

// Host: the kernel for a type, a number of elements in a piece and a vector's length; head_norm_*.cu instantiate it.
template <class T>
cudaError_t launch_head_norm(const HeadParams &p, int piece, int pairing, bool grad, bool bias, int grid, cudaStream_t st);

}  // namespace fo
