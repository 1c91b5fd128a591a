// Head norms with rotation: y = R(position) norm(x) for every head's vector of queries and keys, and the gradient.
//
// A vector belongs to L lanes (a power of two up to 32), so that a warp works on 32 / L vectors at a time (a turn): on a head of as many
// tokens or on as many heads of one token; a
// lane holds I items of two pieces of V elements each: with halves the two pieces that are turned against each other, else two
// neighbouring ones.  Everything of a vector stays in registers between its one load and its one store, and what a token's heads
// share (cosines, sines, weights) is loaded once per token or once per CTA.  A lane's pieces of the next turns are on their way to
// a ring of its own in shared memory (asynchronous copies that no other thread has to wait for).
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
    int heads, kind;
    int blocks, turns, each;            // blocks of tokens, turns of a block and of a warp
    const void *weight, *bias;
    double eps;
    void *partial_w, *partial_b;        // gradient: ctas lines of dim values each, or NULL
};

struct HeadParams {
    HeadTensor t[2];
    int ctas0;                          // CTAs [0, ctas0) work on tensor 0, the rest on tensor 1
    int tokens, all_tokens;             // of a sequence, and of all of them
    int wide;                           // a block is as many tokens as a warp has groups; else it is one
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
    if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4 *>(&r) = *reinterpret_cast<const uint4 *>(p);
    else if constexpr (V * sizeof(T) == 8 && V > 1) *reinterpret_cast<uint2 *>(&r) = *reinterpret_cast<const uint2 *>(p);
    else
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = p[j];
    return r;
}

// The unit of arithmetic: two neighbouring values in one register pair, or a single one where elements move alone.
__device__ __forceinline__ float joined(float v) { return v; }
__device__ __forceinline__ double joined(double v) { return v; }
template <class U, class A>
__device__ __forceinline__ U head_all(A v)
{
    if constexpr (std::is_same<U, A>::value) return v;
    else return both(v);
}

// What a lane holds of a vector: item i is the pieces at a[i] and b[i] (-1: none), of which ta and tb are turned.  Pieces that are
// not turned against each other are dealt out so that neighbouring lanes have neighbouring pieces.
template <int V, int I, int PAIRING>
struct HeadItems {
    static constexpr bool HALVES = PAIRING == FO_PAIR_HALVES || V == 1;
    int a[I], b[I];
    int pairs;
    __device__ __forceinline__ HeadItems(int lane, int lanes, int dim, int pairs_) : pairs(pairs_)
    {
        const int turned = HALVES ? pairs / V : 0;             // items whose pieces are halves of pairs
        const int rest = (dim + V - 1) / V - 2 * turned, half = (rest + 1) / 2;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int u = lane + i * lanes;
            if (u < turned) {
                a[i] = PAIRING == FO_PAIR_HALVES ? u * V : 2 * u;
                b[i] = PAIRING == FO_PAIR_HALVES ? pairs + u * V : 2 * u + 1;
            } else {
                a[i] = (2 * turned + u - turned) * V, b[i] = a[i] + half * V;
                if (u - turned >= half) a[i] = -1;
                if (a[i] < 0 || b[i] >= dim) b[i] = -1;
            }
        }
    }
    __device__ __forceinline__ bool ta(int i) const { return a[i] >= 0 && a[i] < 2 * pairs; }
    __device__ __forceinline__ bool tb(int i) const { return b[i] >= 0 && b[i] < 2 * pairs; }
    // the first pair of a piece
    __device__ __forceinline__ int pair_a(int i) const { return PAIRING == FO_PAIR_HALVES ? a[i] : a[i] / 2; }
    __device__ __forceinline__ int pair_b(int i) const { return b[i] / 2; }
};

// The rows of the tables at which a token's positions lie; -1: outside, or there is no such token (and then perhaps no row either).
struct HeadRows {
    int at[FO_MAX_AXES];
};
__device__ __forceinline__ HeadRows head_rows(const HeadParams &p, unsigned token)
{
    HeadRows r = {{-1, -1, -1, -1}};
    static_assert(FO_MAX_AXES == 4, "a row for each axis");
    if (token >= (unsigned)p.all_tokens) return r;
    const long long b = token / (unsigned)p.tokens, t = token - b * p.tokens;
    const long long place = b * p.position_batch + t * p.position_token;
    const auto row_at = [&](long long at) {
        const long long row = p.long_positions ? static_cast<const long long *>(p.positions)[at] : static_cast<const int *>(p.positions)[at];
        return row >= 0 && row < p.rows ? (int)row : -1;
    };
    r.at[0] = row_at(place);
    if (p.axes > 1)
#pragma unroll
        for (int k = 1; k < FO_MAX_AXES; ++k) r.at[k] = k < p.axes ? row_at(place + k * p.position_axis) : -1;
    return r;
}

template <class T, int V, int I, int PAIRING>
struct HeadWork {
    using A = Acc<T>;
    using U = typename std::conditional<V == 1, A, Two<A>>::type;
    using Piece = HeadPiece<T, V>;
    using Items = HeadItems<V, I, PAIRING>;
    static constexpr int N = V == 1 ? 1 : V / 2;             // units of a piece
    static constexpr bool HALVES = PAIRING == FO_PAIR_HALVES || V == 1;

    // Cosines and sines of a lane's pairs.  Halves: of the units of a piece, with the sine's negative; neighbours: of every unit, which is a
    // pair, of both pieces (turned value by value: two products and two sums, as many instructions as packed with the two values
    // swapped, and half the registers).
    using Angle = typename std::conditional<HALVES, U, A>::type;
    struct Angles {
        Angle c[I][HALVES ? N : 2 * N], s[I][HALVES ? N : 2 * N], minus[HALVES ? I : 1][N];
    };
    // n values of both tables from `pair` on, of which the first `there` exist; NaN outside the table
    template <int M>
    static __device__ __forceinline__ void table(const HeadParams &p, const HeadRows &rows, int pair, bool on, A (&c)[M], A (&s)[M])
    {
        const A *const ct = static_cast<const A *>(p.cos_table), *const st = static_cast<const A *>(p.sin_table);
        constexpr int W = 16 / (int)sizeof(A) < M ? 16 / (int)sizeof(A) : M;         // values in one load
        auto row_of = [&](int q) {
            int r = rows.at[0];
            if (p.axes > 1)
#pragma unroll
                for (int k = 1; k < FO_MAX_AXES; ++k)
                    if (k < p.axes && q >= p.section_end[k - 1]) r = rows.at[k];
            return r;
        };
#pragma unroll
        for (int j0 = 0; j0 < M; j0 += W) {
            const int q0 = pair + j0;
#pragma unroll
            for (int j = 0; j < W; ++j) c[j0 + j] = s[j0 + j] = A(NAN);
            if (W > 1 && p.table_pieces) {
                const int r = row_of(q0);
                if (on && q0 < p.pairs && r >= 0) {
                    const HeadPiece<A, W> u = head_load<A, W>(ct + r * p.ld_cos + q0), v = head_load<A, W>(st + r * p.ld_sin + q0);
#pragma unroll
                    for (int j = 0; j < W; ++j) c[j0 + j] = u.v[j], s[j0 + j] = v.v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const int r = row_of(q0 + j);
                    if (on && q0 + j < p.pairs && r >= 0) c[j0 + j] = ct[r * p.ld_cos + q0 + j], s[j0 + j] = st[r * p.ld_sin + q0 + j];
                }
            }
        }
    }
    template <int SIGN>
    static __device__ __forceinline__ void angles(const HeadParams &p, const Items &at, const HeadRows &rows, Angles &g)
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (V == 1) {
                A c[1], s[1];
                table<1>(p, rows, at.pair_a(i), at.ta(i), c, s);
                g.c[i][0] = c[0], g.s[i][0] = A(SIGN) * s[0], g.minus[i][0] = A(-SIGN) * s[0];
            } else if constexpr (HALVES) {
                A c[V], s[V];
                table<V>(p, rows, at.pair_a(i), at.ta(i), c, s);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    g.c[i][j] = two(c[2 * j], c[2 * j + 1]);
                    g.s[i][j] = two(A(SIGN) * s[2 * j], A(SIGN) * s[2 * j + 1]), g.minus[i][j] = two(A(-SIGN) * s[2 * j], A(-SIGN) * s[2 * j + 1]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    A c[N], s[N];
                    table<N>(p, rows, k ? at.pair_b(i) : at.pair_a(i), k ? at.tb(i) : at.ta(i), c, s);
#pragma unroll
                    for (int j = 0; j < N; ++j) g.c[i][k * N + j] = c[j], g.s[i][k * N + j] = A(SIGN) * s[j];
                }
            }
        }
    }
    // Asks for what angles() will load of the next task's token.
    static __device__ __forceinline__ void expect(const HeadParams &p, const Items &at, const HeadRows &rows)
    {
        const A *const ct = static_cast<const A *>(p.cos_table), *const st = static_cast<const A *>(p.sin_table);
        auto ask = [&](int pair) {
            int r = rows.at[0];
            if (p.axes > 1)
#pragma unroll
                for (int k = 1; k < FO_MAX_AXES; ++k)
                    if (k < p.axes && pair >= p.section_end[k - 1]) r = rows.at[k];
            if (r < 0) return;
            asm volatile("prefetch.global.L1 [%0];" ::"l"(ct + r * p.ld_cos + pair));
            asm volatile("prefetch.global.L1 [%0];" ::"l"(st + r * p.ld_sin + pair));
        };
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (at.ta(i)) ask(at.pair_a(i));
            if (!HALVES && at.tb(i)) ask(at.pair_b(i));
        }
    }
    static __device__ __forceinline__ U turned(U u, A c, A s)
    {
        const A x = part(u, 0), y = part(u, 1);
        if constexpr (V == 1) return u;
        else return two(fused_ma(-y, s, x * c), fused_ma(x, s, y * c));
    }
    // Turns a lane's pieces.
    static __device__ __forceinline__ void turn(const Items &at, const Angles &g, U (&a)[I][N], U (&b)[I][N])
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (HALVES) {
                if (at.ta(i))
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const U x = a[i][j], y = b[i][j];
                        a[i][j] = fused_ma(y, g.minus[i][j], x * g.c[i][j]);
                        b[i][j] = fused_ma(x, g.s[i][j], y * g.c[i][j]);
                    }
            } else {
                if (at.ta(i))
#pragma unroll
                    for (int j = 0; j < N; ++j) a[i][j] = turned(a[i][j], g.c[i][j], g.s[i][j]);
                if (at.tb(i))
#pragma unroll
                    for (int j = 0; j < N; ++j) b[i][j] = turned(b[i][j], g.c[i][N + j], g.s[i][N + j]);
            }
        }
    }

    static __device__ __forceinline__ A part(U v, int k)
    {
        if constexpr (V == 1) return v;
        else return k ? second(v) : first(v);
    }
    static __device__ __forceinline__ A sum(U v, int lanes)
    {
        A s = joined(v);
        if (lanes > 8) {
            if (lanes > 16) s += __shfl_xor_sync(0xffffffffu, s, 16);
            s += __shfl_xor_sync(0xffffffffu, s, 8);
        }
        if (lanes > 4) s += __shfl_xor_sync(0xffffffffu, s, 4);
        if (lanes > 2) s += __shfl_xor_sync(0xffffffffu, s, 2);
        if (lanes > 1) s += __shfl_xor_sync(0xffffffffu, s, 1);
        return s;
    }
    // n = (x - mu) r of a vector, in place; returns r
    static __device__ __forceinline__ A normalise(int lanes, A inv_dim, const Items &at, int kind, A eps, U (&a)[I][N], U (&b)[I][N])
    {
        if (kind == FO_NORM_LAYER) {
            U s = head_all<U>(A(0));
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) s = s + (a[i][j] + b[i][j]);             // absent pieces are zeros
            const U mean = head_all<U>(-sum(s, lanes) * inv_dim);
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (at.a[i] >= 0) a[i][j] = a[i][j] + mean;
                    if (at.b[i] >= 0) b[i][j] = b[i][j] + mean;
                }
        }
        U sq = head_all<U>(A(0)), sr = sq;
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) sq = fused_ma(a[i][j], a[i][j], sq), sr = fused_ma(b[i][j], b[i][j], sr);
        const A r = group_rsqrt(fused_ma(sum(sq + sr, lanes), inv_dim, eps));
        const U all = head_all<U>(r);
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) a[i][j] = a[i][j] * all, b[i][j] = b[i][j] * all;
        return r;
    }
    static __device__ __forceinline__ void widen_piece(const Piece &q, U (&f)[N])
    {
        if constexpr (V == 1) {
            f[0] = widen(q.v[0]);
        } else if constexpr (V * sizeof(T) == 16) {
            const Packed<T, V> &w = reinterpret_cast<const Packed<T, V> &>(q);
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = w.get2(2 * j);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = two(widen(q.v[2 * j]), widen(q.v[2 * j + 1]));
        }
    }
    static __device__ __forceinline__ void store_piece(T *to, const U (&f)[N])
    {
        if constexpr (V == 1) {
            to[0] = narrow<T>(f[0]);
        } else {
            Packed<T, V * sizeof(T) == 8 ? 2 * V : V> w;
            w.clear();
#pragma unroll
            for (int j = 0; j < N; ++j) w.put2(2 * j, f[j]);
            if constexpr (V * sizeof(T) == 8) *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(&w);
            else store16(to, w.w);
        }
    }
    static __device__ __forceinline__ void store(T *row, const Items &at, const U (&a)[I][N], const U (&b)[I][N])
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (at.a[i] >= 0) store_piece(row + at.a[i], a[i]);
            if (at.b[i] >= 0) store_piece(row + at.b[i], b[i]);
        }
    }
    // A piece of a weight or bias vector.
    static __device__ __forceinline__ void vector_piece(const HeadParams &p, const void *v, int at, U (&f)[N])
    {
        A s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = p.wide_vec ? (A) static_cast<const float *>(v)[at + j] : widen(static_cast<const T *>(v)[at + j]);
        if constexpr (V == 1) f[0] = s[0];
        else
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = two(s[2 * j], s[2 * j + 1]);
    }
    // A piece of a vector in shared memory.
    static __device__ __forceinline__ void shared_piece(const A *v, U (&f)[N])
    {
        if constexpr (V == 1) {
            f[0] = *v;
        } else {
            constexpr int W = 16 / (int)sizeof(A);
#pragma unroll
            for (int j0 = 0; j0 < V; j0 += W) {
                const HeadPiece<A, W> s = head_load<A, W>(v + j0);
#pragma unroll
                for (int j = 0; j < W; j += 2) f[(j0 + j) / 2] = two(s.v[j], s.v[j + 1]);
            }
        }
    }
    static __device__ __forceinline__ void weights(const HeadParams &p, const HeadTensor &t, const Items &at, U (&a)[I][N], U (&b)[I][N])
    {
#pragma unroll
        for (int i = 0; i < I; ++i) {
#pragma unroll
            for (int j = 0; j < N; ++j) a[i][j] = b[i][j] = head_all<U>(A(1));
            if (t.weight && at.a[i] >= 0) vector_piece(p, t.weight, at.a[i], a[i]);
            if (t.weight && at.b[i] >= 0) vector_piece(p, t.weight, at.b[i], b[i]);
        }
    }
};

// The pieces of a lane's next turns, of TENSORS tensors.  Pieces of 8 and 16 bytes go through a ring in shared memory: piece k
// of turn s of thread t lies at ((s * pieces + k) * CTA + t) pieces, so that a warp's accesses meet all banks alike.  Single elements are fetched
// into registers a turn ahead.
template <class T, int V, int I, int TENSORS>
struct HeadRing {
    using Piece = HeadPiece<T, V>;
    static constexpr bool RING = V > 1;
    static constexpr int kTurns = RING ? (TENSORS == 1 ? 4 : 3) : 1;
    static constexpr int kPieces = 2 * I * TENSORS;
    static constexpr size_t kBytes = RING ? (size_t)kTurns * kPieces * kHeadCta * sizeof(Piece) : 0;
    Piece held[RING ? 1 : TENSORS][RING ? 1 : 2 * I];
    unsigned in, out, base;             // places of the next turn to come and to take, in bytes
    const Piece *memory;
    static constexpr unsigned kTurn = kPieces * kHeadCta * sizeof(Piece);

    __device__ __forceinline__ explicit HeadRing(void *m) : memory(static_cast<const Piece *>(m))
    {
        base = (unsigned)__cvta_generic_to_shared(m) + threadIdx.x * (unsigned)sizeof(Piece);
        in = out = 0;
    }

    // row[n]: the lane's vector of tensor n, or NULL for zeros
    template <class Items>
    __device__ __forceinline__ void issue(const T *const (&row)[TENSORS], const Items &at, bool on)
    {
#pragma unroll
        for (int n = 0; n < TENSORS; ++n)
#pragma unroll
            for (int k = 0; k < 2 * I; ++k) {
                const int e = k & 1 ? at.b[k / 2] : at.a[k / 2];
                if constexpr (RING) {
                    // with nothing to copy the place becomes zeros
                    const unsigned to = base + in + (n * 2 * I + k) * (unsigned)(kHeadCta * sizeof(Piece)), bytes = on && row[n] && e >= 0 ? sizeof(Piece) : 0;
                    const T *from = row[n] + (e >= 0 ? e : 0);
                    if constexpr (sizeof(Piece) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
                    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
                } else {
                    held[n][k] = on && row[n] && e >= 0 ? head_load<T, V>(row[n] + e) : Piece{};
                }
            }
        if constexpr (RING) {
            asm volatile("cp.async.commit_group;" ::: "memory");
            in = in == (kTurns - 1) * kTurn ? 0 : in + kTurn;
        }
    }
    // Before a turn's take(): what it takes has arrived.
    __device__ __forceinline__ void arrived() const
    {
        if constexpr (RING) asm volatile("cp.async.wait_group %0;" ::"n"(kTurns - 1) : "memory");
    }
    __device__ __forceinline__ Piece take(int n, int k) const
    {
        if constexpr (RING) {
            Piece r;
            uint32_t *w = reinterpret_cast<uint32_t *>(&r);
            const unsigned from = base + out + (n * 2 * I + k) * (unsigned)(kHeadCta * sizeof(Piece));
            if constexpr (sizeof(Piece) == 16)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from) : "memory");
            else asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(from) : "memory");
            return r;
        } else return held[n][k];
    }
    __device__ __forceinline__ void taken()
    {
        if constexpr (RING) out = out == (kTurns - 1) * kTurn ? 0 : out + kTurn;
    }
};

// The turns of a warp, one behind the other, through blocks of tokens: in a turn the groups work on a head of a token each (wide), or on
// as many heads of one token.  Every warp has the same number of turns and begins where the one before it ends, within a block.
struct HeadTurns {
    unsigned block, h0;                 // h0: the first group's head
    int left, by;                       // left: turns to come
    int group, beside;                  // group: of the lane; beside: its head is h0 + beside
    int wide, groups;
    __device__ __forceinline__ HeadTurns(const HeadParams &p, const HeadTensor &t, int cta, int group_)
        : group(group_), wide(p.wide), groups(32 / p.lanes)
    {
        const unsigned first = (unsigned)(cta * kHeadWarps + (int)(threadIdx.x / 32)) * (unsigned)t.each, all = (unsigned)t.blocks * (unsigned)t.turns;
        left = first < all ? (int)min(all - first, (unsigned)t.each) : 0;
        by = wide ? 1 : groups, beside = wide ? 0 : group;
        block = first / (unsigned)t.turns, h0 = (first - block * (unsigned)t.turns) * by;
    }
    __device__ __forceinline__ bool there() const { return left > 0; }
    // the lane's token, of this block or a later one
    __device__ __forceinline__ unsigned token(unsigned later = 0) const { return wide ? (block + later) * (unsigned)groups + group : block + later; }
    __device__ __forceinline__ bool on(const HeadParams &p, const HeadTensor &t) const { return h0 + beside < (unsigned)t.heads && token() < (unsigned)p.all_tokens; }
    // true: a new block
    __device__ __forceinline__ bool next(const HeadTensor &t)
    {
        --left, h0 += by;
        if (h0 < (unsigned)t.heads) return false;
        h0 = 0, ++block;
        return true;
    }
};
// A lane's way through a tensor along its warp's turns: the vector of its group's head.
template <class T>
struct HeadWay {
    T *at = nullptr;
    long long step;
    __device__ __forceinline__ void enter(const HeadParams &p, const void *x, const fo_strides &s, const HeadTurns &turn)
    {
        const unsigned token = turn.token(), b = token / (unsigned)p.tokens, t = token - b * (unsigned)p.tokens;
        at = static_cast<T *>(const_cast<void *>(x)) + b * s.batch + t * s.token + (turn.h0 + turn.beside) * s.head;
        step = turn.by * s.head;
    }
    __device__ __forceinline__ void next() { at += step; }
};

// Bound by the instructions of a turn, about 260 of a warp (backwards 410), at the rate at which 16 warps an SM issue them, 0.55 to 0.6 of
// a cycle: 4 x 2048 tokens with 32 + 8 heads of 128 in bfloat16 take 36 us (4.8 TB/s), backwards 59 us (4.3 TB/s).
template <class T, int V, int I, int PAIRING>
__global__ void __launch_bounds__(kHeadCta, sizeof(Acc<T>) == 8 ? 1 : 2) head_norm_kernel(const __grid_constant__ HeadParams p)
{
    using W = HeadWork<T, V, I, PAIRING>;
    using A = Acc<T>;
    using U = typename W::U;
    constexpr int N = W::N;
    extern __shared__ __align__(16) unsigned char head_memory[];
    wait_for_earlier();
    const int which = blockIdx.x >= (unsigned)p.ctas0;
    const HeadTensor &t = p.t[which];
    const int lane = threadIdx.x & (p.lanes - 1), group = (threadIdx.x & 31) / p.lanes, kind = t.kind;
    const A eps = A(t.eps), inv_dim = A(p.inv_dim);
    const int cta = which ? blockIdx.x - p.ctas0 : blockIdx.x;
    const typename W::Items at(lane, p.lanes, p.dim, p.pairs);
    HeadTurns ahead(p, t, cta, group), now = ahead;
    if (!now.there()) return;
    const bool bias = t.bias != nullptr;
    HeadRing<T, V, I, 1> ring(head_memory);
    HeadWay<T> x, y;
    x.enter(p, t.x, t.x_at, ahead), y.enter(p, t.y, t.y_at, now);
    auto issue = [&]() {
        const T *const rows[1] = {x.at};
        const bool there = ahead.there();
        ring.issue(rows, at, there && ahead.on(p, t));
        if (!there) return;
        if (!ahead.next(t)) x.next();
        else if (ahead.there()) x.enter(p, t.x, t.x_at, ahead);
    };
    for (int k = 0; k < ring.kTurns; ++k) issue();
    U wa[I][N], wb[I][N];
    W::weights(p, t, at, wa, wb);
    typename W::Angles g;
    HeadRows rows = {};
    if (p.pairs) rows = head_rows(p, now.token());
    for (bool fresh = true; now.there();) {
        if (fresh && p.pairs) {
            W::template angles<1>(p, at, rows, g);
            rows = head_rows(p, now.token(1));
        }
        U a[I][N], b[I][N];
        ring.arrived();
#pragma unroll
        for (int i = 0; i < I; ++i) W::widen_piece(ring.take(0, 2 * i), a[i]), W::widen_piece(ring.take(0, 2 * i + 1), b[i]);
        ring.taken();
        issue();
        if (kind != FO_NORM_NONE) {
            W::normalise(p.lanes, inv_dim, at, kind, eps, a, b);
#pragma unroll
            for (int i = 0; i < I; ++i) {
#pragma unroll
                for (int j = 0; j < N; ++j) a[i][j] = a[i][j] * wa[i][j], b[i][j] = b[i][j] * wb[i][j];
                if (bias) {
                    U bias[N];
                    if (at.a[i] >= 0) {
                        W::vector_piece(p, t.bias, at.a[i], bias);
#pragma unroll
                        for (int j = 0; j < N; ++j) a[i][j] = a[i][j] + bias[j];
                    }
                    if (at.b[i] >= 0) {
                        W::vector_piece(p, t.bias, at.b[i], bias);
#pragma unroll
                        for (int j = 0; j < N; ++j) b[i][j] = b[i][j] + bias[j];
                    }
                }
            }
        }
        if (p.pairs) W::turn(at, g, a, b);
        if (now.on(p, t)) W::store(y.at, at, a, b);
        if (fresh && p.pairs) W::expect(p, at, rows);
        fresh = now.next(t);
        if (!fresh) y.next();
        else if (now.there()) y.enter(p, t.y, t.y_at, now);
    }
}

// The gradient.  Every lane keeps the sums of its own elements of dweight and dbias; at the end a CTA writes a line of
// them, and head_sum_kernel adds the lines in order.
template <class T, int V, int I, int PAIRING, bool BIAS>
__global__ void __launch_bounds__(kHeadCta, sizeof(Acc<T>) == 8 ? 1 : 2) head_norm_grad_kernel(const __grid_constant__ HeadParams p)
{
    using W = HeadWork<T, V, I, PAIRING>;
    using A = Acc<T>;
    using U = typename W::U;
    constexpr int N = W::N;
    extern __shared__ __align__(16) unsigned char head_memory[];
    __shared__ __align__(16) A weights[FO_HEAD_MAX_DIM + 16];
    wait_for_earlier();
    const int which = blockIdx.x >= (unsigned)p.ctas0;
    const HeadTensor &t = p.t[which];
    const int lane = threadIdx.x & (p.lanes - 1), group = (threadIdx.x & 31) / p.lanes, kind = t.kind;
    const A eps = A(t.eps), inv_dim = A(p.inv_dim);
    const int cta = which ? blockIdx.x - p.ctas0 : blockIdx.x;
    const typename W::Items at(lane, p.lanes, p.dim, p.pairs);
    const bool normed = kind != FO_NORM_NONE;
    HeadTurns ahead(p, t, cta, group), now = ahead;
    HeadRing<T, V, I, 2> ring(head_memory);
    HeadWay<T> x, dy, dx;
    auto enter = [&]() {
        if (normed) x.enter(p, t.x, t.x_at, ahead);
        dy.enter(p, t.dy, t.dy_at, ahead);
    };
    if (now.there()) enter(), dx.enter(p, t.y, t.y_at, now);
    auto issue = [&]() {
        const T *const rows[2] = {dy.at, x.at};
        const bool there = ahead.there();
        ring.issue(rows, at, there && ahead.on(p, t));
        if (!there) return;
        if (!ahead.next(t)) {
            if (normed) x.next();
            dy.next();
        } else if (ahead.there()) enter();
    };
    for (int k = 0; k < ring.kTurns; ++k) issue();
    U da[I][N], db[I][N], ea[BIAS ? I : 1][N], eb[BIAS ? I : 1][N];
    // the weights, with zeros for pieces that are none (in registers they made the loop spill others)
    for (int j = threadIdx.x; j < p.dim + V; j += kHeadCta)
        weights[j] = j >= p.dim ? A(0) : !t.weight ? A(1) : p.wide_vec ? (A) static_cast<const float *>(t.weight)[j] : widen(static_cast<const T *>(t.weight)[j]);
    __syncthreads();
    const U zero = head_all<U>(A(0));
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            da[i][j] = db[i][j] = zero;
            if (BIAS) ea[i][j] = eb[i][j] = zero;
        }
    typename W::Angles g;
    HeadRows rows = {};
    if (p.pairs && now.there()) rows = head_rows(p, now.token());
    for (bool fresh = true; now.there();) {
        if (fresh && p.pairs) {
            W::template angles<-1>(p, at, rows, g);
            rows = head_rows(p, now.token(1));
        }
        U a[I][N], b[I][N], u[I][N], v[I][N];
        ring.arrived();
#pragma unroll
        for (int i = 0; i < I; ++i) {
            W::widen_piece(ring.take(0, 2 * i), u[i]), W::widen_piece(ring.take(0, 2 * i + 1), v[i]);
            W::widen_piece(ring.take(1, 2 * i), a[i]), W::widen_piece(ring.take(1, 2 * i + 1), b[i]);
        }
        ring.taken();
        issue();
        const bool on = now.on(p, t);
        if (p.pairs && on) W::turn(at, g, u, v);           // a group without a head keeps its zeros, whatever the angles are
        if (normed) {
            // a group without a head has zeros throughout, and with eps 0 its r would not be finite
            const A r = W::normalise(p.lanes, inv_dim, at, kind, on ? eps : A(1), a, b);
            U with_n = zero, alone = zero;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                U wa[N], wb[N];
                W::shared_piece(weights + (at.a[i] >= 0 ? at.a[i] : p.dim), wa), W::shared_piece(weights + (at.b[i] >= 0 ? at.b[i] : p.dim), wb);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    da[i][j] = fused_ma(u[i][j], a[i][j], da[i][j]);
                    db[i][j] = fused_ma(v[i][j], b[i][j], db[i][j]);
                    if (BIAS) ea[i][j] = ea[i][j] + u[i][j], eb[i][j] = eb[i][j] + v[i][j];
                    u[i][j] = u[i][j] * wa[j], v[i][j] = v[i][j] * wb[j];
                    with_n = fused_ma(u[i][j], a[i][j], fused_ma(v[i][j], b[i][j], with_n));
                    alone = alone + (u[i][j] + v[i][j]);
                }
            }
            const U back = head_all<U>(-W::sum(with_n, p.lanes) * inv_dim), all = head_all<U>(r);
            const U mean = kind == FO_NORM_LAYER ? head_all<U>(-W::sum(alone, p.lanes) * inv_dim) : zero;
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    u[i][j] = (fused_ma(back, a[i][j], u[i][j]) + mean) * all;
                    v[i][j] = (fused_ma(back, b[i][j], v[i][j]) + mean) * all;
                }
        }
        if (on) W::store(dx.at, at, u, v);
        if (fresh && p.pairs) W::expect(p, at, rows);
        fresh = now.next(t);
        if (!fresh) dx.next();
        else if (now.there()) dx.enter(p, t.y, t.y_at, now);
    }
    if (!t.partial_w && !t.partial_b) return;
    // every group of lanes writes its sums (where the ring was), and they are added in order
    A *const lines = reinterpret_cast<A *>(head_memory);
    const int count = kHeadWarps * (32 / p.lanes), mine = threadIdx.x / p.lanes;
    if constexpr (V > 1) asm volatile("cp.async.wait_all;" ::: "memory");
    for (int which_sum = 0; which_sum < (BIAS ? 2 : 1); ++which_sum) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int k = 0; k < V / N; ++k) {
                    const int e = j * (V / N) + k;
                    const U sa = BIAS && which_sum ? ea[BIAS ? i : 0][j] : da[i][j], sb = BIAS && which_sum ? eb[BIAS ? i : 0][j] : db[i][j];
                    if (at.a[i] >= 0) lines[mine * p.dim + at.a[i] + e] = W::part(sa, k);
                    if (at.b[i] >= 0) lines[mine * p.dim + at.b[i] + e] = W::part(sb, k);
                }
        __syncthreads();
        A *const to = static_cast<A *>(which_sum ? t.partial_b : t.partial_w);
        if (to)
            for (int j = threadIdx.x; j < p.dim; j += kHeadCta) {
                A s = A(0);
                for (int l = 0; l < count; ++l) s += lines[l * p.dim + j];
                to[(size_t)cta * p.dim + j] = s;
            }
    }
}

// Host: the kernel for a type, a number of elements in a piece and a vector's length; head_norm_*.cu instantiate it.
template <class T>
cudaError_t launch_head_norm(const HeadParams &p, int piece, int pairing, bool grad, bool bias, int grid, cudaStream_t st);

}  // namespace fo
