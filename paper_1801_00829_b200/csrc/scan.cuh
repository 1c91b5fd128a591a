// A gated linear recurrence over the tokens, h_t = a_t h_{t-1} + m(a_t) x_t, and its gradient, the same recurrence backwards.
//
// A thread works on V neighbouring channels over S successive tokens (a segment), a CTA on 32 V channels over as many segments as
// it has warps, a cluster on as many as its CTAs have together: that is one round, and rounds follow each other over
// the sequence.  In a round every warp runs its segment from zero, which gives the map h -> A h + H of the whole segment, the maps
// are put one behind the other in the order of the tokens, and with the state that comes in the segment is run again, from
// registers.  So the inputs are read once and no CTA waits for another outside its cluster, whose CTAs run together.
// The inputs of the next rounds are on their way meanwhile, to a ring in shared memory: asynchronous copies, which a warp makes
// for itself.
// A round in a cluster takes 2.5 us or more, however few its channels are.  So long sequences of few channels are cut into chunks instead, as many as
// make CTAs for all SMs: a first kernel reads the chunks and leaves the map of each, a second one puts these together to the states that
// come into them, and then the chunks are run like sequences of their own.
#pragma once

#include "elem.cuh"
#include "../../include/fusedops_lm.h"

namespace fo {

constexpr int kScanCta = 256;
constexpr int kScanMostWarps = kScanCta / 32;
constexpr int kScanMostCluster = 8;
constexpr int kScanLeastChunked = 8 * kScanMostCluster * kScanMostWarps * 4;   // tokens: eight rounds of a cluster in segments of four
constexpr int kScanMostSms = 256;       // chunks make CTAs for two on each of these at most

enum ScanTensor { kScanX = 1, kScanGate = 2, kScanDh = 4, kScanH = 8, kScanOut = 16, kScanOutGate = 32, kScanNear = 64, kScanAll = 127 };

struct ScanParams {
    long long channels, batch;
    int tokens, tiles;                  // tiles: of 32 V channels
    int mode, long_lengths;             // mode: decay * 3 + mix
    int whole;                          // which tensors' rows begin at 16-byte boundaries (ScanTensor), outputs' at those of two channels; near:
                                        // the rows of a segment lie within 32 bits of each other
    const void *x, *gate, *state, *lengths;
    const unsigned char *reset;
    void *h, *last;                     // gradient: dx, dstate
    fo_rows x_at, gate_at, reset_at, h_at;
    // the gradient's own
    const void *dh, *dlast, *h_in;
    void *dgate;
    // chunks of `chunk` tokens each (the last one's are what is left), their maps and the states that come into them
    int chunks, chunk;
    void *map_a, *map_h, *carry;        // batch x chunks x channels
    int *map_drops;                     // batch x chunks: a reset lies in it
    fo_rows dh_at, h_in_at, dgate_at;
};

// ------------------------------------------------------------------------------------------------ clusters
__device__ __forceinline__ unsigned scan_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned scan_cluster()
{
    unsigned n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}
__device__ __forceinline__ void scan_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void scan_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned scan_peer(const void *p, unsigned rank)
{
    unsigned a = (unsigned)__cvta_generic_to_shared(p), r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}

// ------------------------------------------------------------------------------------------------ pieces of V channels
template <class T, int V>
struct ScanPiece {
    alignas(V * sizeof(T)) T v[V];
};
template <class T, int V>
__device__ __forceinline__ ScanPiece<T, V> scan_piece(const char *p)
{
    ScanPiece<T, V> r;
    if constexpr (V * sizeof(T) == 4) *reinterpret_cast<uint32_t *>(&r) = *reinterpret_cast<const uint32_t *>(p);
    else if constexpr (V * sizeof(T) == 8) *reinterpret_cast<uint2 *>(&r) = *reinterpret_cast<const uint2 *>(p);
    else r.v[0] = *reinterpret_cast<const T *>(p);
    return r;
}
template <class T, int V>
__device__ __forceinline__ void scan_store(char *row, unsigned offset, const ScanPiece<T, V> &r)
{
    char *p = row + offset;
    if constexpr (V * sizeof(T) == 4) *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(&r);
    else if constexpr (V * sizeof(T) == 8) *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(&r);
    else *reinterpret_cast<T *>(p) = r.v[0];
}
// A lane's channels of a row, which is found by a base that is the same for the whole warp and the lane's offset.  count: of
// the channels that there are; whole: they can move together.
template <class T, int V>
__device__ __forceinline__ void scan_store(char *row, unsigned offset, const ScanPiece<T, V> &r, int count, bool whole)
{
    char *p = row + offset;
    if constexpr (V == 1) {
        if (count > 0) *reinterpret_cast<T *>(p) = r.v[0];
    } else {
        if (whole) {
            if (count == 2) {
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(&r);
                else *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(&r);
                return;
            }
        }
        if (count > 0) reinterpret_cast<T *>(p)[0] = r.v[0];
        if (count > 1) reinterpret_cast<T *>(p)[1] = r.v[1];
    }
}

// Copies of a warp's segment, S rows of W channels, into its place in the ring.  Row r is at base + r * stride (the stride is
// negative where segments run backwards).  Pieces of 16 bytes where all rows begin at such a boundary, the last one of a row
// cut off where its channels end; else single elements of 4 or 8 bytes; those of 2 bytes, which no asynchronous copy can
// move, by loads.
template <class T, int S, int W>
struct ScanCopy {
    static constexpr int kBytes = S * W * (int)sizeof(T);
    static constexpr int kRowPieces = W * (int)sizeof(T) / 16, kRows = 32 / kRowPieces, kTurns = S / kRows;
    int row, bytes, channels;
    unsigned place, from[kTurns];       // from: offsets from the segment's lowest row in memory
    bool whole;
    __device__ __forceinline__ ScanCopy(bool whole_, int lane, int channels_, long long stride) : channels(channels_), whole(whole_)
    {
        row = lane / kRowPieces;
        const int at = lane % kRowPieces * 16;
        bytes = min(16, min(channels, W) * (int)sizeof(T) - at);         // (all channels' bytes may be 2^31)
        place = row * W * (int)sizeof(T) + at;
#pragma unroll
        for (int j = 0; j < kTurns; ++j) {
            const int r = row + j * kRows;
            from[j] = (unsigned)((stride < 0 ? (S - 1 - r) * -stride : r * stride) + at);
        }
    }
    // All rows and all channels of the tile are there, and whole, and within 32 bits of `lowest`.
    __device__ __forceinline__ void issue_all(char *to, const char *lowest) const
    {
        const unsigned at = (unsigned)__cvta_generic_to_shared(to) + place;
#pragma unroll
        for (int j = 0; j < kTurns; ++j)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + j * 512), "l"(lowest + from[j]) : "memory");
    }
    template <class Valid>
    __device__ __forceinline__ void issue(char *to, const char *base, long long stride, Valid valid) const
    {
        if (whole) {
#pragma unroll
            for (int j = 0; j < kTurns; ++j)
                if (valid(row + j * kRows) && bytes > 0)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(to) + place + j * 512),
                                 "l"(base + (row + j * kRows) * stride + (place - row * W * (int)sizeof(T))), "r"(bytes) : "memory");
            return;
        }
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int j = 0; j < S; ++j)
#pragma unroll
            for (int v = 0; v < W / 32; ++v) {
                const int c = v * 32 + lane;
                if (!valid(j) || c >= channels) continue;
                const T *from = reinterpret_cast<const T *>(base + j * stride) + c;
                T *dst = reinterpret_cast<T *>(to) + j * W + c;
                if constexpr (sizeof(T) == 2) *dst = *from;
                else
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(from), "n"((int)sizeof(T)) : "memory");
            }
    }
};
template <int N>
__device__ __forceinline__ void scan_arrived()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}
__device__ __forceinline__ void scan_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// The unit of arithmetic: a lane's V channels, two of them in one register pair.
template <class A, int V> struct ScanUnit { using U = Two<A>; };
template <class A> struct ScanUnit<A, 1> { using U = A; };
__device__ __forceinline__ float scan_part(float u, int) { return u; }
__device__ __forceinline__ double scan_part(double u, int) { return u; }
template <class A> __device__ __forceinline__ A scan_part(Two<A> u, int v) { return v ? second(u) : first(u); }
template <class U, class A>
__device__ __forceinline__ U scan_all(A v)
{
    if constexpr (std::is_same<U, A>::value) return v;
    else return both(v);
}
// f of every channel
template <class F> __device__ __forceinline__ float scan_each(float u, F f) { return f(u); }
template <class F> __device__ __forceinline__ double scan_each(double u, F f) { return f(u); }
template <class A, class F> __device__ __forceinline__ Two<A> scan_each(Two<A> u, F f) { return two(f(first(u)), f(second(u))); }
template <class F> __device__ __forceinline__ float scan_each(float u, float w, F f) { return f(u, w); }
template <class F> __device__ __forceinline__ double scan_each(double u, double w, F f) { return f(u, w); }
template <class A, class F> __device__ __forceinline__ Two<A> scan_each(Two<A> u, Two<A> w, F f) { return two(f(first(u), first(w)), f(second(u), second(w))); }
template <class U, class T, int V>
__device__ __forceinline__ U scan_widen(const ScanPiece<T, V> &p)
{
    if constexpr (V == 1) return (U)widen(p.v[0]);
    else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(&p);
        return two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    } else return two(widen(p.v[0]), widen(p.v[1]));
}
template <class T, int V, class U>
__device__ __forceinline__ ScanPiece<T, V> scan_narrow(U u)
{
    ScanPiece<T, V> r;
    if constexpr (V == 2 && sizeof(T) == 2) {
        Packed<T, 8> w;
        w.put2(0, u);
        *reinterpret_cast<uint32_t *>(&r) = w.w[0];
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) r.v[v] = narrow<T>(scan_part(u, v));
    }
    return r;
}

// ------------------------------------------------------------------------------------------------ decays
// a and 1 - a, both without cancellation.  A decay near 1 multiplies a state very many times, so that its error adds up over
// 1 / (1 - a) tokens: it is 1 minus its small complement, and so rounded once.  EXACT (32- and 64-bit x): by CUDA's functions; else by
// the hardware's exponential and reciprocal, whose relative error, up to (10 + |gate|) 2^-23 by the exponent's rounding, is then one of the smaller
// of a decay and its complement.
__device__ __forceinline__ float scan_exp2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float scan_rcp(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float scan_sqrt(float v)
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
template <bool EXACT> __device__ __forceinline__ float scan_root(float v) { return EXACT ? sqrtf(v) : scan_sqrt(v); }
template <bool EXACT> __device__ __forceinline__ double scan_root(double v) { return sqrt(v); }
template <bool EXACT> __device__ __forceinline__ float scan_over(float v) { return EXACT ? 1.0f / v : scan_rcp(v); }
template <bool EXACT> __device__ __forceinline__ double scan_over(double v) { return 1.0 / v; }
// exp(-|g|)
template <bool EXACT> __device__ __forceinline__ float scan_exp_down(float g) { return EXACT ? expf(-fabsf(g)) : scan_exp2(fabsf(g) * -1.4426950408889634f); }
template <bool EXACT> __device__ __forceinline__ double scan_exp_down(double g) { return exp(-fabs(g)); }

// exp(g) and 1 - exp(g)
template <bool EXACT>
__device__ __forceinline__ void scan_exponential(float g, float &a, float &rest)
{
    if constexpr (EXACT) {
        rest = -expm1f(g);
        a = g > -0.5f ? 1.0f - rest : expf(g);
    } else {
        // exp(g) - 1 by its series up to g^6 / 720 where it is small: what that leaves out is below 2^-24 of it
        float m = fused_ma(g, 1.0f / 720.0f, 1.0f / 120.0f);
        m = fused_ma(m, g, 1.0f / 24.0f);
        m = fused_ma(m, g, 1.0f / 6.0f);
        m = fused_ma(m, g, 0.5f);
        m = fused_ma(m * g, g, g);
        const float e = scan_exp2(g * 1.4426950408889634f);
        const bool near = fabsf(g) < 0.25f;
        a = near ? 1.0f + m : e, rest = near ? -m : 1.0f - e;
    }
}
template <bool EXACT>
__device__ __forceinline__ void scan_exponential(double g, double &a, double &rest)
{
    rest = -expm1(g);
    a = g > -0.5 ? 1.0 - rest : exp(g);
}
// e * rest in place of a where e is at most 1
__device__ __forceinline__ float scan_below(float a, float e, float rest)
{
    asm("{\n\t.reg .pred p;\n\tsetp.le.f32 p, %1, 0f3F800000;\n\t@p mul.f32 %0, %1, %2;\n\t}" : "+f"(a) : "f"(e), "f"(rest));
    return a;
}
// SLOPES: a product of a and rest is wanted, to which a small a counts by its own size; otherwise by that of what it multiplies.
template <int DECAY, bool EXACT, bool SLOPES, class A, class U>
__device__ __forceinline__ void scan_decay(U g, U &a, U &rest)
{
    const U one = scan_all<U>(A(1)), less = scan_all<U>(A(-1));
    if constexpr (DECAY == FO_DECAY_VALUE) {
        a = g, rest = fused_ma(g, less, one);
    } else if constexpr (DECAY == FO_DECAY_SIGMOID && !EXACT && !SLOPES) {
        // rest is 1 / (1 + exp(g)).  A decay above a half is 1 minus that, rounded once; one below, the exponential times it, which
        // keeps its bits however small it is (8 x 4096 x 2048 in bfloat16 72 to 74 us; as 1 minus the rest throughout, with 2^-23 of 1 lost to
        // it, 72)
        const U e = scan_each(g * scan_all<U>(A(1.4426950408889634)), [](A v) { return scan_exp2(v); });
        rest = scan_each(e + one, [](A v) { return scan_over<EXACT>(v); });
        a = fused_ma(rest, less, one);
        if constexpr (std::is_same<U, A>::value) a = e > A(1) ? a : e * rest;
        else a = two(scan_below(first(a), first(e), first(rest)), scan_below(second(a), second(e), second(rest)));
    } else if constexpr (DECAY == FO_DECAY_SIGMOID) {
        const U e = scan_each(g, [](A v) { return scan_exp_down<EXACT>(v); });
        const U small = e * scan_each(e + one, [](A v) { return scan_over<EXACT>(v); }), big = fused_ma(small, less, one);
        if constexpr (std::is_same<U, A>::value) {
            a = g >= A(0) ? big : small, rest = g >= A(0) ? small : big;
        } else {
            const bool p = first(g) >= A(0), q = second(g) >= A(0);
            a = two(p ? first(big) : first(small), q ? second(big) : second(small));
            rest = two(p ? first(small) : first(big), q ? second(small) : second(big));
        }
    } else if constexpr (std::is_same<U, A>::value) {
        scan_exponential<EXACT>(g, a, rest);
    } else {
        A a0, a1, r0, r1;
        scan_exponential<EXACT>(first(g), a0, r0);
        scan_exponential<EXACT>(second(g), a1, r1);
        a = two(a0, a1), rest = two(r0, r1);
    }
}
// m(a)
template <int MIX, bool EXACT, class A, class U>
__device__ __forceinline__ U scan_mix(U a, U rest)
{
    if constexpr (MIX == FO_MIX_ONE) return scan_all<U>(A(1));
    else if constexpr (MIX == FO_MIX_REST) return rest;
    else return scan_each(fused_ma(rest, a, rest), [](A v) { return scan_root<EXACT>(v); });
}
// The derivatives of a and of m to the gate.
template <int DECAY, int MIX, bool EXACT, class A, class U>
__device__ __forceinline__ void scan_slopes(U a, U rest, U m, U &da, U &dm)
{
    const U less = scan_all<U>(A(-1));
    if constexpr (DECAY == FO_DECAY_VALUE) da = scan_all<U>(A(1));
    else if constexpr (DECAY == FO_DECAY_EXP) da = a;
    else da = a * rest;
    if constexpr (MIX == FO_MIX_ONE) dm = scan_all<U>(A(0));
    else if constexpr (MIX == FO_MIX_REST) dm = da * less;
    else if constexpr (DECAY == FO_DECAY_SIGMOID)            // a' = a (1 - a) has m in it
        dm = a * (a * less) * m * scan_each(a + scan_all<U>(A(1)), [](A v) { return scan_over<EXACT>(v); });
    else dm = a * (da * less) * scan_each(m, [](A v) { return scan_over<EXACT>(v); });
}

// Calls go(decay, mix) with compile-time numbers.
template <class Go>
__device__ __forceinline__ void with_mode(int mode, Go go)
{
#define FO_MODE(d, m) \
    case d * 3 + m: go(std::integral_constant<int, d>(), std::integral_constant<int, m>()); break;
    switch (mode) {
        FO_MODE(0, 0) FO_MODE(0, 1) FO_MODE(0, 2) FO_MODE(1, 0) FO_MODE(1, 1) FO_MODE(1, 2) FO_MODE(2, 0) FO_MODE(2, 1) FO_MODE(2, 2)
    }
#undef FO_MODE
}
template <class Go>
__device__ __forceinline__ void with_decay(int mode, Go go)
{
    if (mode < 3) go(std::integral_constant<int, FO_DECAY_VALUE>());
    else if (mode < 6) go(std::integral_constant<int, FO_DECAY_SIGMOID>());
    else go(std::integral_constant<int, FO_DECAY_EXP>());
}

// ------------------------------------------------------------------------------------------------ segments put together
// h -> a h + h of V channels
template <class U>
struct ScanMap {
    U a, h;
};

// The shared memory of a CTA, twice (one round's is written while another warp still reads the last one's).
template <class U>
struct ScanShared {
    ScanMap<U> *warp_maps, *cta_maps;                    // of every warp's segment, and of every CTA's segments
    U *carry;                                            // what comes into the round
    unsigned long long *bars;                            // of the maps that the cluster's CTAs send
    int *warp_drops, *cta_drops;                         // a reset lies in them: nothing comes through
    int warps, ctas;

    static __host__ __device__ size_t bytes(int warps, int ctas)
    {
        if (warps * ctas == 1) return 0;
        return 2 * ((warps + ctas) * 32 * sizeof(ScanMap<U>) + 32 * sizeof(U) + (kScanMostCluster + kScanMostWarps) * sizeof(int) + sizeof(unsigned long long));
    }
    __device__ __forceinline__ ScanShared(void *at, int w, int c) : warps(w), ctas(c)
    {
        warp_maps = static_cast<ScanMap<U> *>(at) + (threadIdx.x & 31), cta_maps = warp_maps + 2 * w * 32;
        carry = reinterpret_cast<U *>(static_cast<ScanMap<U> *>(at) + 2 * (w + c) * 32) + (threadIdx.x & 31);
        cta_drops = reinterpret_cast<int *>(reinterpret_cast<U *>(static_cast<ScanMap<U> *>(at) + 2 * (w + c) * 32) + 2 * 32);
        warp_drops = cta_drops + 2 * kScanMostCluster;
        bars = reinterpret_cast<unsigned long long *>(warp_drops + 2 * kScanMostWarps);
    }
    __device__ __forceinline__ ScanMap<U> *warp(int parity) const { return warp_maps + parity * warps * 32; }
    __device__ __forceinline__ ScanMap<U> *cta(int parity) const { return cta_maps + parity * ctas * 32; }
    __device__ __forceinline__ unsigned bar(int parity) const { return (unsigned)__cvta_generic_to_shared(bars + parity); }
};

template <class U>
__device__ __forceinline__ U scan_apply(const ScanMap<U> &m, int drops, U c)
{
    return drops ? m.h : fused_ma(m.a, c, m.h);
}
// To another CTA of the cluster, which counts the bytes that have come at its barrier `bar`.  A barrier of the cluster in every
// round would have each thread wait until all that it has stored has arrived, the results among it (7 us a round).
template <class U>
__device__ __forceinline__ void scan_push(unsigned to, unsigned bar, const ScanMap<U> &m)
{
    static_assert(sizeof(m) == 16, "a map is 16 bytes");
    const uint32_t *w = reinterpret_cast<const uint32_t *>(&m);
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to), "r"(w[0]), "r"(w[1]),
                 "r"(w[2]), "r"(w[3]), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void scan_push(unsigned to, unsigned bar, int v)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(to), "r"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void scan_expect(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// False if what is waited for has not come after very many polls: then the results are NaN, and no later round waits (scan_join).  What
// has come was sent by other CTAs, whose stores are a release at the cluster's scope: the wait acquires at that scope too (its default is the
// CTA's, which orders nothing of another CTA).  1 x 65536 x 2560, gates in 32 bits: 363 us, with the weaker wait 374 to 379.
__device__ __forceinline__ bool scan_await(unsigned bar, unsigned phase)
{
    for (unsigned i = 0; i < (1u << 22); ++i) {
        unsigned ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(phase)
            : "memory");
        if (ok) return true;
    }
    return false;
}
// `c` through maps [from, to), where any of them drops what comes (DROPS) by their marks.
template <bool DROPS, class U>
__device__ __forceinline__ U scan_through(const ScanMap<U> *maps, const int *drops, int from, int to, U c)
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k >= from && k < to) c = scan_apply(maps[k * 32], DROPS ? drops[k] : 0, c);
    return c;
}

// Before the first round: `carry` is what comes into it, in every warp and CTA.
template <class U>
__device__ __forceinline__ void scan_begin(const ScanShared<U> &sh, int warp, U carry)
{
    if (sh.warps * sh.ctas == 1) return;
    if (warp == sh.warps - 1) sh.carry[0] = carry;
    if (sh.ctas == 1) return;
    if (threadIdx.x < 2 * kScanMostCluster) sh.cta_drops[threadIdx.x] = 0;
    if (threadIdx.x < 2) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(sh.bar(threadIdx.x)) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();                                     // and every CTA has started
    scan_arrive();
    scan_wait();
}
template <bool DROPS, class A, class U>
__device__ __forceinline__ U scan_joined(const ScanShared<U> &sh, int parity, unsigned rank, unsigned cluster, int warp, const ScanMap<U> &own, int drops)
{
    const ScanMap<U> *const maps = sh.warp(parity);
    const int *const marks = sh.warp_drops + parity * kScanMostWarps;
    const bool last = warp == sh.warps - 1;
    U in = sh.carry[parity * 32];
    if (cluster > 1) {
        const ScanMap<U> *const ctas = sh.cta(parity);
        const int *const cta_marks = sh.cta_drops + parity * kScanMostCluster;
        in = scan_through<DROPS>(ctas, cta_marks, 0, (int)rank, in);
        if (last) sh.carry[(parity ^ 1) * 32] = scan_through<DROPS>(ctas, cta_marks, (int)rank, (int)cluster, in);
        return scan_through<DROPS>(maps, marks, 0, warp, in);
    }
    in = scan_through<DROPS>(maps, marks, 0, warp, in);
    if (last) sh.carry[(parity ^ 1) * 32] = scan_apply(own, DROPS ? drops : 0, in);
    return in;
}

// Every warp gives its segment's map (and whether it drops what comes in); returns what comes into the segment.  `carry` is
// what comes into the round and what leaves it where a warp is alone; otherwise the last warp of each CTA writes what leaves the round
// for the next one, whose barrier lies between.  turn: the round's number.
template <class A, class U>
__device__ __forceinline__ U scan_join(const ScanShared<U> &sh, int turn, unsigned rank, unsigned cluster, int warp, const ScanMap<U> &own,
                                       bool resets, int drops, U &carry, bool &lost)
{
    const int lane = threadIdx.x & 31, warps = sh.warps, parity = turn & 1;
    if (warps == 1 && cluster == 1) {
        const U in = carry;
        carry = scan_apply(own, drops, carry);
        return in;
    }
    sh.warp(parity)[warp * 32] = own;
    int any = 0;
    if (resets) {
        if (lane == 0) sh.warp_drops[parity * kScanMostWarps + warp] = drops;
        any = __syncthreads_or(drops);
    } else {
        __syncthreads();
    }
    if (cluster > 1) {
        if (warp == warps - 1) {
            const ScanMap<U> *const maps = sh.warp(parity);
            const int *const marks = sh.warp_drops + parity * kScanMostWarps;
            ScanMap<U> m = maps[0];
#pragma unroll 4
            for (int w = 1; w < warps; ++w) {
                const ScanMap<U> s = maps[w * 32];
                m.h = scan_apply(s, any ? marks[w] : 0, m.h);
                m.a = m.a * s.a;
            }
            if (lane == 0) scan_expect(sh.bar(parity), cluster * (32 * sizeof(ScanMap<U>) + (resets ? sizeof(int) : 0)));
            for (unsigned k = 0; k < cluster; ++k) {
                const unsigned bar = scan_peer(sh.bars + parity, k);
                scan_push(scan_peer(sh.cta(parity) + rank * 32, k), bar, m);
                if (resets && lane == 0) scan_push(scan_peer(sh.cta_drops + parity * kScanMostCluster + rank, k), bar, any);
            }
        }
        __syncwarp();
        lost = lost || !scan_await(sh.bar(parity), (turn >> 1) & 1);         // no later round waits for what is lost
        if (lost) {
            const U none = scan_all<U>(A(NAN));
            if (warp == warps - 1) sh.carry[(parity ^ 1) * 32] = none;
            return none;
        }
        if (resets) {
            const int4 *const q = reinterpret_cast<const int4 *>(sh.cta_drops + parity * kScanMostCluster);
            const int4 d = q[0], e = q[1];
            any = d.x | d.y | d.z | d.w | e.x | e.y | e.z | e.w;
        }
    }
    return any ? scan_joined<true, A>(sh, parity, rank, cluster, warp, own, drops) : scan_joined<false, A>(sh, parity, rank, cluster, warp, own, drops);
}
// After the last round, whose parity was the other one: what has left it.
template <class U>
__device__ __forceinline__ U scan_left(const ScanShared<U> &sh, int parity, U carry)
{
    if (sh.warps * sh.ctas == 1) return carry;
    __syncthreads();
    return sh.carry[parity * 32];
}

// The tokens of sequence b.
__device__ __forceinline__ int scan_length(const ScanParams &p, long long b)
{
    if (!p.lengths) return p.tokens;
    const long long n = p.long_lengths ? static_cast<const long long *>(p.lengths)[b] : static_cast<const int *>(p.lengths)[b];
    return n < 0 ? 0 : n > p.tokens ? p.tokens : (int)n;
}

// The end of the sequence, counted from the chunk's first token.
template <class Place>
__device__ __forceinline__ int scan_end(const ScanParams &p, const Place &at)
{
    return min(max(scan_length(p, at.b) - at.base, 0), at.tokens);
}
// A lane's channels of a state.
template <class U, class A, int V>
__device__ __forceinline__ U scan_state(const void *p, long long at, int count)
{
    const A *s = static_cast<const A *>(p) + at;
    const A s0 = p && count > 0 ? s[0] : A(0);
    if constexpr (V == 1) return s0;
    else return two(s0, p && count > 1 ? s[1] : A(0));
}
template <class U, class A, int V>
__device__ __forceinline__ void scan_keep(void *p, long long at, U u, int count)
{
    A *s = static_cast<A *>(p) + at;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v < count) s[v] = scan_part(u, v);
}

// Where a warp is in the call.
template <int V, bool CLUSTER>
struct ScanPlace {
    unsigned rank, cluster;
    int lane, warp, warps;
    long long b, state, piece;          // state: of the lane's first channel; piece: the same of its chunk's
    int base, tokens;                   // the chunk's first token, and its number of them
    int first, channel, count;          // first channel of the tile and of the lane, channels of the lane
    __device__ __forceinline__ explicit ScanPlace(const ScanParams &p) : rank(CLUSTER ? scan_rank() : 0), cluster(CLUSTER ? scan_cluster() : 1)
    {
        // the same for all lanes, and known to be: the addresses of rows are then computed once for the warp
        warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        const unsigned item = blockIdx.x / cluster, part = item / (unsigned)p.tiles, sequence = part / (unsigned)p.chunks;
        b = sequence;
        base = (int)(part - sequence * (unsigned)p.chunks) * p.chunk, tokens = min(p.chunk, p.tokens - base);
        first = (int)(item - part * (unsigned)p.tiles) * 32 * V, channel = first + lane * V;
        count = max(0, min(V, (int)p.channels - channel));
        state = b * p.channels + channel, piece = part * p.channels + channel;
    }
};

// A warp's ring: the segment that is worked on and one or two on their way, as leave two CTAs room on an SM.
template <class T, class G, int V, int S, bool GRAD>
struct ScanRing {
    static constexpr int kPart = ScanCopy<T, S, 32 * V>::kBytes;
    static constexpr int kSegment = (GRAD ? 3 : 1) * kPart + ScanCopy<G, S, 32 * V>::kBytes;
    static constexpr int kStages = kSegment <= 4096 ? 3 : 2;
    static constexpr int kBytes = kStages * kSegment;        // of a warp
};

// Bound by DRAM where there are CTAs enough (8 x 4096 x 2048 in bfloat16 72 to 77 us, 5.3 TB/s and more), by the rounds' exchange in clusters (1 x 65536 x
// 2560, gates in 32 bits, 352 to 358 us).  Segments of 16 tokens and rings of their own for the warps leave one barrier to a round.
// CLUSTER: launched in clusters.  Without them the code for them costs 3 to 5 us of 75 to 163 (8 x 4096 x 2048 in bfloat16).
template <class T, class G, int V, int S, bool CLUSTER>
__global__ void __launch_bounds__(kScanCta, 2) scan_kernel(const __grid_constant__ ScanParams p)
{
    using A = Acc<T>;
    using U = typename ScanUnit<A, V>::U;
    using Ring = ScanRing<T, G, V, S, false>;
    constexpr bool EXACT = sizeof(T) >= 4;
    extern __shared__ __align__(16) char scan_memory[];
    const ScanPlace<V, CLUSTER> at(p);
    wait_for_earlier();
    char *const ring = scan_memory + at.warp * Ring::kBytes;
    const ScanShared<U> sh(scan_memory + at.warps * Ring::kBytes, at.warps, at.cluster);
    // tokens are counted from the chunk's first one
    const int end = scan_end(p, at), round = at.cluster * at.warps * S;
    int t0 = (at.rank * at.warps + at.warp) * S;
    const long long xs = p.x_at.token * (int)sizeof(T), gs = p.gate_at.token * (int)sizeof(G), hs = p.h_at.token * (int)sizeof(T);
    const unsigned ho = at.channel * (unsigned)sizeof(T), hs_near = (unsigned)hs;
    const char *x = static_cast<const char *>(p.x) + (at.b * p.x_at.batch + at.first) * (int)sizeof(T) + (at.base + t0) * xs;
    const char *gate = static_cast<const char *>(p.gate) + (at.b * p.gate_at.batch + at.first) * (int)sizeof(G) + (at.base + t0) * gs;
    char *h = static_cast<char *>(p.h) + at.b * p.h_at.batch * (int)sizeof(T) + (at.base + t0) * hs;
    const ScanCopy<T, S, 32 * V> copy_x(p.whole & kScanX, at.lane, (int)p.channels - at.first, xs);
    const ScanCopy<G, S, 32 * V> copy_gate(p.whole & kScanGate, at.lane, (int)p.channels - at.first, gs);
    // easy: everything is in whole pieces and near, and the tile's channels are all there
    constexpr int kEasy = kScanX | kScanGate | kScanOut | kScanNear;
    const bool pairs = p.whole & kScanOut, easy = (p.whole & kEasy) == kEasy && at.first + 32 * V <= p.channels;
    const long long x_round = round * xs, gate_round = round * gs, h_round = round * hs;
    const unsigned char *reset = p.reset ? p.reset + at.b * p.reset_at.batch + at.base * p.reset_at.token : nullptr;
    int ahead = t0, in_stage = 0, stage = 0;
    auto issue = [&]() {
        char *to = ring + in_stage * Ring::kSegment;
        if (easy && ahead + S <= end) {
            copy_x.issue_all(to, x);
            copy_gate.issue_all(to + copy_x.kBytes, gate);
        } else {
            const auto valid = [&](int r) { return ahead + r < end; };
            copy_x.issue(to, x, xs, valid);
            copy_gate.issue(to + copy_x.kBytes, gate, gs, valid);
        }
        scan_issued();
        ahead += round, x += x_round, gate += gate_round, in_stage = in_stage + 1 == Ring::kStages ? 0 : in_stage + 1;
    };
    for (int k = 0; k < Ring::kStages - 1; ++k) issue();
    U carry = p.chunks > 1 ? scan_state<U, A, V>(p.carry, at.piece, at.count) : scan_state<U, A, V>(p.state, at.state, at.count);
    scan_begin(sh, at.warp, carry);
    auto marks = [&](int t) -> unsigned char { return reset && at.lane < S && t + at.lane < end ? reset[(t + at.lane) * p.reset_at.token] : 0; };
    unsigned char mark = marks(t0);
    int turn = 0;
    bool lost = false;
    for (int first = 0; first < at.tokens; first += round, ++turn) {
        const unsigned drops = __ballot_sync(0xffffffffu, mark != 0);
        scan_arrived<Ring::kStages - 2>();
        issue();                                         // where the stage before was
        const char *const from = ring + stage * Ring::kSegment + at.lane * V * (int)sizeof(T);
        const char *const from_gate = ring + stage * Ring::kSegment + copy_x.kBytes + at.lane * V * (int)sizeof(G);
        stage = stage + 1 == Ring::kStages ? 0 : stage + 1;
        U a[S], m[S];                                    // m becomes m(a) x
        with_mode(p.mode, [&](auto decay, auto mix) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                U rest;
                scan_decay<decay.value, EXACT, false, A>(scan_widen<U>(scan_piece<G, V>(from_gate + s * 32 * V * (int)sizeof(G))), a[s], rest);
                const U v = scan_widen<U>(scan_piece<T, V>(from + s * 32 * V * (int)sizeof(T)));
                if constexpr (mix.value == FO_MIX_ONE) m[s] = v;
                else m[s] = scan_mix<mix.value, EXACT, A>(a[s], rest) * v;
            }
        });
        mark = marks(t0 + round);
        const bool full = t0 + S <= end;
        if (!full)
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (t0 + s >= end) a[s] = scan_all<U>(A(1)), m[s] = scan_all<U>(A(0));      // the state stays as it is
        ScanMap<U> own = {a[0], m[0]};
        if (drops == 0) {
#pragma unroll
            for (int s = 1; s < S; ++s) own.h = fused_ma(a[s], own.h, m[s]), own.a = own.a * a[s];
        } else {
#pragma unroll
            for (int s = 1; s < S; ++s) own.h = (drops >> s) & 1u ? m[s] : fused_ma(a[s], own.h, m[s]), own.a = own.a * a[s];
        }
        U in = scan_join<A>(sh, turn, at.rank, at.cluster, at.warp, own, reset != nullptr, drops != 0, carry, lost);
        if (easy && full && drops == 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                in = fused_ma(a[s], in, m[s]);
                scan_store<T, V>(h, ho + s * hs_near, scan_narrow<T, V>(in));
            }
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                in = (drops >> s) & 1u ? m[s] : fused_ma(a[s], in, m[s]);
                if (t0 + s < at.tokens) scan_store<T, V>(h + s * hs, ho, scan_narrow<T, V>(t0 + s < end ? in : scan_all<U>(A(0))), at.count, pairs);
            }
        }
        t0 += round, h += h_round;
    }
    carry = scan_left(sh, turn & 1, carry);
    if (p.last && p.chunks == 1 && at.rank == 0 && at.warp == 0) scan_keep<U, A, V>(p.last, at.state, carry, at.count);
}

// The gradient: l_t = dh_t + u_{t+1}, u_t = a_t l_t is what comes to the token before (nothing through a reset), from the last token to
// the first.  Segments are counted from the end, and a segment's map is that of u.  8 x 4096 x 2048 in bfloat16 154 to 165 us (4.9 TB/s), at 59 % of
// issue; in float32 latencies come first, those of CUDA's exponential, division and root and of odd rows copied by elements (5 x 777 x 1001
// 51 us, 1.8 TB/s, 44 % of issue).
template <class T, class G, int V, int S, bool CLUSTER>
__global__ void __launch_bounds__(kScanCta, 2) scan_grad_kernel(const __grid_constant__ ScanParams p)
{
    using A = Acc<T>;
    using U = typename ScanUnit<A, V>::U;
    using Ring = ScanRing<T, G, V, S, true>;
    constexpr bool EXACT = sizeof(T) >= 4;
    constexpr int kPart = ScanCopy<T, S, 32 * V>::kBytes, kRow = 32 * V * (int)sizeof(T), kGateRow = 32 * V * (int)sizeof(G);
    extern __shared__ __align__(16) char scan_memory[];
    const ScanPlace<V, CLUSTER> at(p);
    wait_for_earlier();
    char *const ring = scan_memory + at.warp * Ring::kBytes;
    const ScanShared<U> sh(scan_memory + at.warps * Ring::kBytes, at.warps, at.cluster);
    // tokens are counted from the chunk's first one
    const int end = scan_end(p, at), round = at.cluster * at.warps * S;
    // element s of a segment is token t0 - s
    int t0 = at.tokens - 1 - (int)(at.rank * at.warps + at.warp) * S;
    const long long xs = p.x_at.token * (int)sizeof(T), gs = p.gate_at.token * (int)sizeof(G), ds = p.dh_at.token * (int)sizeof(T),
                    hs = p.h_in_at.token * (int)sizeof(T), dxs = p.h_at.token * (int)sizeof(T), dgs = p.dgate_at.token * (int)sizeof(G);
    const unsigned xo = at.channel * (unsigned)sizeof(T), go = at.channel * (unsigned)sizeof(G), dxs_near = (unsigned)dxs, dgs_near = (unsigned)dgs;
    // pointers are to the segment's last element, the lowest in memory
    const int lowest = at.base + t0 - (S - 1);
    const char *x = static_cast<const char *>(p.x) + (at.b * p.x_at.batch + at.first) * (int)sizeof(T) + lowest * xs;
    const char *dh = static_cast<const char *>(p.dh) + (at.b * p.dh_at.batch + at.first) * (int)sizeof(T) + lowest * ds;
    const char *hin = static_cast<const char *>(p.h_in) + (at.b * p.h_in_at.batch + at.first) * (int)sizeof(T) + (lowest - 1) * hs;  // of the token before
    const char *gate = static_cast<const char *>(p.gate) + (at.b * p.gate_at.batch + at.first) * (int)sizeof(G) + lowest * gs;
    char *dx = static_cast<char *>(p.h) + at.b * p.h_at.batch * (int)sizeof(T) + lowest * dxs;
    char *dgate = static_cast<char *>(p.dgate) + at.b * p.dgate_at.batch * (int)sizeof(G) + lowest * dgs;
    const int channels = (int)p.channels - at.first;
    const ScanCopy<G, S, 32 * V> copy_gate(p.whole & kScanGate, at.lane, channels, -gs);
    const ScanCopy<T, S, 32 * V> copy_x(p.whole & kScanX, at.lane, channels, -xs), copy_dh(p.whole & kScanDh, at.lane, channels, -ds),
        copy_h(p.whole & kScanH, at.lane, channels, -hs);
    // easy: everything is in whole pieces and near, and the tile's channels are all there
    const bool pairs = p.whole & kScanOut, gate_pairs = p.whole & kScanOutGate, easy = p.whole == kScanAll && at.first + 32 * V <= p.channels;
    const long long x_round = round * xs, dh_round = round * ds, h_round = round * hs, gate_round = round * gs, dx_round = round * dxs,
                    dgate_round = round * dgs;
    const unsigned char *reset = p.reset ? p.reset + at.b * p.reset_at.batch + at.base * p.reset_at.token : nullptr;
    const bool with_x = p.mode % 3 != FO_MIX_ONE, with_dh = p.dh != nullptr;
    const int lead = at.base == 0 ? S : S - 1;           // segments from this token on have a token of the sequence before each of theirs
    int ahead = t0, in_stage = 0, stage = 0;
    auto issue = [&]() {
        char *to = ring + in_stage * Ring::kSegment;
        if (easy && ahead < end && ahead >= lead) {
            if (with_dh) copy_dh.issue_all(to, dh);
            if (with_x) copy_x.issue_all(to + kPart, x);
            copy_h.issue_all(to + 2 * kPart, hin);
            copy_gate.issue_all(to + 3 * kPart, gate);
        } else {
            const auto valid = [&](int r) { return ahead - r >= 0 && ahead - r < end; };
            if (with_dh) copy_dh.issue(to, dh + (S - 1) * ds, -ds, valid);
            if (with_x) copy_x.issue(to + kPart, x + (S - 1) * xs, -xs, valid);
            copy_h.issue(to + 2 * kPart, hin + (S - 1) * hs, -hs, [&](int r) { return at.base + ahead - r > 0 && ahead - r >= 0 && ahead - r < end; });
            copy_gate.issue(to + 3 * kPart, gate + (S - 1) * gs, -gs, valid);
        }
        scan_issued();
        ahead -= round, x -= x_round, dh -= dh_round, hin -= h_round, gate -= gate_round;
        in_stage = in_stage + 1 == Ring::kStages ? 0 : in_stage + 1;
    };
    for (int k = 0; k < Ring::kStages - 1; ++k) issue();
    U carry = p.chunks > 1 ? scan_state<U, A, V>(p.carry, at.piece, at.count) : scan_state<U, A, V>(p.dlast, at.state, at.count);
    const U start = scan_state<U, A, V>(p.state, at.state, at.count), none = scan_all<U>(A(0));
    scan_begin(sh, at.warp, carry);
    auto marks = [&](int t) -> unsigned char {
        return reset && at.lane < S && t - at.lane >= 0 && t - at.lane < end ? reset[(t - at.lane) * p.reset_at.token] : 0;
    };
    unsigned char mark = marks(t0);
    int turn = 0;
    bool lost = false;
    for (int first = 0; first < at.tokens; first += round, ++turn) {
        const unsigned drops = __ballot_sync(0xffffffffu, mark != 0);
        scan_arrived<Ring::kStages - 2>();
        issue();                                         // where the stage before was
        const char *const from = ring + stage * Ring::kSegment + at.lane * V * (int)sizeof(T);
        const char *const from_gate = ring + stage * Ring::kSegment + 3 * kPart + at.lane * V * (int)sizeof(G);
        stage = stage + 1 == Ring::kStages ? 0 : stage + 1;
        auto d_of = [&](int s) { return with_dh ? scan_widen<U>(scan_piece<T, V>(from + s * kRow)) : none; };
        auto x_of = [&](int s) { return scan_widen<U>(scan_piece<T, V>(from + kPart + s * kRow)); };
        auto h_of = [&](int s) { return scan_widen<U>(scan_piece<T, V>(from + 2 * kPart + s * kRow)); };
        U a[S], rest[S];
        with_decay(p.mode, [&](auto decay) {
#pragma unroll
            for (int s = 0; s < S; ++s) scan_decay<decay.value, EXACT, true, A>(scan_widen<U>(scan_piece<G, V>(from_gate + s * kGateRow)), a[s], rest[s]);
        });
        mark = marks(t0 - round);
        // plain: all of the segment's tokens are the sequence's, and none of them its first one or drops what comes
        const bool plain = t0 < end && t0 >= lead && drops == 0;
        ScanMap<U> own = {scan_all<U>(A(1)), none};
        if (plain) {
#pragma unroll
            for (int s = 0; s < S; ++s) own.h = a[s] * (d_of(s) + own.h), own.a = own.a * a[s];
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (t0 - s >= 0 && t0 - s < end) own.h = (drops >> s) & 1u ? none : a[s] * (d_of(s) + own.h), own.a = own.a * a[s];
        }
        U in = scan_join<A>(sh, turn, at.rank, at.cluster, at.warp, own, reset != nullptr, drops != 0, carry, lost);
        auto finish = [&](auto decay, auto mix, auto masked) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                U da, dm;
                const U m = scan_mix<mix.value, EXACT, A>(a[s], rest[s]), l = d_of(s) + in;
                scan_slopes<decay.value, mix.value, EXACT, A>(a[s], rest[s], m, da, dm);
                U to_x = m * l, before = h_of(s), through = a[s] * l, slope;
                if constexpr (masked.value) {
                    const bool drop = (drops >> s) & 1u;
                    if (at.base + t0 - s == 0) before = start;
                    if (drop) before = none, through = none;
                }
                if constexpr (mix.value == FO_MIX_ONE) slope = da * before;
                else if constexpr (mix.value == FO_MIX_REST) slope = da * fused_ma(x_of(s), scan_all<U>(A(-1)), before);
                else slope = fused_ma(dm, x_of(s), da * before);
                U to_g = l * slope;
                if constexpr (masked.value) {
                    const bool live = t0 - s >= 0 && t0 - s < end;
                    if (!live) to_x = none, to_g = none, through = in;
                }
                if constexpr (!masked.value) {
                    scan_store<T, V>(dx, xo + (S - 1 - s) * dxs_near, scan_narrow<T, V>(to_x));
                    scan_store<G, V>(dgate, go + (S - 1 - s) * dgs_near, scan_narrow<G, V>(to_g));
                } else if (t0 - s >= 0) {
                    scan_store<T, V>(dx + (S - 1 - s) * dxs, xo, scan_narrow<T, V>(to_x), at.count, pairs);
                    scan_store<G, V>(dgate + (S - 1 - s) * dgs, go, scan_narrow<G, V>(to_g), at.count, gate_pairs);
                }
                in = through;
            }
        };
        if (plain && easy) with_mode(p.mode, [&](auto decay, auto mix) { finish(decay, mix, std::false_type()); });
        else with_mode(p.mode, [&](auto decay, auto mix) { finish(decay, mix, std::true_type()); });
        t0 -= round, dx -= dx_round, dgate -= dgate_round;
    }
    carry = scan_left(sh, turn & 1, carry);
    if (p.last && p.chunks == 1 && at.rank == 0 && at.warp == 0) scan_keep<U, A, V>(p.last, at.state, carry, at.count);
}

// The map of each chunk: its warps take an equal part of its tokens each, segment after segment, and put their maps together.
// GRAD: the map of u, from the last token to the first.  Bound by its reading: with the two kernels after it 1 x 16384 x 512 in float32 takes
// 41 us forwards and 58 backwards, 1.5 and 1.7 TB/s.
template <class T, class G, int V>
struct ScanMapRing {
    static constexpr int S = 8;
    static constexpr int kPart = ScanCopy<T, S, 32 * V>::kBytes, kSegment = kPart + ScanCopy<G, S, 32 * V>::kBytes;
    static constexpr int kStages = 12288 / kSegment < 6 ? 12288 / kSegment : 6;
    static constexpr int kBytes = kStages * kSegment;        // of a warp
};
template <class T, class G, int V, bool GRAD>
__global__ void __launch_bounds__(kScanCta, 2) scan_map_kernel(const __grid_constant__ ScanParams p)
{
    using A = Acc<T>;
    using U = typename ScanUnit<A, V>::U;
    using Ring = ScanMapRing<T, G, V>;
    constexpr bool EXACT = sizeof(T) >= 4;
    constexpr int S = Ring::S;
    extern __shared__ __align__(16) char scan_memory[];
    const ScanPlace<V, false> at(p);
    wait_for_earlier();
    char *const ring = scan_memory + at.warp * Ring::kBytes;
    // the part is tokens low .. high - 1 of the chunk; element s of a segment is token t0 + s, of the gradient's t0 - s
    const int part = (at.tokens + at.warps * S - 1) / (at.warps * S) * S;
    const int low = min(at.tokens, at.warp * part), high = max(low, min(scan_end(p, at), low + part));
    constexpr int kWay = GRAD ? -1 : 1;
    int t0 = GRAD ? high - 1 : low;
    const int lowest = at.base + (GRAD ? t0 - (S - 1) : t0);         // the pointers' token, the segment's first in memory
    const fo_rows x_at = GRAD ? p.dh_at : p.x_at;
    const long long xs = x_at.token * (int)sizeof(T), gs = p.gate_at.token * (int)sizeof(G);
    const char *x = static_cast<const char *>(GRAD ? p.dh : p.x) + (at.b * x_at.batch + at.first) * (int)sizeof(T) + lowest * xs;
    const char *gate = static_cast<const char *>(p.gate) + (at.b * p.gate_at.batch + at.first) * (int)sizeof(G) + lowest * gs;
    constexpr int kX = GRAD ? kScanDh : kScanX, kEasy = kX | kScanGate | kScanNear;
    const ScanCopy<T, S, 32 * V> copy_x(p.whole & kX, at.lane, (int)p.channels - at.first, kWay * xs);
    const ScanCopy<G, S, 32 * V> copy_gate(p.whole & kScanGate, at.lane, (int)p.channels - at.first, kWay * gs);
    const bool easy = (p.whole & kEasy) == kEasy && at.first + 32 * V <= p.channels, with_x = !GRAD || p.dh;
    const unsigned char *const reset = p.reset ? p.reset + at.b * p.reset_at.batch + at.base * p.reset_at.token : nullptr;
    int left = high - low, to_come = left, in_stage = 0, stage = 0;       // tokens of the part that are not worked on, not asked for
    auto issue = [&]() {
        char *const to = ring + in_stage * Ring::kSegment;
        if (easy && to_come >= S) {
            if (with_x) copy_x.issue_all(to, x);
            copy_gate.issue_all(to + Ring::kPart, gate);
        } else {
            const auto valid = [&](int r) { return r < to_come; };
            if (with_x) copy_x.issue(to, GRAD ? x + (S - 1) * xs : x, kWay * xs, valid);
            copy_gate.issue(to + Ring::kPart, GRAD ? gate + (S - 1) * gs : gate, kWay * gs, valid);
        }
        scan_issued();
        to_come -= S, x += kWay * S * xs, gate += kWay * S * gs, in_stage = in_stage + 1 == Ring::kStages ? 0 : in_stage + 1;
    };
    for (int k = 0; k < Ring::kStages - 1; ++k) issue();
    auto marks = [&](int t, int there) -> unsigned char {
        return reset && at.lane < S && at.lane < there ? reset[(t + kWay * at.lane) * p.reset_at.token] : 0;
    };
    unsigned char mark = marks(t0, left);
    ScanMap<U> own = {scan_all<U>(A(1)), scan_all<U>(A(0))};
    unsigned dropped = 0;
    for (; left > 0; left -= S) {
        const unsigned drops = __ballot_sync(0xffffffffu, mark != 0);
        dropped |= drops;
        scan_arrived<Ring::kStages - 2>();
        issue();                                         // where the stage before was
        const char *const from = ring + stage * Ring::kSegment + at.lane * V * (int)sizeof(T);
        const char *const from_gate = ring + stage * Ring::kSegment + Ring::kPart + at.lane * V * (int)sizeof(G);
        stage = stage + 1 == Ring::kStages ? 0 : stage + 1;
        U a[S], m[S];                                    // m: m(a) x forwards, dh backwards
        with_mode(p.mode, [&](auto decay, auto mix) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                U rest;
                scan_decay<decay.value, EXACT, GRAD, A>(scan_widen<U>(scan_piece<G, V>(from_gate + s * 32 * V * (int)sizeof(G))), a[s], rest);
                m[s] = with_x ? scan_widen<U>(scan_piece<T, V>(from + s * 32 * V * (int)sizeof(T))) : scan_all<U>(A(0));
                if constexpr (!GRAD && mix.value != FO_MIX_ONE) m[s] = scan_mix<mix.value, EXACT, A>(a[s], rest) * m[s];
            }
        });
        t0 += kWay * S;
        mark = marks(t0, left - S);
        if (left < S)
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (s >= left) a[s] = scan_all<U>(A(1)), m[s] = scan_all<U>(A(0));      // the state stays as it is
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const bool drop = (drops >> s) & 1u;
            if constexpr (GRAD) own.h = drop ? scan_all<U>(A(0)) : a[s] * (m[s] + own.h);
            else own.h = drop ? m[s] : fused_ma(a[s], own.h, m[s]);
            own.a = own.a * a[s];
        }
    }
    scan_arrived<0>();
    __syncthreads();                                     // the rings' memory is taken for the maps
    ScanMap<U> *const maps = reinterpret_cast<ScanMap<U> *>(scan_memory);
    int *const parts_drop = reinterpret_cast<int *>(maps + kScanMostWarps * 32);
    maps[at.warp * 32 + at.lane] = own;
    if (at.lane == 0) parts_drop[at.warp] = dropped != 0;
    __syncthreads();
    if (at.warp) return;
    int any = 0;
    ScanMap<U> all = {scan_all<U>(A(1)), scan_all<U>(A(0))};
    for (int k = 0; k < at.warps; ++k) {
        const int w = GRAD ? at.warps - 1 - k : k;
        any |= parts_drop[w];
        all.h = scan_apply(maps[w * 32 + at.lane], parts_drop[w], all.h), all.a = all.a * maps[w * 32 + at.lane].a;
    }
    scan_keep<U, A, V>(p.map_a, at.piece, all.a, at.count);
    scan_keep<U, A, V>(p.map_h, at.piece, all.h, at.count);
    if (at.first == 0 && at.lane == 0) p.map_drops[at.b * p.chunks + at.base / p.chunk] = any;
}
// What comes into every chunk, and what leaves the last one: a thread to a channel of a sequence.
template <class A, bool GRAD>
__global__ void __launch_bounds__(kScanCta) scan_carry_kernel(const __grid_constant__ ScanParams p)
{
    constexpr int kAhead = 16;                           // maps that are on their way together
    wait_for_earlier();
    const long long at = (long long)blockIdx.x * kScanCta + threadIdx.x, b = at / p.channels, c = at - b * p.channels;
    if (b >= p.batch) return;
    const void *const in = GRAD ? p.dlast : p.state;
    A carry = in ? static_cast<const A *>(in)[at] : A(0);
    for (int first = 0; first < p.chunks; first += kAhead) {
        ScanMap<A> m[kAhead];
        int drops[kAhead];
        const auto part = [&](int k) { return b * p.chunks + (GRAD ? p.chunks - 1 - k : k); };
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (first + k >= p.chunks) continue;
            const long long q = part(first + k) * p.channels + c;
            m[k] = {static_cast<const A *>(p.map_a)[q], static_cast<const A *>(p.map_h)[q]}, drops[k] = p.map_drops[part(first + k)];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (first + k >= p.chunks) continue;
            static_cast<A *>(p.carry)[part(first + k) * p.channels + c] = carry;
            carry = scan_apply(m[k], drops[k], carry);
        }
    }
    if (p.last) static_cast<A *>(p.last)[at] = carry;
}

// A few tokens (a decoding step): every thread takes its channels through them, one after the other.
template <class T, class G, int V>
__global__ void __launch_bounds__(kScanCta) scan_step_kernel(const __grid_constant__ ScanParams p)
{
    using A = Acc<T>;
    using U = typename ScanUnit<A, V>::U;
    constexpr bool EXACT = sizeof(T) >= 4;
    wait_for_earlier();
    const long long per = (p.channels + V - 1) / V, at = (long long)blockIdx.x * kScanCta + threadIdx.x, b = at / per;
    if (b >= p.batch) return;
    const int c = (int)(at - b * per) * V, count = min(V, (int)(p.channels - c));
    const int end = scan_length(p, b);
    const T *x = static_cast<const T *>(p.x) + b * p.x_at.batch + c;
    const G *gate = static_cast<const G *>(p.gate) + b * p.gate_at.batch + c;
    T *h = static_cast<T *>(p.h) + b * p.h_at.batch + c;
    const unsigned char *reset = p.reset ? p.reset + b * p.reset_at.batch : nullptr;
    constexpr int kPairs = kScanX | kScanGate | kScanOut;
    const bool whole = count == V && (p.whole & kPairs) == kPairs;
    U state = scan_state<U, A, V>(p.state, b * p.channels + c, count);
    for (int t = 0; t < p.tokens; ++t, x += p.x_at.token, gate += p.gate_at.token, h += p.h_at.token) {
        U out = scan_all<U>(A(0));
        if (t < end) {
            ScanPiece<T, V> xv;
            ScanPiece<G, V> gv;
            if (whole) {
                xv = scan_piece<T, V>(reinterpret_cast<const char *>(x)), gv = scan_piece<G, V>(reinterpret_cast<const char *>(gate));
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) xv.v[v] = x[v < count ? v : 0], gv.v[v] = gate[v < count ? v : 0];
            }
            const bool drop = reset && reset[t * p.reset_at.token];
            with_mode(p.mode, [&](auto decay, auto mix) {
                U a, rest;
                scan_decay<decay.value, EXACT, false, A>(scan_widen<U>(gv), a, rest);
                const U m = scan_mix<mix.value, EXACT, A>(a, rest) * scan_widen<U>(xv);
                state = drop ? m : fused_ma(a, state, m);
            });
            out = state;
        }
        scan_store<T, V>(reinterpret_cast<char *>(h), 0, scan_narrow<T, V>(out), count, whole);
    }
    if (p.last) scan_keep<U, A, V>(p.last, b * p.channels + c, state, count);
}

// Host: one kernel of a pair of types; scan_*.cu instantiate it.
template <class T, class G>
cudaError_t launch_scan(ScanParams p, bool grad, void *ws, cudaStream_t st);

}  // namespace fo
