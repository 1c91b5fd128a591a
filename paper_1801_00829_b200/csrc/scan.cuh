// A gated linear recurrence over the tokens, h_t = a_t h_{t-1} + m(a_t) x_t, and its gradient, the same recurrence backwards.
//
// A thread works on V neighbouring channels over S successive tokens (a segment), a CTA on 32 V channels over as many segments as
// it has warps, a cluster on as many as its CTAs have together: that is one round, and rounds follow each other over
// the sequence.  In a round every warp runs its segment from zero, which gives the map h -> A h + H of the whole segment, the maps
// are put one behind the other in the order of the tokens, and with the state that comes in the segment is run again, from
// registers.  So the inputs are read once and no CTA waits for another outside its cluster, whose CTAs run together.
// The next round's inputs are on their way meanwhile.
#pragma once

#include "elem.cuh"
#include "../../include/fusedops_lm.h"

namespace fo {

constexpr int kScanMostWarps = 16;
constexpr int kScanMostCluster = 8;

struct ScanParams {
    long long tokens, channels, tiles;  // tiles: of 32 V channels
    int mode, long_lengths;             // mode: decay * 3 + mix
    const void *x, *gate, *state, *lengths;
    const unsigned char *reset;
    void *h, *last;                     // gradient: dx, dstate
    fo_rows x_at, gate_at, reset_at, h_at;
    // the gradient's own
    const void *dh, *dlast, *h_in;
    void *dgate;
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
__device__ __forceinline__ ScanPiece<T, V> scan_load(const T *p)
{
    ScanPiece<T, V> r;
    if constexpr (V * sizeof(T) == 4) *reinterpret_cast<uint32_t *>(&r) = *reinterpret_cast<const uint32_t *>(p);
    else if constexpr (V * sizeof(T) == 8) *reinterpret_cast<uint2 *>(&r) = *reinterpret_cast<const uint2 *>(p);
    else if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4 *>(&r) = *reinterpret_cast<const uint4 *>(p);
    else r.v[0] = p[0];
    return r;
}
template <class T, int V>
__device__ __forceinline__ void scan_store(T *p, const ScanPiece<T, V> &r)
{
    if constexpr (V * sizeof(T) == 4) *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(&r);
    else if constexpr (V * sizeof(T) == 8) *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(&r);
    else if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(&r);
    else p[0] = r.v[0];
}

// ------------------------------------------------------------------------------------------------ decays
// a and 1 - a, both without cancellation.  A decay near 1 multiplies a state very many times, so that its error adds up over
// 1 / (1 - a) tokens: it is 1 minus its small complement, and so rounded once.  EXACT (32- and 64-bit x): by CUDA's functions; else by
// the hardware's exponential and reciprocal, whose relative error of a few 2^-23 is then one of the complement.
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

constexpr float kLog2e = 1.4426950408889634f;

template <int DECAY, bool EXACT>
__device__ __forceinline__ void scan_decay(float g, float &a, float &rest)
{
    if constexpr (DECAY == FO_DECAY_VALUE) {
        a = g, rest = 1.0f - g;
    } else if constexpr (DECAY == FO_DECAY_SIGMOID) {
        const float e = EXACT ? expf(-fabsf(g)) : scan_exp2(-fabsf(g) * kLog2e);
        const float small = e * scan_over<EXACT>(1.0f + e), big = 1.0f - small;
        a = g >= 0.0f ? big : small, rest = g >= 0.0f ? small : big;
    } else if constexpr (EXACT) {
        rest = -expm1f(g);
        a = g > -0.5f ? 1.0f - rest : expf(g);
    } else {
        // exp(g) - 1 by its series up to g^6 / 720 where it is small: the rest is below 2^-25 of it
        float m = fused_ma(g, 1.0f / 720.0f, 1.0f / 120.0f);
        m = fused_ma(m, g, 1.0f / 24.0f);
        m = fused_ma(m, g, 1.0f / 6.0f);
        m = fused_ma(m, g, 0.5f);
        m = fused_ma(m * g, g, g);
        const float e = scan_exp2(g * kLog2e);
        const bool near = fabsf(g) < 0.25f;
        a = near ? 1.0f + m : e, rest = near ? -m : 1.0f - e;
    }
}
template <int DECAY, bool EXACT>
__device__ __forceinline__ void scan_decay(double g, double &a, double &rest)
{
    if constexpr (DECAY == FO_DECAY_VALUE) {
        a = g, rest = 1.0 - g;
    } else if constexpr (DECAY == FO_DECAY_SIGMOID) {
        const double e = exp(-fabs(g)), small = e / (1.0 + e), big = 1.0 - small;
        a = g >= 0.0 ? big : small, rest = g >= 0.0 ? small : big;
    } else {
        rest = -expm1(g);
        a = g > -0.5 ? 1.0 - rest : exp(g);
    }
}
// m(a)
template <int MIX, bool EXACT, class A>
__device__ __forceinline__ A scan_mix(A a, A rest)
{
    if constexpr (MIX == FO_MIX_ONE) return A(1);
    else if constexpr (MIX == FO_MIX_REST) return rest;
    else return scan_root<EXACT>(rest * (A(1) + a));
}
// The derivatives of a and of m to the gate.
template <int DECAY, int MIX, bool EXACT, class A>
__device__ __forceinline__ void scan_slopes(A a, A rest, A m, A &da, A &dm)
{
    da = DECAY == FO_DECAY_VALUE ? A(1) : DECAY == FO_DECAY_EXP ? a : a * rest;
    if constexpr (MIX == FO_MIX_ONE) dm = A(0);
    else if constexpr (MIX == FO_MIX_REST) dm = -da;
    else if constexpr (DECAY == FO_DECAY_SIGMOID) dm = -a * a * m * scan_over<EXACT>(A(1) + a);      // a' = a (1 - a) has m in it
    else dm = -a * da * scan_over<EXACT>(m);
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

// ------------------------------------------------------------------------------------------------ segments put together
template <class A>
struct alignas(2 * sizeof(A)) ScanMap {
    A a, h;
};

// The shared memory of a CTA, twice (one round's is written while another warp still reads the last one's).
template <class A, int V>
struct ScanShared {
    ScanMap<A> *warp_maps, *cta_maps;                    // of every warp's segment, and of every CTA's segments
    int *warp_drops, *cta_drops;                         // a reset lies in them: nothing comes through
    int warps, ctas;

    static __host__ __device__ size_t bytes(int warps, int ctas)
    {
        return warps * ctas == 1 ? 0 : 2 * (warps + ctas) * (V * 32 * sizeof(ScanMap<A>) + sizeof(int));
    }
    __device__ __forceinline__ ScanShared(void *at, int w, int c) : warps(w), ctas(c)
    {
        warp_maps = static_cast<ScanMap<A> *>(at), cta_maps = warp_maps + 2 * w * V * 32;
        warp_drops = reinterpret_cast<int *>(cta_maps + 2 * c * V * 32), cta_drops = warp_drops + 2 * w;
    }
    __device__ __forceinline__ ScanMap<A> &warp(int parity, int w, int v) const { return warp_maps[((parity * warps + w) * V + v) * 32 + (threadIdx.x & 31)]; }
    __device__ __forceinline__ ScanMap<A> &cta(int parity, int c, int v) const { return cta_maps[((parity * ctas + c) * V + v) * 32 + (threadIdx.x & 31)]; }
    __device__ __forceinline__ int &warp_drop(int parity, int w) const { return warp_drops[parity * warps + w]; }
    __device__ __forceinline__ int &cta_drop(int parity, int c) const { return cta_drops[parity * ctas + c]; }
};

template <class A>
__device__ __forceinline__ A scan_apply(const ScanMap<A> &m, int drops, A c)
{
    return drops ? m.h : fused_ma(m.a, c, m.h);
}
__device__ __forceinline__ void scan_push(unsigned to, const ScanMap<float> &m)
{
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(m.a), "f"(m.h) : "memory");
}
__device__ __forceinline__ void scan_push(unsigned to, const ScanMap<double> &m)
{
    asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(to), "d"(m.a), "d"(m.h) : "memory");
}

// Every warp gives its segment's map (and whether it drops what comes in); carry is what comes into the round.  Returns what
// comes into the warp's segment, and sets carry to what leaves the round.  One barrier, a second one of the cluster.
template <class A, int V>
__device__ __forceinline__ void scan_join(const ScanShared<A, V> &sh, int parity, unsigned rank, unsigned cluster, const A (&a)[V],
                                          const A (&h)[V], int drops, A (&carry)[V], A (&in)[V])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = sh.warps;
    if (warps == 1 && cluster == 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = carry[v], carry[v] = scan_apply({a[v], h[v]}, drops, carry[v]);
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) sh.warp(parity, warp, v) = {a[v], h[v]};
    if (lane == 0) sh.warp_drop(parity, warp) = drops;
    __syncthreads();
    if (cluster > 1) {
        if (warp == 0) {
            int any = 0;
            ScanMap<A> m[V];
#pragma unroll
            for (int v = 0; v < V; ++v) m[v] = {A(1), A(0)};
            for (int w = 0; w < warps; ++w) {
                const int d = sh.warp_drop(parity, w);
                any |= d;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const ScanMap<A> s = sh.warp(parity, w, v);
                    m[v].h = scan_apply(s, d, m[v].h);
                    m[v].a *= s.a;
                }
            }
            for (unsigned k = 0; k < cluster; ++k) {
#pragma unroll
                for (int v = 0; v < V; ++v) scan_push(scan_peer(&sh.cta(parity, rank, v), k), m[v]);
                if (lane == 0)
                    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(scan_peer(&sh.cta_drop(parity, rank), k)), "r"(any) : "memory");
            }
        }
        __syncwarp();
        scan_arrive();
        scan_wait();
        A c[V];
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = in[v] = carry[v];
        for (unsigned k = 0; k < cluster; ++k) {
            const int d = sh.cta_drop(parity, k);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (k == rank) in[v] = c[v];
                c[v] = scan_apply(sh.cta(parity, k, v), d, c[v]);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = c[v];
        for (int w = 0; w < warp; ++w) {
            const int d = sh.warp_drop(parity, w);
#pragma unroll
            for (int v = 0; v < V; ++v) in[v] = scan_apply(sh.warp(parity, w, v), d, in[v]);
        }
        return;
    }
    A c[V];
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = in[v] = carry[v];
    for (int w = 0; w < warps; ++w) {
        const int d = sh.warp_drop(parity, w);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (w == warp) in[v] = c[v];
            c[v] = scan_apply(sh.warp(parity, w, v), d, c[v]);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = c[v];
}

// The tokens of sequence b.
__device__ __forceinline__ long long scan_length(const ScanParams &p, long long b)
{
    if (!p.lengths) return p.tokens;
    const long long n = p.long_lengths ? static_cast<const long long *>(p.lengths)[b] : static_cast<const int *>(p.lengths)[b];
    return n < 0 ? 0 : n > p.tokens ? p.tokens : n;
}

template <class T, class G, int V, int S>
__global__ void __launch_bounds__(kScanMostWarps * 32) scan_kernel(const __grid_constant__ ScanParams p)
{
    using A = Acc<T>;
    constexpr bool EXACT = sizeof(T) >= 4;
    extern __shared__ __align__(16) unsigned char scan_memory[];
    const unsigned rank = scan_rank(), cluster = scan_cluster();
    const ScanShared<A, V> sh(scan_memory, blockDim.x >> 5, cluster);
    if (cluster > 1) scan_arrive();                      // waited for before the first push: every CTA has started by then
    wait_for_earlier();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const long long item = blockIdx.x / cluster, b = item / p.tiles, c = (item - b * p.tiles) * (32 * V) + lane * V;
    const bool on = c < p.channels;
    const long long end = scan_length(p, b);
    const T *x = static_cast<const T *>(p.x) + b * p.x_at.batch + c;
    const G *gate = static_cast<const G *>(p.gate) + b * p.gate_at.batch + c;
    const unsigned char *reset = p.reset ? p.reset + b * p.reset_at.batch : nullptr;
    T *h = static_cast<T *>(p.h) + b * p.h_at.batch + c;
    A carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = p.state && on ? static_cast<const A *>(p.state)[b * p.channels + c + v] : A(0);
    if (cluster > 1) scan_wait();

    ScanPiece<T, V> xn[S];
    ScanPiece<G, V> gn[S];
    unsigned char mark = 0;
    const long long round = (long long)cluster * warps * S;
    long long t0 = ((long long)rank * warps + warp) * S;
    auto fetch = [&](long long t) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (on && t + s < end) {
                xn[s] = scan_load<T, V>(x + (t + s) * p.x_at.token);
                gn[s] = scan_load<G, V>(gate + (t + s) * p.gate_at.token);
            }
        }
        mark = reset && lane < S && t + lane < end ? reset[(t + lane) * p.reset_at.token] : 0;
    };
    fetch(t0);
    int parity = 0;
    for (long long first = 0; first < p.tokens; first += round, t0 += round, parity ^= 1) {
        const unsigned drops = __ballot_sync(0xffffffffu, mark != 0);
        A a[S][V], m[S][V];                              // m becomes m(a) x
        with_mode(p.mode, [&](auto decay, auto mix) {
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    A rest;
                    scan_decay<decay.value, EXACT>((A)widen(gn[s].v[v]), a[s][v], rest);
                    m[s][v] = scan_mix<mix.value, EXACT>(a[s][v], rest) * widen(xn[s].v[v]);
                    if (!on || t0 + s >= end) a[s][v] = A(1), m[s][v] = A(0);    // the state stays as it is
                }
        });
        fetch(t0 + round);
        A through[V], hs[V], in[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            through[v] = A(1), hs[v] = A(0);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const bool drop = (drops >> s) & 1u;
                hs[v] = drop ? m[s][v] : fused_ma(a[s][v], hs[v], m[s][v]);
                through[v] *= a[s][v];
            }
        }
        scan_join(sh, parity, rank, cluster, through, hs, drops != 0, carry, in);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            ScanPiece<T, V> out;
            const bool drop = (drops >> s) & 1u;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                in[v] = drop ? m[s][v] : fused_ma(a[s][v], in[v], m[s][v]);
                out.v[v] = narrow<T>(t0 + s < end ? in[v] : A(0));
            }
            if (on && t0 + s < p.tokens) scan_store<T, V>(h + (t0 + s) * p.h_at.token, out);
        }
    }
    if (p.last && on && rank == 0 && warp == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) static_cast<A *>(p.last)[b * p.channels + c + v] = carry[v];
}

// The gradient: l_t = dh_t + u_{t+1}, u_t = a_t l_t is what comes to the token before (nothing through a reset), from the last token to
// the first.  Segments are counted from the end, and a segment's map is that of u.
template <class T, class G, int V, int S>
__global__ void __launch_bounds__(kScanMostWarps * 32) scan_grad_kernel(const __grid_constant__ ScanParams p)
{
    using A = Acc<T>;
    constexpr bool EXACT = sizeof(T) >= 4;
    extern __shared__ __align__(16) unsigned char scan_memory[];
    const unsigned rank = scan_rank(), cluster = scan_cluster();
    const ScanShared<A, V> sh(scan_memory, blockDim.x >> 5, cluster);
    if (cluster > 1) scan_arrive();
    wait_for_earlier();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const long long item = blockIdx.x / cluster, b = item / p.tiles, c = (item - b * p.tiles) * (32 * V) + lane * V;
    const bool on = c < p.channels;
    const long long end = scan_length(p, b);
    const T *x = static_cast<const T *>(p.x) + b * p.x_at.batch + c;
    const T *dh = static_cast<const T *>(p.dh) + b * p.dh_at.batch + c;
    const T *hin = static_cast<const T *>(p.h_in) + b * p.h_in_at.batch + c;
    const G *gate = static_cast<const G *>(p.gate) + b * p.gate_at.batch + c;
    const unsigned char *reset = p.reset ? p.reset + b * p.reset_at.batch : nullptr;
    T *dx = static_cast<T *>(p.h) + b * p.h_at.batch + c;
    G *dgate = static_cast<G *>(p.dgate) + b * p.dgate_at.batch + c;
    const bool with_x = p.mode % 3 != FO_MIX_ONE, with_dh = p.dh != nullptr;
    A carry[V], start[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        carry[v] = p.dlast && on ? static_cast<const A *>(p.dlast)[b * p.channels + c + v] : A(0);
        start[v] = p.state && on ? static_cast<const A *>(p.state)[b * p.channels + c + v] : A(0);
    }
    if (cluster > 1) scan_wait();

    ScanPiece<T, V> xn[S], dn[S], hn[S];
    ScanPiece<G, V> gn[S];
    unsigned char mark = 0;
    const long long round = (long long)cluster * warps * S;
    // element s of a segment is token t0 - s
    long long t0 = p.tokens - 1 - ((long long)rank * warps + warp) * S;
    auto fetch = [&](long long t) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const long long at = t - s;
            if (on && at >= 0 && at < end) {
                gn[s] = scan_load<G, V>(gate + at * p.gate_at.token);
                if (with_x) xn[s] = scan_load<T, V>(x + at * p.x_at.token);
                if (with_dh) dn[s] = scan_load<T, V>(dh + at * p.dh_at.token);
                if (at > 0) hn[s] = scan_load<T, V>(hin + (at - 1) * p.h_in_at.token);
            }
        }
        mark = reset && lane < S && t - lane >= 0 && t - lane < end ? reset[(t - lane) * p.reset_at.token] : 0;
    };
    fetch(t0);
    int parity = 0;
    for (long long first = 0; first < p.tokens; first += round, t0 -= round, parity ^= 1) {
        const unsigned drops = __ballot_sync(0xffffffffu, mark != 0);
        ScanPiece<T, V> xs[S], ds[S], hs[S];
        ScanPiece<G, V> gs[S];
#pragma unroll
        for (int s = 0; s < S; ++s) xs[s] = xn[s], ds[s] = dn[s], hs[s] = hn[s], gs[s] = gn[s];
        fetch(t0 - round);
        A through[V], u[V], in[V];
#pragma unroll
        for (int v = 0; v < V; ++v) through[v] = A(1), u[v] = A(0);
        with_mode(p.mode, [&](auto decay, auto) {
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    A a, rest;
                    scan_decay<decay.value, EXACT>((A)widen(gs[s].v[v]), a, rest);
                    const bool live = on && t0 - s >= 0 && t0 - s < end;
                    const A l = (with_dh ? widen(ds[s].v[v]) : A(0)) + u[v];
                    if (live) u[v] = (drops >> s) & 1u ? A(0) : a * l, through[v] *= a;
                }
        });
        scan_join(sh, parity, rank, cluster, through, u, drops != 0, carry, in);
        with_mode(p.mode, [&](auto decay, auto mix) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                ScanPiece<T, V> to_x;
                ScanPiece<G, V> to_g;
                const bool live = on && t0 - s >= 0 && t0 - s < end, drop = (drops >> s) & 1u;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    A a, rest, da, dm;
                    scan_decay<decay.value, EXACT>((A)widen(gs[s].v[v]), a, rest);
                    const A m = scan_mix<mix.value, EXACT>(a, rest);
                    scan_slopes<decay.value, mix.value, EXACT>(a, rest, m, da, dm);
                    const A l = (with_dh ? widen(ds[s].v[v]) : A(0)) + in[v];
                    const A before = t0 - s > 0 ? widen(hs[s].v[v]) : start[v];
                    A slope = drop ? A(0) : da * before;
                    if (mix.value != FO_MIX_ONE) slope = fused_ma(dm, widen(xs[s].v[v]), slope);
                    to_x.v[v] = narrow<T>(live ? m * l : A(0));
                    to_g.v[v] = narrow<G>(live ? l * slope : A(0));
                    if (live) in[v] = drop ? A(0) : a * l;
                }
                if (on && t0 - s >= 0) {
                    scan_store<T, V>(dx + (t0 - s) * p.h_at.token, to_x);
                    scan_store<G, V>(dgate + (t0 - s) * p.dgate_at.token, to_g);
                }
            }
        });
    }
    if (p.last && on && rank == 0 && warp == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) static_cast<A *>(p.last)[b * p.channels + c + v] = carry[v];
}

// Host: one kernel of a pair of types; scan_*.cu instantiate it.
template <class T, class G>
cudaError_t launch_scan(const ScanParams &p, bool wide, bool grad, long long batch, cudaStream_t st);

}  // namespace fo
