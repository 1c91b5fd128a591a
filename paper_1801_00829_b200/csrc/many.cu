// Operators over many tensors in one launch: the global gradient norm, clipping by it, and AdamW.
//
// The tensors' addresses and sizes travel as kernel parameters (no device table, nothing kept between
// calls); a longer list takes several launches.  All tensors together are one line of tiles, of which each
// CTA takes every gridDim-th: at any time the GPU works on one stretch of every stream, not on
// one per CTA and stream.  Tiles begin where pieces are aligned; the elements of a tensor before the first
// piece and after the last are handled singly.  What is written decides the pieces' alignment; what is read at
// another one is put together from aligned 16 bytes.
#include <math.h>

#include "elem.cuh"

namespace fo {
namespace {

constexpr int kCta = 256;
// A tile is 1 to 4 times kTile elements: small enough that a short list still fills the SMs, large enough that
// finding a tile's tensor and addresses costs a long list little (AdamW over 25M, 50M and 130M parameters in up to 72
// tensors: 119, 235 and 614 us with twice kTile, 122, 233 and 606 with 4 times, 124, 243 and 605 with 8 times).
constexpr int kTile = 2048, kMostTile = 4 * kTile;

// ------------------------------------------------------------------- lists
template <int N>
struct NormList {
    int count;
    unsigned tiles;
    int tile;                                // elements of one
    unsigned first[N + 1];                   // first tile of each tensor
    const void *in[N];
    long long n[N];
};
template <int N>
struct ClipList {
    int count;
    unsigned tiles;
    int tile;                                // elements of one
    unsigned first[N + 1];
    const void *in[N];
    void *out[N];
    long long n[N];
};
template <int N>
struct AdamList {
    int count;
    unsigned tiles;
    int tile;                                // elements of one
    unsigned first[N + 1];
    const void *p[N], *g[N], *m[N], *v[N];
    void *p_out[N], *m_out[N], *v_out[N], *weights[N];
    long long n[N];
    double decay[N];
};

// The tensor that holds tile `t`: the last one whose first tile is not behind it (tensors without
// elements have no tile and are never found).
template <class List>
__device__ __forceinline__ int tensor_of(const List &l, unsigned t)
{
    int lo = 0, hi = l.count;                // first[lo] <= t < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A tile of a tensor: `pieces` aligned pieces of V elements from element `at`, `head` single ones from the
// tensor's beginning (its first tile) and `tail` behind the pieces (its last).  The host counts tiles without
// the head, so a last tile may be empty.
struct Cut {
    long long at;
    int pieces, head, tail;
    __device__ __forceinline__ long long single(int i, int v) const      // element of single number i, -1: none
    {
        return i < head ? i : i - head < tail ? at + (long long)pieces * v + (i - head) : -1;
    }
};
template <int V>
__device__ __forceinline__ Cut cut_tile(const void *p, int bytes, long long n, unsigned tile, int size)
{
    const int mis = (int)(((uintptr_t)p / bytes) & (V - 1));
    const long long lead = min((long long)((V - mis) & (V - 1)), n);
    Cut c;
    c.at = lead + (long long)tile * size;
    const long long left = n - c.at;
    const int len = left < size ? (left > 0 ? (int)left : 0) : size;
    c.pieces = len / V;
    c.head = tile == 0 ? (int)lead : 0;
    c.tail = len - c.pieces * V;
    return c;
}

// -------------------------------------------------------------------- norm
struct NormOut {
    double *partial;                         // one per CTA
    double *carry;                           // what the launches of earlier parts of the list found
    WsHead *head;
    void *result;                            // NULL: not the last part
    int result_type, first_part;
    double max_norm, eps;
};

// |g| as an unsigned number: ordered as the values are, NaN above infinity.
__device__ __forceinline__ unsigned long long magnitude(double v)
{
    return (unsigned long long)__double_as_longlong(v) & 0x7fffffffffffffffULL;
}
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ double larger(double a, double b)     // of two magnitudes, NaN before all
{
    return magnitude(a) > magnitude(b) ? a : b;
}

// The norm reads 520 MB of bf16 in 86 us, 6.0 TB/s: DRAM.
// Sum of squares of N values.  In 32 bits, and again in 64 where the 32-bit sum is so small or so
// large that squares may have left the normal range: below 2^-60 what underflowed (each square under
// 2^-126) could show, above 2^100 an overflow is near.
template <class T, int N>
__device__ __forceinline__ double sum_squares(const Packed<T, N> &r)
{
    if constexpr (sizeof(T) < 8) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) s = fmaf(r.get(k), r.get(k), s);
        if (s >= 0x1p-60f && s <= 0x1p100f) return (double)s;
    }
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) d = fma((double)r.get(k), (double)r.get(k), d);
    return d;
}
template <class T, int N>
__device__ __forceinline__ double max_magnitude(const Packed<T, N> &r)
{
    Acc<T> best = Acc<T>(0);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const Acc<T> g = r.get(k);
        if (magnitude(g) > magnitude(best)) best = g;
    }
    return fabs((double)best);
}

template <int KIND>
__device__ __forceinline__ double join(double a, double b)
{
    return KIND == FO_NORM_L2 ? a + b : larger(a, b);
}
template <int KIND>
__device__ __forceinline__ double cta_join(double v, double *smem)     // result in thread 0
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = join<KIND>(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kCta / 32; ++w) v = join<KIND>(v, smem[w]);
    return v;
}

constexpr int kNormPerSm = 5;                // CTAs, of 51 registers a thread: four 16-byte pieces and their sums

template <class T, int N, int KIND>
__global__ void __launch_bounds__(kCta, sizeof(T) == 8 ? 4 : kNormPerSm)
grad_norm_kernel(const __grid_constant__ NormList<N> l, const NormOut o)
{
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int kBatch = 4;                // pieces of a thread in flight
    __shared__ double smem[kCta / 32];
    __shared__ unsigned s_flag;
    double acc = 0.0;
    for (unsigned t = blockIdx.x; t < l.tiles; t += gridDim.x) {
        const int k = tensor_of(l, t);
        const T *p = static_cast<const T *>(l.in[k]);
        const Cut c = cut_tile<V>(p, sizeof(T), l.n[k], t - l.first[k], l.tile);
        const long long e = c.single(threadIdx.x, V);
        const double g = e >= 0 ? (double)widen<T>(p[e]) : 0.0;
        for (int i0 = threadIdx.x; i0 < c.pieces; i0 += kBatch * kCta) {
            Packed<T, V * kBatch> r;
            r.clear();
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
                if (i0 + b * kCta < c.pieces) load16(r.w + 4 * b, p + c.at + (i0 + b * kCta) * V);
            acc = join<KIND>(acc, KIND == FO_NORM_L2 ? sum_squares<T>(r) : max_magnitude<T>(r));
        }
        if (e >= 0) acc = join<KIND>(acc, KIND == FO_NORM_L2 ? g * g : fabs(g));
    }
    let_later_start();                                       // its CTAs wait for this kernel's end
    acc = cta_join<KIND>(acc, smem);
    if (threadIdx.x == 0) o.partial[blockIdx.x] = acc;
    if (!publish_and_is_last(o.head, &s_flag)) return;
    acc = 0.0;
    for (int g = threadIdx.x; g < (int)gridDim.x; g += kCta) acc = join<KIND>(acc, __ldcg(o.partial + g));
    __syncthreads();
    acc = cta_join<KIND>(acc, smem);
    if (threadIdx.x != 0) return;
    if (!o.first_part) acc = join<KIND>(acc, *o.carry);
    if (!o.result) {
        *o.carry = acc;
        return;
    }
    const double norm = KIND == FO_NORM_L2 ? sqrt(acc) : acc;
    const double q = o.max_norm / (norm + o.eps), factor = q >= 1.0 ? 1.0 : q;      // NaN stays
    if (o.result_type == FO_F64) {
        static_cast<double *>(o.result)[0] = norm;
        static_cast<double *>(o.result)[1] = factor;
    } else {
        static_cast<float *>(o.result)[0] = (float)norm;
        static_cast<float *>(o.result)[1] = (float)factor;
    }
}

// -------------------------------------------------------------------- clip
// V elements, 16 or 32 bytes, of a tensor that lies in [begin, end): at once where they are `aligned` to their size, else
// put together from aligned 16 bytes.
template <class T, int V>
__device__ __forceinline__ void load_some(Packed<T, V> &r, const T *p, bool aligned, const T *begin, const T *end)
{
    constexpr int kStep = 16 / (int)sizeof(T);
    if (aligned) {
        if constexpr (V == 2 * kStep) load32(r.w, p);
        else load16(r.w, p);
    } else {
#pragma unroll
        for (int k = 0; k < V; k += kStep) load16_any<false>(r.w + k * (int)sizeof(T) / 4, p + k, begin, end);
    }
}
template <class T, int V>
__device__ __forceinline__ void store_some(T *p, const Acc<T> (&v)[V], bool aligned)
{
    constexpr int kStep = 16 / (int)sizeof(T);
    if (aligned) {
        Packed<T, V> r;
#pragma unroll
        for (int k = 0; k < V; k += 2) r.put2(k, two(v[k], v[k + 1]));
        if constexpr (V == 2 * kStep) store32(p, r.w);
        else store16(p, r.w);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] = narrow<T>(v[k]);
    }
}
template <int V, class T>
__device__ __forceinline__ bool aligned_for(const T *p)
{
    return ((uintptr_t)p & (V * sizeof(T) - 1)) == 0;
}

__device__ __forceinline__ double read_factor(const void *factor, int type)
{
    return type == FO_F64 ? *static_cast<const double *>(factor) : (double)*static_cast<const float *>(factor);
}

// The tiles in the opposite order of the norm's: what it read last is still in L2.
constexpr int kClipPerSm = 7;                // CTAs (260M bf16, with the norm: 349 us; 8 of them 357; 5 with 4 pieces each 376)

template <class TI, class TO, int N>
__global__ void __launch_bounds__(kCta, sizeof(TI) == 8 ? 4 : kClipPerSm)
clip_kernel(const __grid_constant__ ClipList<N> l, const void *result, int result_type)
{
    using A = Acc<TI>;
    constexpr int V = 16 / (int)sizeof(TI);
    constexpr int kBatch = 2;                // pieces of a thread in flight
    A factor = A(0);
    bool known = false;
    for (unsigned u = blockIdx.x; u < l.tiles; u += gridDim.x) {
        const unsigned t = l.tiles - 1u - u;
        const int k = tensor_of(l, t);
        const TI *begin = static_cast<const TI *>(l.in[k]);
        const long long n = l.n[k];
        TO *out = static_cast<TO *>(l.out[k]);
        const Cut c = cut_tile<V>(out, sizeof(TO), n, t - l.first[k], l.tile);
        const TI *p = begin + c.at;
        TO *q = out + c.at;
        const bool in_ok = aligned_for<V>(p);
        const long long e = c.single(threadIdx.x, V);
        const A one = e >= 0 ? widen<TI>(begin[e]) : A(0);
        bool keep = false;                                   // in place, and nothing to clip
        for (int i0 = 0; i0 == 0 || i0 < c.pieces; i0 += kBatch * kCta) {
            Packed<TI, V> g[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int i = i0 + threadIdx.x + b * kCta;
                if (i < c.pieces) load_some<TI, V>(g[b], p + i * V, in_ok, begin, begin + n);
            }
            if (!known) {                                    // the first elements were on their way meanwhile
                wait_for_earlier();
                factor = (A)(result_type == FO_F64 ? static_cast<const double *>(result)[1]
                                                   : (double)static_cast<const float *>(result)[1]);
                known = true;
            }
            keep = (const void *)begin == (const void *)out && factor == A(1);
            if (keep) break;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int i = i0 + threadIdx.x + b * kCta;
                if (i >= c.pieces) continue;
                A v[V];
#pragma unroll
                for (int x = 0; x < V; ++x) v[x] = g[b].get(x) * factor;
                store_some<TO, V>(q + i * V, v, true);
            }
        }
        if (e >= 0 && !keep) out[e] = narrow<TO>(one * factor);
    }
}

// ------------------------------------------------------------------- adamw
struct AdamHyper {
    double lr, beta1, beta2, eps, fix1, fix2;          // fix: 1 / (1 - beta^step)
    const void *factor;
    int factor_type;
};

template <class A>
__device__ __forceinline__ void adam_one(A &p, A g, A &m, A &v, A c, A b1, A b2, A u1, A u2, A fix1, A fix2, A eps,
                                         A lr, A decay)
{
    g *= c;
    m = fused_ma(m, b1, g * u1);
    v = fused_ma(v, b2, g * g * u2);
    const A step = (m * fix1) / (sqrt(v * fix2) + eps);
    p = p - lr * fused_ma(decay, p, step);
}

// Pieces of 8 elements (2 of float64), 32 bytes of each 32-bit tensor.  CTAs per SM: where everything is aligned, two keep
// enough in flight (57 KB), and more make the memory serve reads and writes of seven streams in more and smaller
// turns (100M parameters in one tensor: 436 us, with three 475); misaligned gradients need three (130M in 72 tensors
// behind each other: 606 us, with two 691), and lists that are soon through four (3M: 19 us, with three 21).
constexpr long long kAdamLong = 8 << 20;

template <class TG, class TW, int N>
__global__ void __launch_bounds__(kCta) adamw_kernel(const __grid_constant__ AdamList<N> l, const AdamHyper h)
{
    using A = Acc<TG>;
    constexpr int V = sizeof(A) == 8 ? 2 : 8;
    const A c = h.factor ? (A)read_factor(h.factor, h.factor_type) : A(1);
    const A b1 = (A)h.beta1, b2 = (A)h.beta2, u1 = (A)(1.0 - h.beta1), u2 = (A)(1.0 - h.beta2);
    const A fix1 = (A)h.fix1, fix2 = (A)h.fix2, eps = (A)h.eps, lr = (A)h.lr;
    for (unsigned t = blockIdx.x; t < l.tiles; t += gridDim.x) {
        const int k = tensor_of(l, t);
        const long long n = l.n[k];
        const A *p = static_cast<const A *>(l.p[k]), *m = static_cast<const A *>(l.m[k]), *v = static_cast<const A *>(l.v[k]);
        const TG *g = static_cast<const TG *>(l.g[k]);
        A *po = static_cast<A *>(l.p_out[k]), *mo = static_cast<A *>(l.m_out[k]), *vo = static_cast<A *>(l.v_out[k]);
        TW *wo = static_cast<TW *>(l.weights[k]);
        const A decay = (A)l.decay[k];
        const Cut cut = cut_tile<V>(po, sizeof(A), n, t - l.first[k], l.tile);
        const long long d = cut.at;
        const bool p_ok = aligned_for<V>(p + d), g_ok = aligned_for<V>(g + d), m_ok = aligned_for<V>(m + d),
                   v_ok = aligned_for<V>(v + d), mo_ok = aligned_for<V>(mo + d), vo_ok = aligned_for<V>(vo + d),
                   wo_ok = aligned_for<V>(wo + d);
#pragma unroll 1
        for (int i = threadIdx.x; i < cut.pieces; i += kCta) {
            const long long e0 = d + i * V;
            Packed<A, V> qp, qm, qv;
            Packed<TG, V> qg;
            load_some<A, V>(qp, p + e0, p_ok, p, p + n);
            load_some<TG, V>(qg, g + e0, g_ok, g, g + n);
            load_some<A, V>(qm, m + e0, m_ok, m, m + n);
            load_some<A, V>(qv, v + e0, v_ok, v, v + n);
            A rp[V], rm[V], rv[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                rp[e] = qp.get(e), rm[e] = qm.get(e), rv[e] = qv.get(e);
                adam_one<A>(rp[e], qg.get(e), rm[e], rv[e], c, b1, b2, u1, u2, fix1, fix2, eps, lr, decay);
            }
            store_some<A, V>(po + e0, rp, true);
            store_some<A, V>(mo + e0, rm, mo_ok);
            store_some<A, V>(vo + e0, rv, vo_ok);
            if constexpr (sizeof(TW) == 2) {
                if (wo) store_some<TW, V>(wo + e0, rp, wo_ok);
            }
        }
        const long long e = cut.single(threadIdx.x, V);
        if (e >= 0) {
            A rp = p[e], rm = m[e], rv = v[e];
            adam_one<A>(rp, widen<TG>(g[e]), rm, rv, c, b1, b2, u1, u2, fix1, fix2, eps, lr, decay);
            po[e] = rp, mo[e] = rm, vo[e] = rv;
            if constexpr (sizeof(TW) == 2) {
                if (wo) wo[e] = narrow<TW>(rp);
            }
        }
    }
}

// -------------------------------------------------------------------- host
constexpr int kFew = 40, kMany = 512, kManyAdam = 256;      // tensors of one launch: the parameters fit 32 KB

unsigned tiles_of(long long n, int tile) { return (unsigned)((n + tile - 1) / tile); }

// Tile size of a part of a list: about `per_cta` tiles for each of `per_sm` CTAs on every SM.
template <class Tensor>
int tile_for(const Tensor *t, int count, int per_sm, int per_cta)
{
    long long total = 0;
    for (int k = 0; k < count; ++k) total += t[k].n;
    const long long each = total / ((long long)sm_count() * per_sm * per_cta + 1) / kTile + 1;
    return (int)(each * kTile < kMostTile ? each * kTile : kMostTile);
}
unsigned grid_for(unsigned tiles, int per_sm)
{
    const unsigned cap = (unsigned)(sm_count() * per_sm);
    return tiles < cap ? (tiles ? tiles : 1u) : cap;
}

bool float_type(int t) { return t >= FO_F64 && t <= FO_F16; }

// Sizes and addresses of a list; the tiles of all its tensors have to fit 31 bits (4e12 elements).
template <class Tensor, class Bad>
int check_list(const Tensor *t, int count, Bad bad)
{
    if (count < 0) return FO_ERR_SHAPE;
    if (count > 0 && !t) return FO_ERR_NULL;
    unsigned long long tiles = 0;
    for (int k = 0; k < count; ++k) {
        if (t[k].n < 0) return FO_ERR_SHAPE;
        if (t[k].n > 0 && bad(t[k])) return FO_ERR_NULL;
        tiles += (unsigned long long)(t[k].n / kTile + 1);
    }
    return tiles < (1ULL << 31) ? FO_OK : FO_ERR_UNSUPPORTED;
}

// The pointers of a list are to elements of their types.
template <class Tensor, class Good>
int check_elements(const Tensor *t, int count, Good good)
{
    for (int k = 0; k < count; ++k)
        if (t[k].n > 0 && !good(t[k])) return FO_ERR_UNSUPPORTED;
    return FO_OK;
}

template <class T, int N>
cudaError_t launch_norm_part(const fo_tensor *t, int count, int kind, const NormOut &o, cudaStream_t st)
{
    constexpr int kPerSm = kNormPerSm;
    NormList<N> l;
    l.count = count, l.tiles = 0, l.tile = tile_for(t, count, kPerSm, 4);
    for (int k = 0; k < count; ++k) {
        l.first[k] = l.tiles, l.in[k] = t[k].in, l.n[k] = t[k].n;
        l.tiles += tiles_of(t[k].n, l.tile);
    }
    l.first[count] = l.tiles;
    const unsigned grid = grid_for(l.tiles, kPerSm);
    if (kind == FO_NORM_L2) grad_norm_kernel<T, N, FO_NORM_L2><<<grid, kCta, 0, st>>>(l, o);
    else grad_norm_kernel<T, N, FO_NORM_MAX><<<grid, kCta, 0, st>>>(l, o);
    return cudaGetLastError();
}

template <class T>
cudaError_t launch_norm(const fo_tensor *t, int count, int kind, NormOut o, cudaStream_t st)
{
    void *const result = o.result;
    int at = 0;
    do {
        const int part = count - at < kMany ? count - at : kMany;
        o.first_part = at == 0;
        o.result = at + part == count ? result : nullptr;
        const cudaError_t e = part <= kFew ? launch_norm_part<T, kFew>(t + at, part, kind, o, st)
                                           : launch_norm_part<T, kMany>(t + at, part, kind, o, st);
        if (e != cudaSuccess) return e;
        at += part;
    } while (at < count);
    return cudaSuccess;
}

template <class TI, class TO, int N>
cudaError_t launch_clip_part(const fo_tensor *t, int count, const void *result, int result_type, cudaStream_t st)
{
    constexpr int kPerSm = kClipPerSm;
    ClipList<N> l;
    l.count = count, l.tiles = 0, l.tile = tile_for(t, count, kPerSm, 4);
    for (int k = 0; k < count; ++k) {
        l.first[k] = l.tiles, l.in[k] = t[k].in, l.out[k] = t[k].out, l.n[k] = t[k].n;
        l.tiles += tiles_of(t[k].n, l.tile);
    }
    l.first[count] = l.tiles;
    if (l.tiles == 0) return cudaSuccess;
    return launch_beside(clip_kernel<TI, TO, N>, dim3(grid_for(l.tiles, kPerSm)), kCta, st, l, result, result_type);
}

template <class TI, class TO>
cudaError_t launch_clip(const fo_tensor *t, int count, const void *result, int result_type, cudaStream_t st)
{
    for (int at = 0; at < count; at += kMany) {
        const int part = count - at < kMany ? count - at : kMany;
        const cudaError_t e = part <= kFew ? launch_clip_part<TI, TO, kFew>(t + at, part, result, result_type, st)
                                           : launch_clip_part<TI, TO, kMany>(t + at, part, result, result_type, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <class TG, class TW, int N>
cudaError_t launch_adam_part(const fo_adam_tensor *t, int count, const AdamHyper &h, cudaStream_t st)
{
    long long total = 0;
    bool aligned = true;
    for (int k = 0; k < count; ++k) {
        total += t[k].n;
        for (const void *q : {t[k].p, t[k].g, t[k].m, t[k].v, (const void *)t[k].p_out, (const void *)t[k].m_out,
                              (const void *)t[k].v_out, (const void *)t[k].weights})
            aligned = aligned && ((uintptr_t)q & 31u) == 0;
    }
    const int per_sm = total < kAdamLong ? 4 : aligned ? 2 : 3;
    AdamList<N> l;
    l.count = count, l.tiles = 0, l.tile = tile_for(t, count, per_sm, 4);
    for (int k = 0; k < count; ++k) {
        l.first[k] = l.tiles;
        l.p[k] = t[k].p, l.g[k] = t[k].g, l.m[k] = t[k].m, l.v[k] = t[k].v;
        l.p_out[k] = t[k].p_out, l.m_out[k] = t[k].m_out, l.v_out[k] = t[k].v_out, l.weights[k] = t[k].weights;
        l.n[k] = t[k].n, l.decay[k] = t[k].decay;
        l.tiles += tiles_of(t[k].n, l.tile);
    }
    l.first[count] = l.tiles;
    if (l.tiles == 0) return cudaSuccess;
    adamw_kernel<TG, TW, N><<<grid_for(l.tiles, per_sm), kCta, 0, st>>>(l, h);
    return cudaGetLastError();
}

template <class TG, class TW>
cudaError_t launch_adam(const fo_adam_tensor *t, int count, const AdamHyper &h, cudaStream_t st)
{
    for (int at = 0; at < count; at += kManyAdam) {
        const int part = count - at < kManyAdam ? count - at : kManyAdam;
        const cudaError_t e = part <= kFew ? launch_adam_part<TG, TW, kFew>(t + at, part, h, st)
                                           : launch_adam_part<TG, TW, kManyAdam>(t + at, part, h, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

int run_norm(const fo_tensor *t, int count, int in_type, int kind, double max_norm, double eps, void *result,
             int result_type, void *ws, size_t ws_bytes, cudaStream_t st)
{
    if (!float_type(in_type) || (kind != FO_NORM_L2 && kind != FO_NORM_MAX)
        || (result_type != FO_F32 && result_type != FO_F64))
        return FO_ERR_UNSUPPORTED;
    if (!(max_norm >= 0.0) || !(eps >= 0.0)) return FO_ERR_SHAPE;
    if (!result) return FO_ERR_NULL;
    if (!on_elements(result, result_type)) return FO_ERR_UNSUPPORTED;
    int rc = check_elements(t, count, [=](const fo_tensor &x) { return on_elements(x.in, in_type); });
    if (rc == FO_OK) rc = check_workspace(ws, ws_bytes, fused_grad_workspace_bytes());
    if (rc != FO_OK) return rc;
    NormOut o = {};
    o.head = static_cast<WsHead *>(ws);
    o.carry = reinterpret_cast<double *>(o.head + 1);
    o.partial = o.carry + 1;
    o.result = result, o.result_type = result_type;
    o.max_norm = max_norm, o.eps = eps;
    const cudaError_t e = in_type == FO_F64   ? launch_norm<double>(t, count, kind, o, st)
                          : in_type == FO_F32 ? launch_norm<float>(t, count, kind, o, st)
                          : in_type == FO_BF16 ? launch_norm<__nv_bfloat16>(t, count, kind, o, st)
                                               : launch_norm<__half>(t, count, kind, o, st);
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

size_t fused_grad_workspace_bytes(void) { return sizeof(WsHead) + (size_t)(1 + kMaxPartials) * sizeof(double); }

int fused_grad_norm(const fo_tensor *t, int count, int in_type, int norm_kind, double max_norm, double eps,
                    void *result, int result_type, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_list(t, count, [](const fo_tensor &x) { return !x.in; });
    if (rc != FO_OK) return rc;
    return run_norm(t, count, in_type, norm_kind, max_norm, eps, result, result_type, ws, ws_bytes,
                    (cudaStream_t)stream);
}

int fused_grad_clip(const fo_tensor *t, int count, int in_type, int out_type, int norm_kind, double max_norm,
                    double eps, void *result, int result_type, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_list(t, count, [](const fo_tensor &x) { return !x.in || !x.out; });
    if (rc != FO_OK) return rc;
    if (!float_type(out_type) || (out_type != in_type && !(out_type == FO_F32 && (in_type == FO_BF16 || in_type == FO_F16))))
        return FO_ERR_UNSUPPORTED;
    rc = check_elements(t, count, [=](const fo_tensor &x) { return on_elements(x.out, out_type); });
    if (rc != FO_OK) return rc;
    const cudaStream_t st = (cudaStream_t)stream;
    rc = run_norm(t, count, in_type, norm_kind, max_norm, eps, result, result_type, ws, ws_bytes, st);
    if (rc != FO_OK) return rc;
    cudaError_t e = cudaErrorInvalidValue;
    if (in_type == FO_F64) e = launch_clip<double, double>(t, count, result, result_type, st);
    else if (in_type == FO_F32) e = launch_clip<float, float>(t, count, result, result_type, st);
    else if (in_type == FO_BF16 && out_type == FO_F32) e = launch_clip<__nv_bfloat16, float>(t, count, result, result_type, st);
    else if (in_type == FO_BF16) e = launch_clip<__nv_bfloat16, __nv_bfloat16>(t, count, result, result_type, st);
    else if (out_type == FO_F32) e = launch_clip<__half, float>(t, count, result, result_type, st);
    else e = launch_clip<__half, __half>(t, count, result, result_type, st);
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

int fused_adamw(const fo_adam_tensor *t, int count, int grad_type, int weight_type, double lr, double beta1,
                double beta2, double eps, int64_t step, const void *factor, int factor_type, void *stream)
{
    bool any_weights = false;
    int rc = check_list(t, count, [&](const fo_adam_tensor &x) {
        any_weights = any_weights || x.weights;
        return !x.p || !x.g || !x.m || !x.v || !x.p_out || !x.m_out || !x.v_out;
    });
    if (rc != FO_OK) return rc;
    if (!float_type(grad_type) || (factor && factor_type != FO_F32 && factor_type != FO_F64)) return FO_ERR_UNSUPPORTED;
    if (any_weights && weight_type != FO_BF16 && weight_type != FO_F16) return FO_ERR_UNSUPPORTED;
    if (any_weights && grad_type == FO_F64) return FO_ERR_UNSUPPORTED;
    if (step < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0)) return FO_ERR_SHAPE;
    const int wide = grad_type == FO_F64 ? FO_F64 : FO_F32;
    rc = check_elements(t, count, [=](const fo_adam_tensor &x) {
        for (const void *p : {x.p, x.m, x.v, (const void *)x.p_out, (const void *)x.m_out, (const void *)x.v_out})
            if (!on_elements(p, wide)) return false;
        return on_elements(x.g, grad_type) && on_elements(x.weights, weight_type);
    });
    if (rc != FO_OK || (factor && !on_elements(factor, factor_type))) return FO_ERR_UNSUPPORTED;
    AdamHyper h = {lr, beta1, beta2, eps, 1.0 / (1.0 - pow(beta1, (double)step)), 1.0 / (1.0 - pow(beta2, (double)step)),
                   factor, factor_type};
    const cudaStream_t st = (cudaStream_t)stream;
    const bool half = any_weights && weight_type == FO_F16;
    cudaError_t e;
    if (grad_type == FO_F64) e = launch_adam<double, double>(t, count, h, st);
    else if (grad_type == FO_F32) e = half ? launch_adam<float, __half>(t, count, h, st)
                                           : launch_adam<float, __nv_bfloat16>(t, count, h, st);
    else if (grad_type == FO_BF16) e = half ? launch_adam<__nv_bfloat16, __half>(t, count, h, st)
                                            : launch_adam<__nv_bfloat16, __nv_bfloat16>(t, count, h, st);
    else e = half ? launch_adam<__half, __half>(t, count, h, st) : launch_adam<__half, __nv_bfloat16>(t, count, h, st);
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

}  // extern "C"
