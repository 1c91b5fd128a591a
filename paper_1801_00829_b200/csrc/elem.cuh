// Element types of the training-step operators (float64, float32, bfloat16, float16): rows held
// packed in registers as they lie in memory, conversion to the type sums are held in, and the
// gate's activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"
#include "../../include/fusedops_train.h"

namespace fo {

// Host: bytes of an element type, and whether a pointer may point to such elements.
inline int elem_bytes(int type) { return type == FO_F64 ? 8 : type == FO_F32 ? 4 : 2; }
inline bool on_elements(const void *p, int type) { return ((uintptr_t)p & (uintptr_t)(elem_bytes(type) - 1)) == 0; }

// Acc: what arithmetic, statistics and sums are held in.
template <class T> struct Elem { using Acc = float; };
template <> struct Elem<double> { using Acc = double; };
template <class T> using Acc = typename Elem<T>::Acc;

template <class T>
__device__ __forceinline__ Acc<T> widen(T v)
{
    return (Acc<T>)v;
}
template <class T>
__device__ __forceinline__ T narrow(Acc<T> v);
template <> __device__ __forceinline__ double narrow<double>(double v) { return v; }
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ float fused_ma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double fused_ma(double a, double b, double c) { return fma(a, b, c); }

// Two neighbouring elements' values.  In 32 bits they are one 64-bit register pair, which the
// packed instructions of sm_100 multiply and add with one issue slot.
template <class A>
struct Two {
    A a, b;
};
template <>
struct Two<float> {
    unsigned long long v;
};
__device__ __forceinline__ Two<float> two(float a, float b)
{
    Two<float> t;
    asm("mov.b64 %0, {%1, %2};" : "=l"(t.v) : "f"(a), "f"(b));
    return t;
}
__device__ __forceinline__ Two<double> two(double a, double b) { return {a, b}; }
__device__ __forceinline__ float first(Two<float> t) { return __uint_as_float((unsigned)t.v); }
__device__ __forceinline__ float second(Two<float> t) { return __uint_as_float((unsigned)(t.v >> 32)); }
__device__ __forceinline__ double first(Two<double> t) { return t.a; }
__device__ __forceinline__ double second(Two<double> t) { return t.b; }
__device__ __forceinline__ Two<float> operator*(Two<float> x, Two<float> y)
{
    Two<float> t;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(t.v) : "l"(x.v), "l"(y.v));
    return t;
}
__device__ __forceinline__ Two<float> operator+(Two<float> x, Two<float> y)
{
    Two<float> t;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(t.v) : "l"(x.v), "l"(y.v));
    return t;
}
__device__ __forceinline__ Two<float> fused_ma(Two<float> x, Two<float> y, Two<float> z)
{
    Two<float> t;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(t.v) : "l"(x.v), "l"(y.v), "l"(z.v));
    return t;
}
__device__ __forceinline__ Two<double> operator*(Two<double> x, Two<double> y) { return {x.a * y.a, x.b * y.b}; }
__device__ __forceinline__ Two<double> operator+(Two<double> x, Two<double> y) { return {x.a + y.a, x.b + y.b}; }
__device__ __forceinline__ Two<double> fused_ma(Two<double> x, Two<double> y, Two<double> z)
{
    return {fma(x.a, y.a, z.a), fma(x.b, y.b, z.b)};
}
template <class A>
__device__ __forceinline__ Two<A> both(A v)
{
    return two(v, v);
}
template <class A>
__device__ __forceinline__ A joined(Two<A> t)
{
    return first(t) + second(t);
}

// N elements as 32-bit words, the way they lie in memory.  N * sizeof(T) is a multiple of 16.
template <class T, int N>
struct Packed {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];

    __device__ __forceinline__ Acc<T> get(int k) const
    {
        if constexpr (sizeof(T) == 8) return __hiloint2double((int)w[2 * k + 1], (int)w[2 * k]);
        else if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value)
            return __uint_as_float((k & 1) ? (w[k / 2] & 0xffff0000u) : (w[k / 2] << 16));
        else return __half2float(__ushort_as_half((unsigned short)((k & 1) ? (w[k / 2] >> 16) : (w[k / 2] & 0xffffu))));
    }
    __device__ __forceinline__ void put2(int k, Two<Acc<T>> v)      // k even; rounded once
    {
        const Acc<T> a = first(v), b = second(v);
        if constexpr (sizeof(T) >= 4) {
            put(k, (T)a);
            put(k + 1, (T)b);
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
            memcpy(&w[k / 2], &v, 4);
        } else {
            const __half2 v = __floats2half2_rn(a, b);
            memcpy(&w[k / 2], &v, 4);
        }
    }
    __device__ __forceinline__ Two<Acc<T>> get2(int k) const { return two(get(k), get(k + 1)); }      // k even
    __device__ __forceinline__ T raw(int k) const                     // as it lies in memory
    {
        if constexpr (sizeof(T) >= 4) return (T)get(k);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value)
            return __ushort_as_bfloat16((unsigned short)(w[k / 2] >> (16 * (k & 1))));
        else return __ushort_as_half((unsigned short)(w[k / 2] >> (16 * (k & 1))));
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void put(int k, T v)      // into a cleared place
    {
        if constexpr (sizeof(T) == 8) {
            w[2 * k] = (uint32_t)__double2loint(v);
            w[2 * k + 1] = (uint32_t)__double2hiint(v);
        } else if constexpr (sizeof(T) == 4) {
            w[k] = __float_as_uint(v);
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            w[k / 2] |= (uint32_t)__bfloat16_as_ushort(v) << (16 * (k & 1));
        } else {
            w[k / 2] |= (uint32_t)__half_as_ushort(v) << (16 * (k & 1));
        }
    }
};

// 16 bytes of data that is read once: no place in L1.  Not the read-only path: an output may be the
// matrix it is computed from, element by element.
__device__ __forceinline__ void load16(uint32_t *w, const void *p)
{
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "l"(p));
}
// 32 bytes at once, from a 32-byte boundary: a warp's access then covers whole sectors, where two of 16 bytes would
// touch every sector twice.
__device__ __forceinline__ void load32(uint32_t *w, const void *p)
{
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}
__device__ __forceinline__ void store32(void *p, const uint32_t *w)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
__device__ __forceinline__ void store16(void *p, const uint32_t *w)
{
    asm volatile("st.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                 : "memory");
}

// 16 bytes from byte `q` (0 .. 15, a multiple of the element's SIZE) of 32.
template <int SIZE>
__device__ __forceinline__ void straddle(uint32_t *r, const uint32_t (&w)[8], unsigned q)
{
    uint32_t a[7], b[5];
#pragma unroll
    for (int i = 0; i < 7; ++i) a[i] = SIZE < 8 && (q & 4u) ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) b[i] = (q & 8u) ? a[i + 2] : a[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = SIZE < 4 ? __funnelshift_r(b[i], b[i + 1], (q & 3u) * 8u) : b[i];
}

// 16 bytes from any address, through L1 (the next thread reads the second half too).  Nothing outside
// [begin, end), the matrix's or tensor's own bytes, is read; what lies there is given as zeros.
// OFTEN: addresses are often aligned, and then one load is all (where they seldom are, the second test costs more:
// AdamW over 130M parameters 600 us without it, 640 with).
// inner: known to be far enough from both ends.
template <bool OFTEN, class TE>
__device__ __forceinline__ void load16_any(uint32_t *r, const TE *p, const TE *begin, const TE *end, bool inner = false)
{
    const unsigned q = (unsigned)((uintptr_t)p & 15u);
    const char *base = reinterpret_cast<const char *>(p) - q;
    const uint4 *a = reinterpret_cast<const uint4 *>(base);
    if (OFTEN && q == 0 && (inner || base + 16 <= reinterpret_cast<const char *>(end))) {
        const uint4 u = a[0];
        r[0] = u.x, r[1] = u.y, r[2] = u.z, r[3] = u.w;
    } else if (inner || (base >= reinterpret_cast<const char *>(begin) && base + 32 <= reinterpret_cast<const char *>(end))) {
        uint32_t w[8];
        uint4 u = a[0];
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        if (OFTEN || q) u = a[1];
        w[4] = u.x, w[5] = u.y, w[6] = u.z, w[7] = u.w;
        straddle<(int)sizeof(TE)>(r, w, q);
    } else {
        constexpr int N = 16 / (int)sizeof(TE);
        Packed<TE, N> v;
        v.clear();
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (p + k >= begin && p + k < end) v.put(k, p[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = v.w[i];
    }
}

// The second kernel of a pair is launched while the first still runs: it waits here for the first one's end and what it
// wrote.
__device__ __forceinline__ void wait_for_earlier() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_later_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float group_rsqrt(float v) { return rsqrtf(v); }      // within 2 units
__device__ __forceinline__ double group_rsqrt(double v) { return rsqrt(v); }

// act(g) and its derivative, HOW exactly: by CUDA's functions (results of 32 or 64 bits); CLOSE by the hardware's exponential
// and reciprocal (16-bit gates whose results have 32 bits), a relative error of a few 2^-22 over the range where a
// sigmoid is not 0 or 1; ROUGH the same with a rounded exponent, which adds |g| 2^-24 (results that are rounded to
// 16 bits).  The tangent is the library's in every case, because near zero its relative error is
// what a gate that starts at zero sees.
// A slope is a product with the small side of the gate, which comes from the exponential itself: 1 - s of an s that is
// rounded near 1 has few correct bits (at g = 12 one in a hundred is wrong, beyond 17 nothing is left).
enum How { kExact, kClose, kRough };

__device__ __forceinline__ float tanh_of(float g) { return tanhf(g); }
__device__ __forceinline__ double tanh_of(double g) { return tanh(g); }
__device__ __forceinline__ Two<float> finite(Two<float> e) { return two(fminf(first(e), 0x1p127f), fminf(second(e), 0x1p127f)); }
__device__ __forceinline__ Two<double> finite(Two<double> e) { return two(fmin(e.a, 0x1p1023), fmin(e.b, 0x1p1023)); }
__device__ __forceinline__ Two<float> magnitudes(Two<float> g) { return two(fabsf(first(g)), fabsf(second(g))); }
__device__ __forceinline__ Two<double> magnitudes(Two<double> g) { return two(fabs(g.a), fabs(g.b)); }

__device__ __forceinline__ Two<float> hardware_exp2(Two<float> x)
{
    float a, b;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(first(x)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(second(x)));
    return two(a, b);
}
// exp(factor * g), factor -1 or -2
template <int HOW>
__device__ __forceinline__ Two<float> exponential(Two<float> g, float factor)
{
    if constexpr (HOW == kExact) return two(expf(factor * first(g)), expf(factor * second(g)));
    else if constexpr (HOW == kRough) return hardware_exp2(g * both(1.4426950408889634f * factor));
    // log2(e) in two parts of one sign: times the first, of 13 bits, a number of 16 bits (11 of them significant) is
    // exact, and where one power is 0 or infinite the other does not turn it
    else return hardware_exp2(g * both(0x1.715p+0f * factor)) * hardware_exp2(g * both(0x1.1d94aep-14f * factor));
}
template <int HOW>
__device__ __forceinline__ Two<double> exponential(Two<double> g, double factor)
{
    return two(exp(factor * g.a), exp(factor * g.b));
}
// 1 / (1 + e)
template <int HOW>
__device__ __forceinline__ Two<float> one_over_more(Two<float> e)
{
    const Two<float> d = e + both(1.0f);                      // infinity gives 0
    if constexpr (HOW == kExact) return two(1.0f / first(d), 1.0f / second(d));
    float a, b;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(first(d)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(second(d)));
    return two(a, b);
}
template <int HOW>
__device__ __forceinline__ Two<double> one_over_more(Two<double> e)
{
    return two(1.0 / (1.0 + e.a), 1.0 / (1.0 + e.b));
}

template <int KIND, int HOW, class A>
__device__ __forceinline__ Two<A> activate(Two<A> g)
{
    if constexpr (KIND == FO_ACT_LINEAR) return g;
    else if constexpr (KIND == FO_ACT_TANH) return two(tanh_of(first(g)), tanh_of(second(g)));
    else {
        const Two<A> s = one_over_more<HOW>(exponential<HOW>(g, A(-1)));
        return KIND == FO_ACT_SILU ? g * s : s;
    }
}

// SLOPE: how exactly the slope is needed, where it takes a computation of its own.
template <int KIND, int HOW, int SLOPE, class A>
__device__ __forceinline__ Two<A> activate_slope(Two<A> g, Two<A> &slope)
{
    if constexpr (KIND == FO_ACT_LINEAR) {
        slope = both(A(1));
        return g;
    } else if constexpr (KIND == FO_ACT_TANH) {              // 4 q / (1 + q)^2, q = exp(-2 |g|)
        const Two<A> q = exponential<SLOPE>(magnitudes(g), A(-2)), r = one_over_more<SLOPE>(q);
        slope = q * both(A(4)) * r * r;
        return two(tanh_of(first(g)), tanh_of(second(g)));
    } else {
        const Two<A> e = exponential<HOW>(g, A(-1)), s = one_over_more<HOW>(e);
        const Two<A> rest = finite(e) * s;                   // 1 - s; anything where s is 0 and so the slope
        if constexpr (KIND == FO_ACT_SIGMOID) {
            slope = s * rest;
            return s;
        } else {
            const Two<A> a = g * s;
            slope = fused_ma(a, rest, s);
            return a;
        }
    }
}

// Calls go(kind) with the activation as a compile-time number, so that loops over elements do not
// branch on it.
template <class Go>
__device__ __forceinline__ void with_activation(int kind, Go go)
{
    if (kind == FO_ACT_LINEAR) go(std::integral_constant<int, FO_ACT_LINEAR>());
    else if (kind == FO_ACT_SIGMOID) go(std::integral_constant<int, FO_ACT_SIGMOID>());
    else if (kind == FO_ACT_SILU) go(std::integral_constant<int, FO_ACT_SILU>());
    else go(std::integral_constant<int, FO_ACT_TANH>());
}

// Launches a kernel that calls wait_for_earlier(), beside the kernel before it on the stream.
template <class... Params, class... Args>
cudaError_t launch_beside(void (*kern)(Params...), dim3 grid, int cta, cudaStream_t st, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)cta);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace fo
