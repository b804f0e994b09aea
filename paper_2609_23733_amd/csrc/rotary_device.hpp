// Rotary positions: what the kernels that turn heads' features share.
#pragma once

#include "cache_device.hpp"

namespace vp {

template <typename T>
struct Vec4 {
    typedef T type __attribute__((__vector_size__(4 * sizeof(T))));
};

// Stores that pass the caches by (NT), for outputs larger than these: 43,968 tokens of 16 heads
// 50 -> 44 us.
template <bool NT, typename V>
__device__ __forceinline__ void put(V* p, V v) {
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Eight features in a row, at a 16-byte boundary: 16 bytes at a time.
template <bool NT, typename T>
__device__ __forceinline__ void put8(T* p, typename Vec4<T>::type a, typename Vec4<T>::type b) {
    if constexpr (sizeof(T) == 2) {
        typedef T V8 __attribute__((__vector_size__(16)));
        put<NT>((V8*)p, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        put<NT>((typename Vec4<T>::type*)p, a);
        put<NT>((typename Vec4<T>::type*)(p + 4), b);
    }
}

// Sine and cosine of a fraction of a revolution, 32 bits: the nearest quarter turn from the top bits,
// the rest, |x| <= pi / 4, by the Taylor series to x^9 and x^10 (errors 2e-9 and 2e-9 there).
__device__ __forceinline__ void sincos_turn(uint32_t t, float* sn, float* cs) {
    const uint32_t q = (t + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(t - (q << 30)) * (1.57079632679489662f / 1073741824.f), x2 = x * x;
    float s = fmaf(x2, 1.f / 362880.f, -1.f / 5040.f);
    s = fmaf(x2, s, 1.f / 120.f);
    s = fmaf(x2, s, -1.f / 6.f);
    s = fmaf(x2 * s, x, x);
    float c = fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f);
    c = fmaf(x2, c, -1.f / 720.f);
    c = fmaf(x2, c, 1.f / 24.f);
    c = fmaf(x2, c, -0.5f);
    c = fmaf(x2, c, 1.f);
    const float a = q & 1 ? c : s, b = q & 1 ? s : c;
    *sn = __uint_as_float(__float_as_uint(a) ^ ((q & 2) << 30));
    *cs = __uint_as_float(__float_as_uint(b) ^ (((q + 1) & 2) << 30));
}

// The same in fp64 from all 64 bits of the fraction: Taylor series to x^13 and x^14 (errors below 3e-14).
__device__ __forceinline__ void sincos_turn64(uint64_t t, double* sn, double* cs) {
    const uint64_t q = (t + 0x2000000000000000ull) >> 62;
    const double x = (double)(int64_t)(t - (q << 62)) * (1.57079632679489661923 / 4611686018427387904.), x2 = x * x;
    double s = 1. / 6227020800., c = -1. / 87178291200.;   // 1 / 13!, 1 / 14!
    s = fma(x2, s, -1. / 39916800.);
    s = fma(x2, s, 1. / 362880.);
    s = fma(x2, s, -1. / 5040.);
    s = fma(x2, s, 1. / 120.);
    s = fma(x2, s, -1. / 6.);
    s = fma(x2 * s, x, x);
    c = fma(x2, c, 1. / 479001600.);
    c = fma(x2, c, -1. / 3628800.);
    c = fma(x2, c, 1. / 40320.);
    c = fma(x2, c, -1. / 720.);
    c = fma(x2, c, 1. / 24.);
    c = fma(x2, c, -0.5);
    c = fma(x2, c, 1.);
    const double a = q & 1 ? c : s, b = q & 1 ? s : c;
    *sn = q & 2 ? -a : a;
    *cs = (q + 1) & 2 ? -b : b;
}

// Sum, and largest value, of the eight lanes that share a head's row.
template <int CTRL>
__device__ __forceinline__ int lane_of(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ float sum8(float x) {
    x += __builtin_bit_cast(float, lane_of<0xb1>(__builtin_bit_cast(int, x)));    // lane ^ 1
    x += __builtin_bit_cast(float, lane_of<0x4e>(__builtin_bit_cast(int, x)));    // lane ^ 2
    return x + __builtin_bit_cast(float, lane_of<0x141>(__builtin_bit_cast(int, x)));   // 7 - lane: the other four
}
template <int CTRL>
__device__ __forceinline__ double lane_of64(double x) {
    return __hiloint2double(lane_of<CTRL>(__double2hiint(x)), lane_of<CTRL>(__double2loint(x)));
}
__device__ __forceinline__ double sum8(double x) {
    x += lane_of64<0xb1>(x);
    x += lane_of64<0x4e>(x);
    return x + lane_of64<0x141>(x);
}
__device__ __forceinline__ uint32_t max8(uint32_t x) {
    x = max(x, (uint32_t)lane_of<0xb1>((int)x));
    x = max(x, (uint32_t)lane_of<0x4e>((int)x));
    return max(x, (uint32_t)lane_of<0x141>((int)x));
}

// Eight features of a head's row in one thread (chunk c of eight): pairs 4 c .. 4 c + 3 of those that are
// turned, f[2 e] and f[2 e + 1] the pair's two; past the turned features two neighbours.  VEC: pairs per
// section in fours, so that a thread's features are two runs of four, or one of eight.
template <typename T, bool INTER, bool VEC>
struct HeadTurn {
    float co[4], si[4];
    int pairs;                              // of the four: turned (the first)
    int lo, hi;                             // VEC: first features of the runs
    int sec;                                // and their section
    int i0[VEC ? 1 : 4], i1[VEC ? 1 : 4];   // features of a pair
    // p / r.n of a pair: (p + 1/2) / n lies 1 / 64 from a whole number at least.  (An integer division per pair and
    // thread took longer than the rest of a row.)
    static __device__ __forceinline__ int section(const RotArgs& r, int p) { return (int)(((float)p + 0.5f) * r.inv_n); }
    __device__ __forceinline__ void places(const RotArgs& r, int c) {
        lo = 8 * c;
        hi = lo + 4;
        sec = 0;
        pairs = r.dim / 2 - 4 * c;
        if constexpr (VEC) {
            if (8 * c < r.dim) {
                sec = section(r, 4 * c);
                if (!INTER) {
                    lo = 4 * c + sec * r.n;
                    hi = lo + r.n;
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int p = 4 * c + e;
                i0[e] = 2 * p;
                i1[e] = 2 * p + 1;
                if (!INTER && p < r.dim / 2) {
                    i0[e] = p + section(r, p) * r.n;
                    i1[e] = i0[e] + r.n;
                }
            }
        }
    }
    __device__ __forceinline__ void angles(const RotArgs& r, int64_t t, int c) {
        int pos[4];
        uint64_t freq[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int p = 4 * c + e;
            pos[e] = 0;
            freq[e] = 0;
            if (p >= r.dim / 2) continue;
            pos[e] = VEC && e ? pos[0] : r.pos[t * r.axes + (VEC ? sec : section(r, p))];
            freq[e] = r.freq[p];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // bits 32 .. 63 of pos * freq: exact modulo a revolution
            const uint32_t u = (uint32_t)pos[e], fl = (uint32_t)freq[e], fh = (uint32_t)(freq[e] >> 32);
            const uint32_t turn = __umulhi(u, fl) + u * fh - (pos[e] < 0 ? fl : 0u);
            float s, k;
            sincos_turn(turn, &s, &k);
            const bool turned = 4 * c + e < r.dim / 2;
            co[e] = turned ? k * r.mag : 1.f;
            si[e] = turned ? s * r.mag : 0.f;
        }
    }
    template <typename U>
    __device__ __forceinline__ void load(const U* x, float (&f)[8]) const {
        typedef typename Vec4<U>::type V;
        if constexpr (VEC) {
            struct Run {
                V a, b;
            };
            Run v;
            if constexpr (INTER) {
                v = *(const Run*)(x + lo);
            } else {
                v.a = *(const V*)(x + lo);
                v.b = *(const V*)(x + hi);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[INTER ? e : 2 * e] = (float)v.a[e];
                f[INTER ? 4 + e : 2 * e + 1] = (float)v.b[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[2 * e] = (float)x[i0[e]], f[2 * e + 1] = (float)x[i1[e]];
        }
    }
    template <bool NT>
    __device__ __forceinline__ void store(T* y, const float (&f)[8]) const {
        typedef typename Vec4<T>::type V;
        if constexpr (VEC) {
            V a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = (T)f[INTER ? e : 2 * e];
                b[e] = (T)f[INTER ? 4 + e : 2 * e + 1];
            }
            if constexpr (INTER) {
                put8<NT>(y + lo, a, b);
            } else {
                put<NT>((V*)(y + lo), a);
                put<NT>((V*)(y + hi), b);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[i0[e]] = (T)f[2 * e], y[i1[e]] = (T)f[2 * e + 1];
        }
    }
    // (Features that are not turned stay as they are: an infinity times a sine of 0 would reach its neighbour.)
    __device__ __forceinline__ void turn(float (&f)[8]) const {
        if (VEC && pairs <= 0) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!VEC && e >= pairs) break;
            const float a = f[2 * e], b = f[2 * e + 1];
            // (fused by hand, so that every kernel rounds alike)
            f[2 * e] = fmaf(a, co[e], -(b * si[e]));
            f[2 * e + 1] = fmaf(b, co[e], a * si[e]);
        }
    }
    __device__ __forceinline__ void turn_back(float (&f)[8]) const {   // the transpose
        if (VEC && pairs <= 0) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!VEC && e >= pairs) break;
            const float a = f[2 * e], b = f[2 * e + 1];
            f[2 * e] = fmaf(a, co[e], b * si[e]);
            f[2 * e + 1] = fmaf(b, co[e], -(a * si[e]));
        }
    }
};

// The norm of a head's row over its 64 features: n = (x - mean) / sqrt(var + eps) (layer) or x / sqrt(mean x^2 +
// eps), then n gain + bias.  Mean, then the mean square of what is left: no difference of large sums.
struct NormArgs {
    const float *gain, *bias;   // may be null; [64], or [heads, 64]
    int on, layer, per_head;
    float eps;
};
__device__ __forceinline__ float normalise(const NormArgs& nm, float (&f)[8]) {
    if (nm.layer) {
        const float mean = sum8(((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]))) * (1.f / kD);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] -= mean;
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(f[k], f[k], s);
    const float r = 1.f / sqrtf(fmaf(sum8(s), 1.f / kD, nm.eps));
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] *= r;
    return r;
}
// A thread's eight gains and biases.
struct Affine {
    float gain[8], bias[8];
    template <typename Turn>
    __device__ __forceinline__ void set(const NormArgs& nm, const Turn& w, int h) {
        const int at = nm.per_head ? h * kD : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) gain[k] = 1.f, bias[k] = 0.f;
        if (nm.gain) w.load(nm.gain + at, gain);
        if (nm.bias) w.load(nm.bias + at, bias);
    }
};

// Whether a rotation's pairs come in fours (HeadTurn's VEC).
inline bool pairs_in_fours(const RotArgs& r) { return r.n % 4 == 0; }

// Threads (of eight) per token: one per head while that leaves compute units idle, fewer, each
// reusing its sines over more heads, when tokens alone make `threads` of them.
inline int head_split(int64_t tokens, int heads, int64_t threads) {
    int hs = 1;
    while (hs < heads && tokens * 8 * hs < threads) hs *= 2;
    return hs < heads ? hs : heads;
}

}  // namespace vp
