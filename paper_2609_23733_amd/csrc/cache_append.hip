// Rotary positions, and the append of a chunk of new tokens to a paged key-value cache.
//
// The first `dim` of a head's 64 features form dim / 2 pairs in `axes` equal sections, section a
// turned by position pos[t][a]: half layout pairs feature j with j + n of its section (n pairs),
// interleaved layout 2 j with 2 j + 1.  Pair (x0, x1) becomes
//   mag (x0 cos - x1 sin, x1 cos + x0 sin)  of the angle  2 pi pos f,
// f a 64-bit fraction of a revolution, so that pos f mod 1 is an integer product's low 64 bits:
// exact at any position, where an fp32 product of position and frequency would be off by
// pos 2^-24 radians.  The transpose (sign -1) is the gradient.  Features from `dim` on
// pass unchanged.
//
// Bound by memory (each value read and written once).  A thread owns four pairs of a token, whose
// sines and cosines it computes once and uses for several heads; eight threads cover a head's row.
#include "rotary_device.hpp"

namespace vp {

// Four pairs' sines and cosines: pair indices 4 c .. 4 c + 3 of token t.
struct Turn4 {
    float co[4], si[4];
    __device__ __forceinline__ void set(const RotArgs& r, int64_t t, int p0, int n, int count) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int p = p0 + (e < count ? e : count - 1);
            const uint64_t turn = (uint64_t)(int64_t)r.pos[t * r.axes + p / n] * r.freq[p];
            float s, c;
            sincos_turn((uint32_t)(turn >> 32), &s, &c);
            co[e] = c * r.mag;
            si[e] = s * r.mag * r.sign;
        }
    }
};

// One head's row: the thread's eight features, rotated.  Vector form: n % 4 == 0, the
// thread's pairs are two groups of four features, or eight in a row.
template <typename T, bool NT>
__device__ __forceinline__ void rotate8(const T* x, T* y, const Turn4& w, int lo, int hi, bool inter) {
    typedef typename Vec4<T>::type V;
    V a, b, ya, yb;
    struct Pair {
        V a, b;
    };
    if (inter) {   // eight in a row
        const Pair p = *(const Pair*)(x + lo);
        a = p.a, b = p.b;
    } else {
        a = *(const V*)(x + lo), b = *(const V*)(x + hi);
    }
    float f[8], g[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = (float)a[e], f[4 + e] = (float)b[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i0 = inter ? 2 * e : e, i1 = inter ? 2 * e + 1 : 4 + e;
        // (selected per element so that both layouts keep f in registers)
        const float x0 = f[i0], x1 = f[i1];
        g[i0] = x0 * w.co[e] - x1 * w.si[e];
        g[i1] = x1 * w.co[e] + x0 * w.si[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) ya[e] = (T)g[e], yb[e] = (T)g[4 + e];
    if (inter) {
        put8<NT>(y + lo, ya, yb);
    } else {
        put<NT>((V*)(y + lo), ya);
        put<NT>((V*)(y + hi), yb);
    }
}

template <typename T, bool NT>
__device__ __forceinline__ void copy8(const T* x, T* y) {
    struct __attribute__((aligned(16))) Eight {
        typename Vec4<T>::type a, b;
    };
    const Eight v = *(const Eight*)x;
    put8<NT>(y, v.a, v.b);
}

// What a thread (chunk c of eight, token t) does to a head's row.
template <typename T, bool INTER, bool NT>
struct Rotor {
    Turn4 w;
    int c, lo, hi, n, dim;
    bool vec;      // whole chunks of pairs
    __device__ __forceinline__ void set(const RotArgs& r, int64_t t, int chunk) {
        c = chunk;
        dim = r.dim;
        n = dim / r.axes / 2;
        vec = (n & 3) == 0;
        if (8 * c >= dim) return;
        if (INTER || vec) {
            const int left = dim / 2 - 4 * c;
            w.set(r, t, 4 * c, n, left < 4 ? left : 4);
        } else {
            w.set(r, t, 4 * c, n, dim / 2 - 4 * c < 4 ? dim / 2 - 4 * c : 4);
        }
        if (INTER) {
            lo = 8 * c;
            hi = lo + 4;
        } else {
            const int a = 4 * c / n, j = 4 * c - a * n;
            lo = 2 * a * n + j;
            hi = lo + n;
        }
    }
    // Rows x and y may be the same.
    __device__ __forceinline__ void row(const T* x, T* y) const {
        if (vec) {
            if (8 * c < dim) rotate8<T, NT>(x, y, w, lo, hi, INTER);
            else copy8<T, NT>(x + 8 * c, y + 8 * c);
            return;
        }
        // Sections whose pairs do not come in fours: feature by feature.  The thread owns pairs
        // 4 c .. 4 c + 3 (below dim / 2) and, of the features that pass unchanged, those among
        // 8 c .. 8 c + 7.
        for (int e = 0; e < 4; ++e) {
            const int p = 4 * c + e;
            if (p >= dim / 2) break;
            const int a = p / n, j = p - a * n;
            const int i0 = INTER ? 2 * p : 2 * a * n + j, i1 = INTER ? i0 + 1 : i0 + n;
            float co = w.co[0], si = w.si[0];
#pragma unroll
            for (int q = 1; q < 4; ++q)
                if (q == e) co = w.co[q], si = w.si[q];
            const float x0 = (float)x[i0], x1 = (float)x[i1];
            y[i0] = (T)(x0 * co - x1 * si);
            y[i1] = (T)(x1 * co + x0 * si);
        }
        for (int i = 8 * c > dim ? 8 * c : dim; i < 8 * c + 8; ++i) y[i] = x[i];
    }
};

// hs threads of eight share a token; each takes every hs-th head.
// 43,968 tokens of 16 heads, bf16: 44 us, 4.1 TB/s.
template <typename T, bool INTER, bool NT>
__global__ __launch_bounds__(256) void k_rotary(const T* x, int64_t x_stride, T* y, int64_t y_stride,
                                                int Tn, int H, int hs, RotArgs r) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id & 7), h0 = (int)((id >> 3) % hs);
    const int64_t t = (id >> 3) / hs;
    if (t >= Tn) return;
    Rotor<T, INTER, NT> rot;
    rot.set(r, t, c);
    const T* xr = x + t * x_stride;
    T* yr = y + t * y_stride;
#pragma unroll 4
    for (int h = h0; h < H; h += hs) rot.row(xr + h * kD, yr + h * kD);
}

// Rows of a token: Q's heads (to Q_out), K's (to the page), V's (to the page, as they are).
// 1,374 tokens of 16 + 16 + 16 heads, bf16: 7.4 us, 17 MB.  Bound by the latency of a thread's rows one after the other:
// Q_out may be Q, so no row is loaded before the last one's store.
template <typename T, bool INTER>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a, RotArgs r, int hs) {
    const int b = blockIdx.y;
    const CacheSeq sq = cache_seq(a.c, b);
    const int id = blockIdx.x * 256 + threadIdx.x;
    const int c = id & 7, h0 = (id >> 3) % hs, i = (id >> 3) / hs;
    if (i >= sq.nq) return;
    const int64_t t = sq.q0 + i;
    const int slot = sq.len - sq.n + i;
    int page = -1;
    if (slot >= 0) page = a.c.table[(int64_t)b * a.c.max_pages + (slot >> a.c.page_log2)];
    const bool live = page >= 0 && page < a.c.npages;
    const int in = slot & ((1 << a.c.page_log2) - 1);
    Rotor<T, INTER, false> rot;
    rot.set(r, t, c);
    const int Hkv = a.c.Hkv, hq = a.Q ? a.Hq : 0;
    for (int h = h0; h < hq + 2 * Hkv; h += hs) {
        if (h < hq) {
            rot.row((const T*)a.Q + t * a.q_stride + h * kD, (T*)a.Qo + (t * a.Hq + h) * kD);
            continue;
        }
        if (!live) continue;
        const bool isv = h >= hq + Hkv;
        const int hk = h - hq - (isv ? Hkv : 0);
        const int64_t at = (((int64_t)page * Hkv + hk) << a.c.page_log2) + in;
        if (isv) {
            copy8<T, false>((const T*)a.Vn + t * a.v_stride + hk * kD + 8 * c, (T*)a.c.V + at * kD + 8 * c);
        } else {
            rot.row((const T*)a.Kn + t * a.k_stride + hk * kD, (T*)a.c.K + at * kD);
            if (c == 0) {
                if (a.c.weight) a.c.weight[at] = 0.f;
                if (a.c.stamp) a.c.stamp[at] = a.c.seen[b] - sq.n + i;
            }
        }
    }
}

template <typename T, bool NT>
static void rotary_go(const void* x, int64_t x_stride, void* y, int64_t y_stride, int Tn, int H,
                      const RotArgs& r, hipStream_t st) {
    // (neighbouring heads of a token in one wave: eight rows in a row)
    const int hs = head_split(Tn, H, NT ? 2048 * 1024 : 256 * 1024);
    const dim3 grid((unsigned)(((int64_t)Tn * hs * 8 + 255) / 256));
    if (r.layout == 0)
        hipLaunchKernelGGL((k_rotary<T, true, NT>), grid, dim3(256), 0, st, (const T*)x, x_stride, (T*)y,
                           y_stride, Tn, H, hs, r);
    else
        hipLaunchKernelGGL((k_rotary<T, false, NT>), grid, dim3(256), 0, st, (const T*)x, x_stride, (T*)y,
                           y_stride, Tn, H, hs, r);
}

void launch_rotary(int dtype, const void* x, int64_t x_stride, void* y, int64_t y_stride, int T,
                   int H, const RotArgs& r, hipStream_t st) {
    const bool big = (int64_t)T * H * kD * (dtype == DT_BF16 ? 2 : 4) > ((int64_t)32 << 20);   // the L2s' size
    if (dtype == DT_BF16) {
        if (big) rotary_go<bf16, true>(x, x_stride, y, y_stride, T, H, r, st);
        else rotary_go<bf16, false>(x, x_stride, y, y_stride, T, H, r, st);
    } else {
        if (big) rotary_go<float, true>(x, x_stride, y, y_stride, T, H, r, st);
        else rotary_go<float, false>(x, x_stride, y, y_stride, T, H, r, st);
    }
}

// A view of 1,374 tokens appended takes 7.9 us with three rows per thread, 9.1 with one and a half.
void launch_cache_append(const AppendArgs& a, const RotArgs& r, hipStream_t st) {
    const int hs = head_split((int64_t)a.c.B * a.c.max_q, (a.Q ? a.Hq : 0) + 2 * a.c.Hkv, 128 * 1024);
    const dim3 grid((unsigned)(((int64_t)a.c.max_q * hs * 8 + 255) / 256), a.c.B);
#define GO(TT, IN) hipLaunchKernelGGL((k_cache_append<TT, IN>), grid, dim3(256), 0, st, a, r, hs)
    if (a.c.dtype == DT_BF16) {
        if (r.layout == 0) GO(bf16, true);
        else GO(bf16, false);
    } else {
        if (r.layout == 0) GO(float, true);
        else GO(float, false);
    }
#undef GO
}

}  // namespace vp
