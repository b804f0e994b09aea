// Append to a paged cache with norms and 8-bit codes, and the reading back of slots.
#include "cache_codes.hpp"

namespace vp {

// ------------------------------------------------------------------------
// Append: rows of a token, Q's heads (normalised and turned, to Q_out), K's (normalised, turned and quantised, to
// the page), V's (quantised, to the page); CODE_NONE: stored in the rows' type.  Eight lanes share a row, whose largest value
// takes three exchanges; the row goes from load to codes in registers.  hs threads of eight share a token, each
// takes every hs-th row: of Q, then of K, then of V, the first of each loaded at once (Q_out may be Q).
// Chunks: 32 neighbouring tokens' threads of one row are neighbours, so that what a page gets per slot (codes, scales,
// weight, stamp) is written in runs.
//
// K is normalised and turned in fp64: a row's code follows from its side of a border between two codes, which fp32's
// errors put a few features of a view's 1.4 million on the wrong one of (8.3 us in fp32, 10.0 so).
// ------------------------------------------------------------------------
// d in fp32, cut, the last bit set if anything was cut off: on d's side of every border between codes (fp32 rounding
// might put it on the border itself).
__device__ __forceinline__ float beside(double d) {
    uint32_t lo = (uint32_t)__double2loint(d);
    lo = (lo & 0xe0000000u) | (lo & 0x1fffffffu ? 0x20000000u : 0u);
    return (float)__hiloint2double(__double2hiint(d), (int)lo);
}

template <typename Turn>
struct Row64 {
    double co[4], si[4];
    __device__ __forceinline__ void angles(const RotArgs& r, int64_t t, int c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            co[e] = 1.;
            si[e] = 0.;
            const int p = 4 * c + e;
            if (p >= r.dim / 2) continue;
            sincos_turn64((uint64_t)(int64_t)r.pos[t * r.axes + Turn::section(r, p)] * r.freq[p], &si[e], &co[e]);
            co[e] *= (double)r.mag;
            si[e] *= (double)r.mag;
        }
    }
    __device__ __forceinline__ void turned(const NormArgs& nm, const Turn& w, int h, float (&f)[8]) const {
        double v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (double)f[e];
        if (nm.on) {
            Affine p;
            p.set(nm, w, h);
            if (nm.layer) {
                const double mean = sum8(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]))) * (1. / kD);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] -= mean;
            }
            double s = 0.;
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma(v[e], v[e], s);
            const double inv = rsqrt(fma(sum8(s), 1. / kD, (double)nm.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fma(v[e] * inv, (double)p.gain[e], (double)p.bias[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double a = v[2 * e], b = v[2 * e + 1];
            const bool turn = e < w.pairs;
            f[2 * e] = beside(turn ? fma(a, co[e], -(b * si[e])) : a);
            f[2 * e + 1] = beside(turn ? fma(b, co[e], a * si[e]) : b);
        }
    }
};

struct Spread {
    int hs, runs;
    int k0, v0;      // rows of Q, and of Q and K, modulo hs
};

template <int CODE>
__device__ __forceinline__ uint32_t quantise(float (&f)[8], uint32_t* lo, uint32_t* hi, bool inter) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);   // (a NaN's bits exceed all)
    float inv;
    top = max8(top);
    const float s = code_scale<CODE>(top, &inv), lim = code_limit<CODE>(top);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = inv == 0.f ? 0.f : f[e] * inv;
    if (lim > 0.f)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = fminf(fmaxf(f[e], -lim), lim);
    if (inter) {   // eight in a row
        *lo = encode4<CODE>(f[0], f[1], f[2], f[3]);
        *hi = encode4<CODE>(f[4], f[5], f[6], f[7]);
    } else {
        *lo = encode4<CODE>(f[0], f[2], f[4], f[6]);
        *hi = encode4<CODE>(f[1], f[3], f[5], f[7]);
    }
    return __float_as_uint(s) >> 16;
}

// A row of the page: its eight features (or codes) and, by one lane, its scale.
template <typename T, int CODE, bool INTER, bool VEC>
__device__ __forceinline__ void put_row(const CacheArgs& a, void* pool, int64_t at, int isv, const HeadTurn<T, INTER, VEC>& w,
                                        float (&f)[8], int c) {
    if constexpr (CODE == CODE_NONE) {
        w.template store<false>((T*)pool + at * kD, f);
    } else {
        uint32_t lo, hi;
        const uint32_t s = quantise<CODE>(f, &lo, &hi, INTER || !VEC);
        char* row = (char*)pool + at * kD;
        if constexpr (VEC && INTER) {
            *(uint2*)(row + 8 * c) = make_uint2(lo, hi);
        } else if constexpr (VEC) {
            *(uint32_t*)(row + w.lo) = lo;
            *(uint32_t*)(row + w.hi) = hi;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t two = (e < 2 ? lo : hi) >> (16 * (e & 1));
                row[w.i0[e]] = (char)two;
                row[w.i1[e]] = (char)(two >> 8);
            }
        }
        if (c == 0) ((uint16_t*)(a.scale + at))[isv] = (uint16_t)s;
    }
}

// 1,374 tokens of 16 + 16 + 16 heads, bf16 to int8, with norms: 10.0 us, 20 MB (in fp32 8.3; 15.2 with
// the three kinds of row in one loop, whose arrays the compiler kept in memory).
template <typename T, int CODE, bool INTER, bool VEC>
__global__ __launch_bounds__(256) void k_cache_append8(AppendArgs a, NormArgs qn, NormArgs kn, RotArgs r, Spread sp) {
    const int b = blockIdx.y;
    const CacheSeq sq = cache_seq(a.c, b);
    const int id = blockIdx.x * 256 + threadIdx.x;
    const int c = id & 7, g = id >> 3;
    const int h0 = sp.runs ? (g >> 5) % sp.hs : g % sp.hs, i = sp.runs ? (g >> 5) / sp.hs * 32 + (g & 31) : g / sp.hs;
    if (i >= sq.nq) return;
    const int64_t t = sq.q0 + i;
    const int slot = sq.len - sq.n + i;
    const int Hkv = a.c.Hkv, hq = a.Q ? a.Hq : 0;
    // the first rows
    int hk = h0 - sp.k0, hv = h0 - sp.v0;
    hk += hk < 0 ? sp.hs : 0;
    hv += hv < 0 ? sp.hs : 0;
    HeadTurn<T, INTER, VEC> w;
    HeadTurn<T, true, true> plain;   // V: eight features in a row
    w.places(r, c);
    plain.lo = 8 * c;
    plain.hi = 8 * c + 4;
    const T *qr = (const T*)a.Q + t * a.q_stride, *kr = (const T*)a.Kn + t * a.k_stride, *vr = (const T*)a.Vn + t * a.v_stride;
    float fq[8], fk[8], fv[8];
    if (h0 < hq) w.load(qr + h0 * kD, fq);
    if (hk < Hkv) w.load(kr + hk * kD, fk);
    if (hv < Hkv) plain.load(vr + hv * kD, fv);
    int page = -1;
    if (slot >= 0) page = a.c.table[(int64_t)b * a.c.max_pages + (slot >> a.c.page_log2)];
    Row64<HeadTurn<T, INTER, VEC>> w64;
    if constexpr (CODE != CODE_NONE) {
        if (h0 < hq || hk < Hkv) w64.angles(r, t, c);
#pragma unroll
        for (int e = 0; e < 4; ++e) w.co[e] = (float)w64.co[e], w.si[e] = (float)w64.si[e];
    } else {
        w.angles(r, t, c);
    }
    auto turned = [&](const NormArgs& nm, int h, float (&f)[8]) {
        if (nm.on) {
            Affine p;
            p.set(nm, w, h);
            normalise(nm, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = fmaf(f[e], p.gain[e], p.bias[e]);
        }
        w.turn(f);
    };
    for (int h = h0; h < hq; h += sp.hs) {
        turned(qn, h, fq);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fq[e];
        if (h + sp.hs < hq) w.load(qr + (h + sp.hs) * kD, fq);
        w.template store<false>((T*)a.Qo + (t * a.Hq + h) * kD, v);
    }
    if (page < 0 || page >= a.c.npages) return;
    const int64_t at0 = (((int64_t)page * Hkv) << a.c.page_log2) + (slot & ((1 << a.c.page_log2) - 1));
    for (int h = hk; h < Hkv; h += sp.hs) {
        if constexpr (CODE != CODE_NONE) w64.turned(kn, w, h, fk);
        else turned(kn, h, fk);
        const int64_t at = at0 + ((int64_t)h << a.c.page_log2);
        put_row<T, CODE>(a.c, a.c.K, at, 0, w, fk, c);
        if (c == 0) {
            if (a.c.weight) a.c.weight[at] = 0.f;
            if (a.c.stamp) a.c.stamp[at] = a.c.seen[b] - sq.n + i;
        }
        if (h + sp.hs < Hkv) w.load(kr + (h + sp.hs) * kD, fk);
    }
    for (int h = hv; h < Hkv; h += sp.hs) {
        put_row<T, CODE>(a.c, a.c.V, at0 + ((int64_t)h << a.c.page_log2), 1, plain, fv, c);
        if (h + sp.hs < Hkv) plain.load(vr + (h + sp.hs) * kD, fv);
    }
}

// ------------------------------------------------------------------------
// Read: the last slots of every sequence, as many as its rows, as K and V rows [T, Hkv, 64].  Bound by memory: 132
// bytes of an 8-bit slot and head read, 256 (bf16) written.  Eight neighbouring rows of a wave are neighbouring slots of
// a head, so codes come in runs and every row's 128 bytes or more are written whole.  43,968 slots of 16 heads: 57 us, 4.8
// TB/s, what a copy reaches.
// ------------------------------------------------------------------------
template <typename S, int CODE, typename T, bool NT>
__global__ __launch_bounds__(256) void k_cache_read(ReadArgs a) {
    const int b = blockIdx.z, hk = blockIdx.y;
    const CacheSeq sq = cache_seq(a.c, b);
    const int c = threadIdx.x & 7, i = blockIdx.x * 32 + (threadIdx.x >> 3);
    if (i >= sq.nq) return;
    const int slot = sq.len - sq.n + i;
    int page = -1;
    if (slot >= 0) page = a.c.table[(int64_t)b * a.c.max_pages + (slot >> a.c.page_log2)];
    const int64_t to = ((int64_t)(sq.q0 + i) * a.c.Hkv + hk) * kD;
    float k[8] = {}, v[8] = {};
    HeadTurn<T, true, true> plain;
    plain.lo = 8 * c;
    plain.hi = 8 * c + 4;
    if (page >= 0 && page < a.c.npages) {
        const int64_t at = (((int64_t)page * a.c.Hkv + hk) << a.c.page_log2) + (slot & ((1 << a.c.page_log2) - 1));
        if constexpr (CODE == CODE_NONE) {
            plain.load((const S*)a.c.K + at * kD, k);
            plain.load((const S*)a.c.V + at * kD, v);
        } else {
            const uint2 kc = *(const uint2*)((const char*)a.c.K + at * kD + 8 * c);
            const uint2 vc = *(const uint2*)((const char*)a.c.V + at * kD + 8 * c);
            const uint32_t s = a.c.scale[at];
            float f[4];
            values4<CODE>(kc.x, key_scale(s), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = f[e];
            values4<CODE>(kc.y, key_scale(s), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[4 + e] = f[e];
            values4<CODE>(vc.x, value_scale(s), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = f[e];
            values4<CODE>(vc.y, value_scale(s), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 + e] = f[e];
        }
    }
    plain.template store<NT>((T*)a.Ko + to, k);
    plain.template store<NT>((T*)a.Vo + to, v);
}

// ------------------------------------------------------------------ launchers

// A view of 1,374 tokens (K in fp32): 16 threads of eight per token 8.4 us; 8 9.7, 32 9.4, one for each of the 48 rows 10.0.
static Spread append8_spread(const AppendArgs& a) {
    const int hq = a.Q ? a.Hq : 0, hs = head_split((int64_t)a.c.B * a.c.max_q, hq + 2 * a.c.Hkv, 128 * 1024);
    return Spread{hs, a.c.max_q >= 16, hq % hs, (hq + a.c.Hkv) % hs};
}
static int64_t append8_blocks(const AppendArgs& a, const Spread& sp) {   // per sequence
    const int64_t rows = sp.runs ? (int64_t)(a.c.max_q + 31) / 32 * 32 : a.c.max_q;
    return (rows * sp.hs * 8 + 255) / 256;
}
bool append8_fits(const AppendArgs& a) { return append8_blocks(a, append8_spread(a)) * a.c.B < 1 << 24; }
bool read_fits(const ReadArgs& a) { return (int64_t)((a.c.max_q + 31) / 32) * a.c.Hkv * a.c.B < 1 << 24; }

void launch_cache_append8(const AppendArgs& a, const NormArgs& qn, const NormArgs& kn, const RotArgs& r,
                          hipStream_t st) {
    const Spread sp = append8_spread(a);
    const dim3 grid((unsigned)append8_blocks(a, sp), a.c.B);
    const bool vec = pairs_in_fours(r), inter = r.layout == 0;
#define GO(TT, CO, IN, VE) hipLaunchKernelGGL((k_cache_append8<TT, CO, IN, VE>), grid, dim3(256), 0, st, a, qn, kn, r, sp)
#define GO_TURN(TT, CO)                                                          \
    do {                                                                         \
        if (inter) { if (vec) GO(TT, CO, true, true); else GO(TT, CO, true, false); }  \
        else { if (vec) GO(TT, CO, false, true); else GO(TT, CO, false, false); }      \
    } while (0)
#define GO_CODE(TT)                                               \
    do {                                                          \
        if (a.c.code == CODE_E4M3) GO_TURN(TT, CODE_E4M3);        \
        else if (a.c.code == CODE_INT8) GO_TURN(TT, CODE_INT8);   \
        else GO_TURN(TT, CODE_NONE);                              \
    } while (0)
    if (a.c.dtype == DT_BF16) GO_CODE(bf16);
    else GO_CODE(float);
#undef GO_CODE
#undef GO_TURN
#undef GO
}

void launch_cache_read(const ReadArgs& a, hipStream_t st) {
    const dim3 grid((a.c.max_q + 31) / 32, a.c.Hkv, a.c.B);
    const bool nt = (int64_t)a.c.T * a.c.Hkv * kD * (a.out_dtype == DT_BF16 ? 4 : 8) > ((int64_t)32 << 20);
#define GO(SS, CO, TT)                                                                                 \
    do {                                                                                               \
        if (nt) hipLaunchKernelGGL((k_cache_read<SS, CO, TT, true>), grid, dim3(256), 0, st, a);       \
        else hipLaunchKernelGGL((k_cache_read<SS, CO, TT, false>), grid, dim3(256), 0, st, a);         \
    } while (0)
#define GO_OUT(SS, CO)                                  \
    do {                                                \
        if (a.out_dtype == DT_BF16) GO(SS, CO, bf16);   \
        else GO(SS, CO, float);                         \
    } while (0)
    if (a.c.code == CODE_E4M3) GO_OUT(uint8_t, CODE_E4M3);
    else if (a.c.code == CODE_INT8) GO_OUT(uint8_t, CODE_INT8);
    else if (a.c.dtype == DT_BF16) GO_OUT(bf16, CODE_NONE);
    else GO_OUT(float, CODE_NONE);
#undef GO_OUT
#undef GO
}

}  // namespace vp
