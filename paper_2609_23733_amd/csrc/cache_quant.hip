// Append to a paged cache with norms and 8-bit codes, and the reading back of slots.
#include "cache_codes.hpp"

namespace vp {

// ------------------------------------------------------------------------
// Append: rows of a token, Q's heads (normalised and turned, to Q_out), K's (normalised, turned and quantised, to
// the page), V's (quantised, to the page); CODE_NONE: stored in the rows' type.  Eight lanes share a row, whose largest value
// takes three exchanges; the row goes from load to codes in registers.  hs threads of eight share a token, each
// takes every hs-th row, two loaded at a time (Q_out may be Q).
// ------------------------------------------------------------------------
template <int CODE>
__device__ __forceinline__ uint32_t quantise(float (&f)[8], uint32_t* lo, uint32_t* hi, bool inter) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);   // (a NaN's bits exceed all)
    float inv;
    const float s = code_scale<CODE>(max8(top), &inv);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = inv == 0.f ? 0.f : f[e] * inv;
    if (inter) {   // eight in a row
        *lo = encode4<CODE>(f[0], f[1], f[2], f[3]);
        *hi = encode4<CODE>(f[4], f[5], f[6], f[7]);
    } else {
        *lo = encode4<CODE>(f[0], f[2], f[4], f[6]);
        *hi = encode4<CODE>(f[1], f[3], f[5], f[7]);
    }
    return __float_as_uint(s) >> 16;
}

template <typename T, int CODE, bool INTER, bool VEC>
__global__ __launch_bounds__(256) void k_cache_append8(AppendArgs a, NormArgs qn, NormArgs kn, RotArgs r, int hs) {
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
    const int Hkv = a.c.Hkv, hq = a.Q ? a.Hq : 0, all = live ? hq + 2 * Hkv : hq;
    HeadTurn<T, INTER, VEC> w;
    HeadTurn<T, true, true> plain;   // V: eight features in a row
    w.places(r, c);
    plain.lo = 8 * c;
    plain.hi = 8 * c + 4;
    auto load = [&](int h, float (&f)[8]) {
        if (h < hq) w.load((const T*)a.Q + t * a.q_stride + h * kD, f);
        else if (h < hq + Hkv) w.load((const T*)a.Kn + t * a.k_stride + (h - hq) * kD, f);
        else plain.load((const T*)a.Vn + t * a.v_stride + (h - hq - Hkv) * kD, f);
    };
    float f[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (h0 + k * hs < all) load(h0 + k * hs, f[k]);
    w.angles(r, t, c);
    for (int h = h0; h < all; h += 2 * hs) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int hk = h + k * hs;
            if (hk >= all) break;
            float v[8];
            const bool isq = hk < hq, isv = hk >= hq + Hkv;
            const NormArgs& nm = isq ? qn : kn;
            if (!isv) {
                if (nm.on) {
                    Affine p;
                    p.set(nm, w, isq ? hk : hk - hq);
                    normalise(nm, f[k]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[k][e] = fmaf(f[k][e], p.gain[e], p.bias[e]);
                }
                w.turn(f[k]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = f[k][e];
            if (hk + 2 * hs < all) load(hk + 2 * hs, f[k]);
            if (isq) {
                w.template store<false>((T*)a.Qo + (t * a.Hq + hk) * kD, v);
                continue;
            }
            const int head = hk - hq - (isv ? Hkv : 0);
            const int64_t at = (((int64_t)page * Hkv + head) << a.c.page_log2) + in;
            if constexpr (CODE == CODE_NONE) {
                if (isv) plain.template store<false>((T*)a.c.V + at * kD, v);
                else w.template store<false>((T*)a.c.K + at * kD, v);
            } else {
                uint32_t lo, hi;
                const uint32_t s = quantise<CODE>(v, &lo, &hi, isv || INTER || !VEC);
                if (isv) {
                    *(uint2*)((char*)a.c.V + at * kD + 8 * c) = make_uint2(lo, hi);
                } else if constexpr (VEC && INTER) {
                    *(uint2*)((char*)a.c.K + at * kD + 8 * c) = make_uint2(lo, hi);
                } else if constexpr (VEC) {
                    *(uint32_t*)((char*)a.c.K + at * kD + w.lo) = lo;
                    *(uint32_t*)((char*)a.c.K + at * kD + w.hi) = hi;
                } else {
                    char* kr = (char*)a.c.K + at * kD;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t two = (e < 2 ? lo : hi) >> (16 * (e & 1));
                        kr[w.i0[e]] = (char)two;
                        kr[w.i1[e]] = (char)(two >> 8);
                    }
                }
                if (c == 0) ((uint16_t*)(a.c.scale + at))[isv] = (uint16_t)s;
            }
            if (!isv && c == 0) {
                if (a.c.weight) a.c.weight[at] = 0.f;
                if (a.c.stamp) a.c.stamp[at] = a.c.seen[b] - sq.n + i;
            }
        }
    }
}

// ------------------------------------------------------------------------
// Read: the last slots of every sequence, as many as its rows, as K and V rows [T, Hkv, 64].  Bound by memory: 132
// bytes of an 8-bit slot and head read, 256 (bf16) written.  Eight neighbouring rows of a wave are neighbouring slots of
// a head, so codes come in runs and every row's 128 bytes or more are written whole.
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

void launch_cache_append8(const AppendArgs& a, const NormArgs& qn, const NormArgs& kn, const RotArgs& r,
                          hipStream_t st) {
    const int hs = head_split((int64_t)a.c.B * a.c.max_q, (a.Q ? a.Hq : 0) + 2 * a.c.Hkv, 128 * 1024);
    const dim3 grid((unsigned)(((int64_t)a.c.max_q * hs * 8 + 255) / 256), a.c.B);
    const bool vec = pairs_in_fours(r), inter = r.layout == 0;
#define GO(TT, CO, IN, VE) hipLaunchKernelGGL((k_cache_append8<TT, CO, IN, VE>), grid, dim3(256), 0, st, a, qn, kn, r, hs)
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
