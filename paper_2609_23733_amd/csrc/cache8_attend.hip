// Softmax attention over a paged cache of 8-bit codes, few rows per key head at a time.
//
// Row r = (i, h) of a sequence as in the attention over plain caches; with codes a, b and scales s, t
//   x_j = scale s_j (q . a_j),  lse = log sum e^{x_j},  O = sum e^{x_j - lse} t_j b_j.
// The scales meet fp32 numbers: s_j the logits, t_j the probabilities; the codes enter the MFMAs as bf16, exactly.
//
// A wave takes 32 slots (a tile) with 16 NB rows from global memory through registers, no LDS and no barrier: 16x16x32
// MFMAs take operands as the cache lies.
//   S^T = K Q^T: of 16 slots, lane (n, g) = (lane % 16, lane / 16) loads slot n's features 16 g .. + 15, one 16-byte piece; the
//     two MFMAs of 32 features sum over features in an order of their own, which the queries' loads share.
//     Result register r of lane (n, g): slot 4 g + r, row n.
//   O^T += V^T P^T: lane (n, g) loads features 4 n .. + 3 of its own eight slots (4 g + r of both halves), a dword each; four
//     MFMAs, one per feature of a dword, sum over the 32 slots in the order in which the lanes
//     hold the probabilities.  Result: row n, features 16 g + 4 r + f.
// Both loads fill whole 64-byte rows.  Bound by HBM over long caches, 132 bytes per slot and key head (688,000 slots of four key
// heads, 16 query heads: e4m3 74 us, 4.9 TB/s, int8 79; with the logits kept for the weights, 44 MB written, 94), over short
// ones by a wave's own instructions, some 1,600 cycles a tile (2,748 slots of 16 heads: 6.6 us).  Two or three tiles' loads ahead
// instead of one: 3 to 10 % slower, as are four waves a SIMD, whose registers spill.
#include <type_traits>

#include "attend_device.hpp"
#include "cache_codes.hpp"

namespace vp {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Eight fp32 values as NP bf16 operands: 2, rounded and the rest (2^-16 of each), or 3, exact.
template <int NP>
struct Parts {
    bf16x8 v[NP];
    __device__ __forceinline__ void set(const float (&x)[8]) {
        if constexpr (NP == 2) {
            v[0] = pack_bf16x8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
            float r[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = x[e] - (float)v[0][e];
            v[1] = pack_bf16x8(r[0], r[1], r[2], r[3], r[4], r[5], r[6], r[7]);
        } else {
            const Planes p = split8(x);
            v[0] = p.h, v[1] = p.m, v[2] = p.l;
        }
    }
};

// What a tile's loads bring.
struct Tile8 {
    u32x4 k[2];      // codes of slot 16 i + n, features 16 g .. + 15
    uint32_t v[8];   // codes of slots 4 g + (j & 3) of half j / 4, features 4 n .. + 3
    u32x4 s[2];      // scales of slots 16 i + 4 g .. + 3
};

template <typename T>
constexpr bool kBfRows = sizeof(T) == 2;

// T: the rows' type (bf16: queries as they are, probabilities in two parts; fp32: three parts each).
template <typename T, int CODE, int NB>
__global__ __launch_bounds__(256, NB == 1 && kBfRows<T> ? 3 : 2) void k_cache8_attend(AttendArgs a) {
    constexpr bool kBf = sizeof(T) == 2;
    constexpr int kQ = kBf ? 1 : 3, kP = kBf ? 2 : 3, RT = 16 * NB;
    constexpr int kRow = 68;
    __shared__ __attribute__((aligned(16))) float so[4][RT][kRow];
    __shared__ float sml[4][RT][2], smeet[RT][2];
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (row tiles, ranges and heads in the order of the attention over plain caches)
    const int turn = (blockIdx.x >> 3) / a.row_tiles, rt = (blockIdx.x >> 3) - turn * a.row_tiles;
    const int x8 = turn * 8 + (blockIdx.x & 7), heads = a.c.B * a.c.Hkv;
    const int split = x8 / heads;
    if (split >= a.nsplit) return;
    const int y = (x8 - split * heads + 5 * split) % heads, hk = y % a.c.Hkv, b = y / a.c.Hkv;

    const CacheSeq sq = cache_seq(a.c, b);
    const int nrows = sq.nq * a.G, row0 = rt * RT;
    if (row0 >= nrows) return;
    const int row_last = row0 + RT - 1 < nrows ? row0 + RT - 1 : nrows - 1;
    const int klim = cache_visible(sq, a.causal, row_last / a.G);
    const int c0 = split * a.chunk, c1 = c0 + a.chunk < klim ? c0 + a.chunk : klim;
    if (split > 0 && c0 >= klim) return;

    bf16x8 q[NB][2][kQ];
    f32x4 o[NB][4];
    float m[NB], l[NB];
    int vis[NB];
    float* logits[NB];
    auto zero_rows = [&]() {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            l[nb] = 0.f;
#pragma unroll
            for (int f = 0; f < 4; ++f) o[nb][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    zero_rows();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        int r = row0 + 16 * nb + n;
        const bool real = r < nrows;
        r = real ? r : nrows - 1;
        const int i = r / a.G, head = hk * a.G + r - i * a.G;
        vis[nb] = cache_visible(sq, a.causal, i);
        m[nb] = -INFINITY;
        const int64_t row = (int64_t)(sq.q0 + i) * a.Hq + head;
        logits[nb] = a.logits && real ? a.logits + row * a.logit_stride : nullptr;
        const T* qr = (const T*)a.Q + (int64_t)(sq.q0 + i) * a.q_stride + head * kD + 16 * g;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            if constexpr (kBf) {
                q[nb][st][0] = load_bf16x8((const bf16*)qr + 8 * st);
            } else {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = qr[8 * st + e];
                const Planes p = split8(x);
                q[nb][st][0] = p.h, q[nb][st][kQ > 1 ? 1 : 0] = p.m, q[nb][st][kQ > 2 ? 2 : 0] = p.l;
            }
        }
    }
    // slots that every row of the workgroup sees
    const int all = cache_visible(sq, a.causal, row0 / a.G), seen_by_all = all < c1 ? all : c1;

    const int nt_all = (c1 - c0 + 31) / 32, nt = nt_all > wave ? (nt_all - wave + 3) / 4 : 0;
    if (nt > 0) {
        PageWindow pw;
        const int page_mask = (1 << a.c.page_log2) - 1, last_unit = (c1 - 1) & ~15;
        auto fetch = [&](int t, Tile8& w) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // (halves past the end: the last one again)
                int k = c0 + (wave + 4 * t) * 32 + 16 * i;
                k = k < last_unit ? k : last_unit;
                const int64_t at = (((int64_t)pw.page(k >> a.c.page_log2, lane) * a.c.Hkv + hk) << a.c.page_log2) +
                                   (k & page_mask);
                const char *kp = (const char*)a.c.K + at * kD, *vp_ = (const char*)a.c.V + at * kD;
                w.k[i] = *(const u32x4*)(kp + n * kD + 16 * g);
                w.s[i] = *(const u32x4*)(a.c.scale + at + 4 * g);
#pragma unroll
                for (int j = 0; j < 4; ++j) w.v[4 * i + j] = *(const uint32_t*)(vp_ + (4 * g + j) * kD + 4 * n);
            }
        };
        auto compute = [&](int t, Tile8& w) {
            const int k0 = c0 + (wave + 4 * t) * 32;
            const bool partial = !pw.sane || k0 + 32 > seen_by_all;
            uint32_t units = 3;
            if (!pw.sane) {
                units = 0;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int at = (k0 + 16 * u) >> a.c.page_log2;
                    if (at <= pw.last && pw.valid(pw.row[at])) units |= 1u << u;
                }
            }
            float vs[8], ks[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                ks[j] = key_scale(w.s[j >> 2][j & 3]);
                vs[j] = value_scale(w.s[j >> 2][j & 3]);
            }
            if (partial) {
                // Slots past the end or on no page may hold anything: no value.  An e4m3 code that is a NaN would reach
                // rows that do not see its slot, as a product with their probability of 0: it becomes the slot's scale,
                // which does not.
                bool odd = false;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool live = k0 + 16 * (j >> 2) + 4 * g + (j & 3) < c1 && ((units >> (j >> 2)) & 1);
                    w.v[j] = live ? w.v[j] : 0u;
                    if (CODE == CODE_E4M3) odd = odd || (((w.v[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u);
                }
                if (CODE == CODE_E4M3 && __builtin_amdgcn_ballot_w64(odd)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool nan = (((w.v[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
                        if ((__builtin_amdgcn_ballot_w64(nan) >> (lane & 48)) & 0xffffu) {
                            vs[j] = __builtin_nanf("");
                            w.v[j] = 0u;
                        }
                    }
                }
            }
            float x[NB][8];
            {
                bf16x8 kb[2][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int st = 0; st < 2; ++st) kb[i][st] = decode8<CODE>(w.k[i][2 * st], w.k[i][2 * st + 1]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int p = kQ - 1; p >= 0; --p)
#pragma unroll
                            for (int st = 0; st < 2; ++st) s = mfma16(kb[i][st], q[nb][st][p], s);
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[nb][4 * i + r] = s[r] * ks[4 * i + r];
                    }
            }
            bf16x8 vf[4];
            {
                uint32_t e[8][2];
#pragma unroll
                for (int j = 0; j < 8; ++j) decode4<CODE>(w.v[j], &e[j][0], &e[j][1]);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    u32x4 d;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        d[j] = __builtin_amdgcn_perm(e[2 * j + 1][f >> 1], e[2 * j][f >> 1], f & 1 ? 0x07060302u : 0x05040100u);
                    vf[f] = __builtin_bit_cast(bf16x8, d);
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int left = vis[nb] - k0 - 4 * g;
                auto sees = [&](int j) { return 16 * (j >> 2) + (j & 3) < left && ((units >> (j >> 2)) & 1); };
                if (partial) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[nb][j] = sees(j) ? x[nb][j] : -INFINITY;
                }
                if (logits[nb])
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        *(f32x4*)(logits[nb] + k0 + 16 * i + 4 * g) =
                            f32x4{x[nb][4 * i], x[nb][4 * i + 1], x[nb][4 * i + 2], x[nb][4 * i + 3]};
                float p[8], sum;
                auto powers = [&](float ref) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] = exp2f_fast(fmaf(x[nb][j], a.c2, -ref));
                    sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                };
                powers(m[nb]);   // inf or NaN while m is -inf
                if (__builtin_amdgcn_ballot_w64(!(sum < kMoveAt))) {
                    // the reference moves to the maximum so far, of all lanes that share the row
                    float top = x[nb][0];
#pragma unroll
                    for (int j = 1; j < 8; ++j) top = maximum(top, x[nb][j]);
                    top = maximum(top, __shfl_xor(top, 16));
                    top = maximum(top, __shfl_xor(top, 32)) * a.c2;
                    const float mn = top > m[nb] ? top : m[nb];
                    const float f = m[nb] == mn ? 1.f : exp2f_fast(m[nb] - mn);   // 0 from -inf
                    l[nb] *= f;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[nb][k][r] *= f;
                    m[nb] = mn;
                    powers(mn == -INFINITY ? 0.f : mn);
                }
                l[nb] += sum;
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] *= vs[j];
                if (partial) {   // (an unseen slot's scale may be anything)
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] = sees(j) ? p[j] : 0.f;
                }
                Parts<kP> pb;
                pb.set(p);
#pragma unroll
                for (int k = kP - 1; k >= 0; --k)
#pragma unroll
                    for (int f = 0; f < 4; ++f) o[nb][f] = mfma16(vf[f], pb.v[k], o[nb][f]);
            }
        };
        // Values whose sums leave fp32's range: once more with a reference that is known now, a row's log-sum-exp
        // and one, so that the probabilities sum to 1/2.
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            if (pass) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float s = l[nb] + __shfl_xor(l[nb], 16);
                    s += __shfl_xor(s, 32);
                    const float ref = m[nb] + __log2f(s) + 1.f;
                    m[nb] = fabsf(ref) <= 3.4028235e38f ? ref : -INFINITY;
                }
                zero_rows();
            }
            pw.start(a.c, b, c0, c1 - 1, lane);
            Tile8 w0, w1;
            // A tile's loads are issued before the last one's are waited for; no branch skips them (past the end: the last
            // tile again), as the wait counts the loads behind those it is for on every way there.
            fetch(0, w0);
            for (int t = 0; t < nt; t += 2) {
                fetch(t + 1 < nt ? t + 1 : nt - 1, w1);
                compute(t, w0);
                fetch(t + 2 < nt ? t + 2 : nt - 1, w0);
                if (t + 1 < nt) compute(t + 1, w1);
            }
            float top = 0.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = maximum(top, fabsf(o[nb][f][r]));
            if (!__builtin_amdgcn_ballot_w64(!(top <= 3.4028235e38f))) break;
        }
    }

    // The four waves' results meet in LDS.
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l[nb] += __shfl_xor(l[nb], 16);
        l[nb] += __shfl_xor(l[nb], 32);
        if (g == 0) {
            sml[wave][16 * nb + n][0] = m[nb];
            sml[wave][16 * nb + n][1] = l[nb];
        }
    }
    __syncthreads();
    const int64_t all_rows = (int64_t)a.c.T * a.Hq;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = 16 * nb + n;
        float M = -INFINITY, L = 0.f, mv[4], inv, lse;
#pragma unroll
        for (int v = 0; v < 4; ++v) M = maximum(M, mv[v] = sml[v][r][0]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int v = 0; v < 4; ++v) L += exp2f_fast(mv[v] - ref) * sml[v][r][1];
        row_result(M, L, &inv, &lse);
        const float f = exp2f_fast(m[nb] - ref) * inv;
        if (wave == 0 && g == 0) {
            smeet[r][0] = M;
            smeet[r][1] = L;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {   // features 16 g + 4 k + e
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = f == 0.f ? 0.f : o[nb][e][k] * f;   // (any values)
            *(f32x4*)&so[wave][r][16 * g + 4 * k] = v;
        }
    }
    __syncthreads();
    constexpr int kThreads = 256 / RT, kF = kD / kThreads;   // per row: threads, features of a thread (4 or 8)
    const int rr = tid / kThreads, d0 = tid % kThreads * kF, r = row0 + rr;
    if (r >= nrows) return;
    const int i = r / a.G;
    const int64_t at = (int64_t)(sq.q0 + i) * a.Hq + hk * a.G + r - i * a.G;
    const float M = smeet[rr][0], L = smeet[rr][1];
#pragma unroll
    for (int h = 0; h < kF; h += 4) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const f32x4 z = *(const f32x4*)&so[v][rr][d0 + h];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += z[e];
        }
        if (a.nsplit > 1) {
            *(f32x4*)(a.part + (split * all_rows + at) * kD + d0 + h) = acc;
        } else if constexpr (kBf) {
            bf16x4 z = {(bf16)acc[0], (bf16)acc[1], (bf16)acc[2], (bf16)acc[3]};
            *(bf16x4*)((bf16*)a.O + at * kD + d0 + h) = z;
        } else {
            *(f32x4*)((float*)a.O + at * kD + d0 + h) = acc;
        }
    }
    if (d0 == 0) {
        float inv, lse;
        row_result(M, L, &inv, &lse);
        if (a.nsplit > 1) *(f32x2*)(a.part_ml + (split * all_rows + at) * 2) = f32x2{M, L};
        else put_lse(a, at, lse);
    }
}

// ------------------------------------------------------------------ launchers

template <typename T, int CODE>
static void attend8_go(const AttendArgs& a, hipStream_t st) {
    const int64_t grid = ((int64_t)a.c.B * a.c.Hkv * a.nsplit + 7) / 8 * 8 * a.row_tiles;
    if (attend_rows(a) == 16) hipLaunchKernelGGL((k_cache8_attend<T, CODE, 1>), dim3(grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_cache8_attend<T, CODE, 2>), dim3(grid), dim3(256), 0, st, a);
}

void launch_cache8_attend(const AttendArgs& a, hipStream_t st) {
    if (a.c.dtype == DT_BF16) {
        if (a.c.code == CODE_E4M3) attend8_go<bf16, CODE_E4M3>(a, st);
        else attend8_go<bf16, CODE_INT8>(a, st);
    } else {
        if (a.c.code == CODE_E4M3) attend8_go<float, CODE_E4M3>(a, st);
        else attend8_go<float, CODE_INT8>(a, st);
    }
}

}  // namespace vp
