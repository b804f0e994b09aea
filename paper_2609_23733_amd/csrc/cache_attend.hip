// Softmax attention of a chunk of new tokens over a paged key-value cache, and the gathering of
// the attention weights that fall on every slot.
//
// Row (i, h) of a sequence, token i of the chunk and query head h = hk G + g, sees the first
// vis_i slots of key head hk:
//   x_j = scale q . k_j,  lse = log sum_{j < vis_i} e^{x_j},  O = sum_{j < vis_i} e^{x_j - lse} v_j.
// The G heads that share a key head are rows of one matrix product (row r = i G + g), so their
// keys and values are read once.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attend_device.hpp"
#include "cache_codes.hpp"

namespace vp {

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((__vector_size__(8)));

// ------------------------------------------------------------------------
// Geometry of the two kernel variants.  A wave multiplies groups of 32 rows with 32 slots (a block)
// at a time.  Narrow: 32 rows per workgroup, its four waves split the slots and each
// streams tiles of its own (no barrier until the end).  Wide: the four waves share every tile, with
// 64 rows each (bf16: an operand read from LDS serves two MFMAs; with 32 rows the LDS reads
// alone take as long as the MFMAs) or 32 (fp32, whose MFMAs take eight times as long).
// ------------------------------------------------------------------------
template <typename T, bool WIDE>
struct Geo {
    static constexpr bool kBf = sizeof(T) == 2;
    static constexpr bool kSplit = kBf && !WIDE;                // probabilities as two bf16 values
    static constexpr int NW = 4;                                // waves
    static constexpr int NB = WIDE && kBf ? 2 : 1;              // groups of 32 rows per wave
    static constexpr int TK = WIDE && kBf ? 64 : 32;            // slots per tile
    static constexpr int RT = WIDE ? 32 * NB * NW : 32;         // rows per workgroup
    static constexpr int ROWB = kD * sizeof(T);                 // bytes of a slot's K or V
    static constexpr int kBlock = 32 * ROWB;                    // bytes of a block's K or V
    static constexpr int kTileV = TK * ROWB;                    // a tile's V comes after its K
    static constexpr int kTile = 2 * TK * ROWB;
    // Tiles in LDS, and how many tiles ahead of the arriving one copies are issued: into the
    // place of the tile before it, or (wide bf16, where that one is still in use) of the one before.
    // Narrow fp32: one tile, whose K and V are replaced in turn.
    static constexpr int NST = WIDE ? (kBf ? 4 : 3) : kBf ? 2 : 1;
    static constexpr int AHEAD = WIDE && kBf ? NST - 2 : NST - 1;
    static constexpr int kRing = NST * kTile;
    static constexpr int kLds = WIDE ? kRing : 4 * kRing;
    // fp32, wide: a tile as three bf16 planes of K and three of V, two tiles
    static constexpr int kPlane = 32 * 128, kPlanes = 6 * kPlane;
    static_assert(kBf || !WIDE || 2 * kPlanes <= kLds, "the planes fit the ring");
    static constexpr int UC = 16 * ROWB / 1024;                 // 1 KB copies per 16 slots
    static constexpr int PPW = (TK / 16) * 2 / (WIDE ? NW : 1); // (16 slots of K or V) per wave
    static constexpr int CPT = PPW * UC;                        // copies per wave and tile
    // Slot within a block that result register r of lane half hh belongs to.
    static __device__ __forceinline__ constexpr int key(int r, int hh) {
        return kBf ? 16 * (r >> 3) + 8 * hh + (r & 7) : 8 * (r >> 2) + 4 * hh + (r & 3);
    }
};

// Wide workgroups over 8-bit codes: eight waves, which share the decoding of a tile (1,374 tokens over 43,968 slots of 16
// heads, e4m3, with bf16 probabilities: 273 us, with four waves 298; as they are now 279, of which the kernel takes 271, 920
// TFLOP/s, over a bf16 cache 260).
template <typename T, bool WIDE, int CODE>
struct GeoOf : Geo<T, WIDE> {
    static constexpr int NW = CODE == CODE_NONE ? Geo<T, WIDE>::NW : 8;
    static constexpr int RT = WIDE ? 32 * Geo<T, WIDE>::NB * NW : 32;
};

// Largest of the lanes' numbers of BITS bits, uniform: bit by bit, without the latency of exchanges.
template <int BITS>
__device__ __forceinline__ int top_of_wave(int x) {
    int r = 0;
#pragma unroll
    for (int b = BITS - 1; b >= 0; --b)
        if (__builtin_amdgcn_ballot_w64(x >= r + (1 << b))) r += 1 << b;
    return r;
}

template <int CPT>
__device__ __forceinline__ void wait_tiles(int behind) {
    // Copies are counted in the order of their issue: all but the `behind` youngest tiles' have
    // arrived.  Earlier LDS reads of this wave have returned, too.
    if (behind <= 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else if (behind == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(CPT) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(2 * CPT) : "memory");
}

// ------------------------------------------------------------------------
// The attention of one block by one wave.  S^T = K Q^T, so that a lane owns one query row (lane %
// 32) and its registers run over slots: the softmax's sum is per lane, and the
// probabilities are already the B operand of O^T += V^T P^T.  For that K's rows enter the MFMA
// with index bits 2 and 3 swapped (bf16), which puts eight consecutive slots into each lane half.
// V^T comes from the row-major tile by transposing LDS reads (bf16) or as it lies (fp32: one
// slot and 32 features per 32x32x2 MFMA and half).
//
// Probabilities are 2^(x - m) with a reference m (in log2 units) that is the row's maximum over its
// first block and moves only when a block's sum passes 2^16: fp32 sums and bf16 probabilities
// (see Probs; the sum l takes them unrounded) keep their relative
// precision at any scale, so ordinary blocks need no maximum.  When a block passes the bound (and
// at a row's first slots, where m = -inf makes the sum inf or NaN) its logits are formed again, m
// becomes the maximum so far and O and l are scaled to it.
// ------------------------------------------------------------------------
template <typename T>
struct Rows {
    static constexpr bool kBf = sizeof(T) == 2;
    bf16x8 qb[kBf ? 4 : 1];
    float qf[kBf ? 1 : 32];
    f32x16 o[2];
    float m, l;
    int vis;
};
// A block's probabilities as operands of the value product.  bf16, SPLIT: each as the sum of two bf16
// values, within 2^-16 of it, so that an output's own rounding is all that shows; two MFMAs for one.  Without it
// the rounding of the probabilities adds as much again (errors of 2.35e-3 of the result, with it 1.66e-3).
// Narrow workgroups split, as HBM hides most of it (tokens over 137,400 and 62,724 slots 182.8 us and 183.2, 32
// sequences ragged to 10,992 36.5 and 37.3, a token over 600 slots 8.9 and 9.8; 400 tokens over 5,000
// slots 29.6 and 34.0).  Wide ones, bound by their instructions and their registers, do not (a view over
// 43,968 slots 264 us, split 445).
template <typename T, bool SPLIT>
struct Probs;
template <bool SPLIT>
struct Probs<bf16, SPLIT> {
    bf16x8 v[2], rest[SPLIT ? 2 : 1];
    __device__ __forceinline__ void set(const f32x16& s) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
            v[st] = pack_bf16x8(s[8 * st], s[8 * st + 1], s[8 * st + 2], s[8 * st + 3], s[8 * st + 4],
                                s[8 * st + 5], s[8 * st + 6], s[8 * st + 7]);
        if constexpr (SPLIT)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                float r[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] = s[8 * st + e] - (float)v[st][e];
                rest[st] = pack_bf16x8(r[0], r[1], r[2], r[3], r[4], r[5], r[6], r[7]);
            }
    }
};
template <bool SPLIT>
struct Probs<float, SPLIT> {
    f32x16 v;
    __device__ __forceinline__ void set(const f32x16& s) { v = s; }
};
// In fp16, for values that are there in fp16, too (wide workgroups over 8-bit codes): within 2^-11 of each at the cost of a
// single bf16 value, but for probabilities below 2^-14, whose step is 2^-24, where the row's largest is 2^6 or more
// (errors of 1.66e-3 of the result, with single bf16 values 2.33e-3; a view over 43,968 slots 266 -> 279 us, 16 ragged
// sequences of up to 400 tokens over 3,000 slots 69 -> 75, for the sums of every block that totals() looks at).
struct HalfProbs {
    f16x8 v[2];
    __device__ __forceinline__ void set(const f32x16& s) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i >> 3][i & 7] = (f16)s[i];
    }
};
__device__ __forceinline__ f32x16 mfma_value(bf16x8 f, bf16x8 p, f32x16 c) { return mfma_bf16(f, p, c); }
__device__ __forceinline__ f32x16 mfma_value(bf16x8 f, f16x8 p, f32x16 c) {
    return mfma_f16(__builtin_bit_cast(f16x8, f), p, c);
}

// Logits (without the scale) of the block whose K lies at `k`.
template <typename T>
__device__ __forceinline__ f32x16 block_logits(const Rows<T>& w, lds_char* k, int lane) {
    const int l31 = lane & 31, hh = lane >> 5;
    f32x16 s = zero_f32x16();
    if constexpr (Rows<T>::kBf) {
        typedef __attribute__((address_space(3))) const bf16x8 lds_frag;
        const int row = swap23(l31);
        const int a0 = row * 128 + ((hh ^ ((row >> 1) & 7)) << 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) s = mfma_bf16(*(lds_frag*)(k + (a0 ^ (i << 5))), w.qb[i], s);
    } else {
        typedef __attribute__((address_space(3))) const f32x4 lds_frag;
        const int a0 = l31 * 256 + ((hh ^ (l31 & 15)) << 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x4 f = *(lds_frag*)(k + (a0 ^ (i << 5)));
#pragma unroll
            for (int e = 0; e < 4; ++e) s = mfma_f32(f[e], w.qf[4 * i + e], s);
        }
    }
    return s;
}

// Slots that a row does not see: logits of -inf.  `units`: which of the two groups of 16 slots exist.
template <typename T>
__device__ __forceinline__ void block_mask(const Rows<T>& w, int k0, uint32_t units, int lane, f32x16& s) {
    typedef Geo<T, true> G;
    // (compared with constants: the slots' numbers, which the lane half shifts, would otherwise
    // stay in registers through the loop over the tiles)
    const int left = w.vis - k0 - G::key(0, 1) * (lane >> 5);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int k = G::key(r, 0);
        s[r] = k < left && ((units >> (k >> 4)) & 1) ? s[r] : -INFINITY;
    }
}

// Logits to probabilities and their sum.
__device__ __forceinline__ float block_exp(f32x16& s, float c2, float ref) {
    float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = exp2f_fast(fmaf(s[r], c2, -ref));
        ls[r & 3] += s[r];
    }
    return (ls[0] + ls[1]) + (ls[2] + ls[3]);
}

// The block again, with the reference moved to the maximum so far.
template <typename T, bool SPLIT>
__device__ __forceinline__ float block_move(Rows<T>& w, lds_char* k, float c2, int k0, bool partial,
                                            uint32_t units, int lane, Probs<T, SPLIT>& p) {
    // (read again: the first pass's operands and logits do not stay in registers for this)
    asm volatile("" ::: "memory");
    f32x16 s = block_logits<T>(w, k, lane);
    if (partial) block_mask<T>(w, k0, units, lane, s);
    float top = s[0];
#pragma unroll
    for (int r = 0; r < 16; r += 2) top = maximum(maximum(top, s[r]), s[r + 1]);
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = maximum(__uint_as_float(x[0]), __uint_as_float(x[1])) * c2;
    const float mn = top > w.m ? top : w.m;
    const float f = w.m == mn ? 1.f : exp2f_fast(w.m - mn);   // 0 from -inf
    w.l *= f;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) w.o[m][r] *= f;
    w.m = mn;
    const float sum = block_exp(s, c2, mn == -INFINITY ? 0.f : mn);
    p.set(s);
    return sum;
}

// Transposing read: of 16 lanes, lane i gets column i of the 4 x 16 values whose rows its quads
// address; two of them, four rows (512 bytes) apart, make eight slots of a feature.
__device__ __forceinline__ bf16x8 tr_read(lds_char* a) {
    typedef __attribute__((address_space(3))) s16x4 lds_tr;
    typedef uint32_t u32x2 __attribute__((__vector_size__(8)));
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr*)a));
    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr*)(a + 512)));
    const u32x4 f = {x[0], x[1], y[0], y[1]};
    return __builtin_bit_cast(bf16x8, f);
}

// O^T += V^T P^T of the block whose V lies at `v`.  `rest`: with the second parts of split probabilities
// (which an infinite value would turn into NaN).
__device__ __forceinline__ void block_values(Rows<bf16>& w, lds_char* v, const HalfProbs& p, int lane) {
    const int hh = lane >> 5, i16 = lane & 15, dq = (lane >> 4) & 1;
    const int v0 = (8 * hh + (i16 >> 2)) * 128 + (((2 * dq + ((i16 & 3) >> 1)) ^ (2 * (i16 >> 2))) << 4) + (i16 & 1) * 8;
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int m = 0; m < 2; ++m) w.o[m] = mfma_value(tr_read(v + (v0 ^ (m << 6)) + st * 2048), p.v[st], w.o[m]);
}
template <typename T, bool SPLIT>
__device__ __forceinline__ void block_values(Rows<T>& w, lds_char* v, const Probs<T, SPLIT>& p, bool rest, int lane) {
    const int l31 = lane & 31, hh = lane >> 5;
    if constexpr (Rows<T>::kBf) {
        const int i16 = lane & 15, dq = (lane >> 4) & 1;
        const int v0 = (8 * hh + (i16 >> 2)) * 128 +
                       (((2 * dq + ((i16 & 3) >> 1)) ^ (2 * (i16 >> 2))) << 4) + (i16 & 1) * 8;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const bf16x8 f = tr_read(v + (v0 ^ (m << 6)) + st * 2048);
                w.o[m] = mfma_bf16(f, p.v[st], w.o[m]);
                if (SPLIT && rest) w.o[m] = mfma_bf16(f, p.rest[SPLIT ? st : 0], w.o[m]);
            }
    } else {
        typedef __attribute__((address_space(3))) const float lds_f32;
        lds_char* vt = v + hh * 1024 + l31 * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int m = 0; m < 2; ++m)
                w.o[m] = mfma_f32(*(lds_f32*)(vt + Geo<T, true>::key(r, 0) * 256 + m * 128), p.v[r], w.o[m]);
    }
}

__device__ __forceinline__ f32x16 mfma_planes(const Planes& a, const Planes& b, f32x16 c) {
    c = mfma_bf16(a.m, b.m, c);
    c = mfma_bf16(a.l, b.h, c);
    c = mfma_bf16(a.h, b.l, c);
    c = mfma_bf16(a.m, b.h, c);
    c = mfma_bf16(a.h, b.m, c);
    return mfma_bf16(a.h, b.h, c);
}

// A block's logits and probabilities.
// `logits`: null, or where the row's logits (of slots from 0 on) are kept.
template <typename T, bool SPLIT>
__device__ __forceinline__ void block_probs(Rows<T>& w, lds_char* k, float c2, int k0, bool partial, uint32_t units,
                                            int lane, float* logits, Probs<T, SPLIT>& p) {
    f32x16 s = block_logits<T>(w, k, lane);
    if (partial) block_mask<T>(w, k0, units, lane, s);
    if (logits)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(f32x4*)(logits + k0 + Geo<T, true>::key(4 * g, lane >> 5)) =
                f32x4{s[4 * g], s[4 * g + 1], s[4 * g + 2], s[4 * g + 3]};
    float sum = block_exp(s, c2, w.m);   // inf or NaN while m is -inf
    p.set(s);
    if (__builtin_amdgcn_ballot_w64(!(sum < kMoveAt)))
        sum = block_move<T, SPLIT>(w, k, c2, k0, partial, units, lane, p);
    w.l += sum;
}

// Values of a tile that is seen in part, `rows` slots from slot k of the cache at `v` in LDS, before any
// wave multiplies with them.  Slots from `end` on or on no page may hold anything: cleared.
// Slots that some rows see and others do not may hold infinities or NaN, which a product with a
// probability of 0 would carry into the rows that do not see them: cleared too, and true returned for
// add_odd_values() to give them to their rows.
template <typename T>
__device__ __forceinline__ bool clean_values(lds_char* v, int rows, int k, int end, uint32_t units, int lane) {
    constexpr int kPieces = kD * sizeof(T) / 16;   // per slot
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    bool odd = false;
    for (int c = lane; c < rows * kPieces; c += 64) {
        const int slot = c / kPieces;
        u32x4 x = *(lds_u32x4*)(v + c * 16);
        const bool live = k + slot < end && ((units >> (slot >> 4)) & 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) {
                const bool lo = (x[j] & 0x7f80u) == 0x7f80u, hi = (x[j] & 0x7f800000u) == 0x7f800000u;
                odd = odd || (live && (lo || hi));
                x[j] = !live ? 0u : x[j] & (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0xffffu : 0xffffffffu);
            } else {
                const bool inf = (x[j] & 0x7f800000u) == 0x7f800000u;
                odd = odd || (live && inf);
                x[j] = live && !inf ? x[j] : 0u;
            }
        }
        *(lds_u32x4*)(v + c * 16) = x;
    }
    const bool any = __builtin_amdgcn_ballot_w64(odd) != 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    return any;
}

// Values that are not finite in slots [k0, k1) of a tile seen in part, which clean_values() took
// out, for the rows that see them.  Rare: slot by slot from memory, logits by plain sums, few loads
// at a time (this must not set the kernel's register count).
template <typename T, int CODE>
__device__ __forceinline__ void add_odd_values(const AttendArgs& a, Rows<T>& w, int b, int hk, int k0, int k1,
                                               int lane) {
    const int hh = lane >> 5;
#pragma unroll 1
    for (int k = k0; k < k1; ++k) {
        const int page = a.c.table[(int64_t)b * a.c.max_pages + (k >> a.c.page_log2)];
        if (page < 0 || page >= a.c.npages) continue;
        const int64_t at = ((((int64_t)page * a.c.Hkv + hk) << a.c.page_log2) +
                            (k & ((1 << a.c.page_log2) - 1))) * kD;
        const T *kr = (const T*)a.c.K + at, *vr = (const T*)a.c.V + at;
        float x = 0.f, vs = 0.f;
        if constexpr (CODE != CODE_NONE) {
            const uint32_t sc = a.c.scale[at / kD];
            vs = value_scale(sc);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f[4];
                values4<CODE>(*(const uint32_t*)((const char*)a.c.K + at + 16 * (i >> 1) + 8 * hh + 4 * (i & 1)), key_scale(sc), f);
#pragma unroll
                for (int e = 0; e < 4; ++e) x = fmaf((float)(T)f[e], (float)w.qb[i >> 1][4 * (i & 1) + e], x);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else if constexpr (Rows<T>::kBf) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 kv = load_bf16x8((const bf16*)kr + 16 * i + 8 * hh);
#pragma unroll
                for (int j = 0; j < 8; ++j) x = fmaf((float)kv[j], (float)w.qb[i][j], x);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x4 kv = *(const f32x4*)(kr + 8 * i + 4 * hh);
#pragma unroll
                for (int e = 0; e < 4; ++e) x = fmaf(kv[e], w.qf[4 * i + e], x);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        x += __shfl_xor(x, 32);
        const float p = exp2f_fast(fmaf(x, a.c2, -w.m));
        const bool sees = k < w.vis;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float f[4];
                if constexpr (CODE != CODE_NONE)
                    values4<CODE>(*(const uint32_t*)((const char*)a.c.V + at + 32 * m + 8 * g + 4 * hh), vs, f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v;
                    if constexpr (CODE != CODE_NONE) v = (float)(T)f[e];
                    else v = (float)vr[32 * m + 8 * g + 4 * hh + e];
                    if (sees && !(fabsf(v) <= 3.4028235e38f)) w.o[m][4 * g + e] += p * v;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// A workgroup: RT rows of one key head and sequence over one range of its slots.  Narrow: bound by HBM
// (tokens over 137,400 and 62,724 slots of 16 heads, bf16: 167 us, 4.9 TB/s).  Wide: by the issue of matrix and vector
// instructions together, a fused product, a power, a sum and half a rounding per logit (1,374 tokens over 43,968 slots of
// 16 heads, bf16: 260 us, 950 TFLOP/s, the SIMDs' cycles 58 % in vector instructions and 43 % in MFMAs;
// kernel alone, after some 40 passes: the first ones run at lower clocks, 280-350.  fp32, three prompts of
// 8.6 GFLOP: 63 us).
//
// CODE: K and V are 8-bit codes (wide bf16 rows only).  Tiles lie in LDS as bf16 ones do, K as bf16 values, V as fp16 ones; they come
// through registers: a wave loads a tile's 16 slots two tiles ahead and writes them, decoded, one ahead.
template <typename T, bool WIDE, int CODE>
__global__ __launch_bounds__((64 * GeoOf<T, WIDE, CODE>::NW), 2) void k_cache_attend(AttendArgs a) {
    typedef GeoOf<T, WIDE, CODE> G;
    constexpr bool kCode = CODE != CODE_NONE;
    constexpr bool kSplit = G::kSplit || kCode;                                 // where references may move
    typedef std::conditional_t<kCode, HalfProbs, Probs<T, G::kSplit>> WideP;    // where they stay
    constexpr float kLift = kCode ? 10.f : 0.f;    // probabilities of a row's first block are 2^kLift at most
    static_assert(!kCode || (WIDE && G::kBf), "codes: wide bf16 rows");
    __shared__ __attribute__((aligned(1024))) char smem[G::kLds];
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // The row tiles of one key head and slot range read the same keys and values: they go to
    // one XCD (workgroup i runs on XCD i % 8).  Ranges come in the order of their start, so that
    // those past the end of short sequences, which have nothing to do, come last and in a row, and
    // each turns the heads by five, so that no sequence meets the same XCD and shader engine every time
    // (ranges of a head one after the other: 32 ragged sequences, 8 ranges, 49 us; so: 31).
    const int heads = a.c.B * a.c.Hkv;
    int turn = (blockIdx.x >> 3) / a.row_tiles, rt = (blockIdx.x >> 3) - turn * a.row_tiles;
    int x = turn * 8 + (blockIdx.x & 7), split = x / heads, y = (x - split * heads + 5 * split) % heads;
    if constexpr (kCode) {
        // Codes, one workgroup per compute unit: a row tile of everything before the next, so that the last one, which may
        // have few rows, comes last; and all ranges of a sequence one after the other, as the compute units that an
        // XCD's workgroups go to follow from their numbers (with those of a long sequence always every fourth, 149 us
        // for 82), turned by three from tile to tile.  Ragged, 16 heads: six sequences of up to 700 tokens over 20,000 slots, four
        // key heads, 135 us, in the order of the other caches 170; 16 of up to 400 over 3,000, 16 key heads, 75 and 92.
        const int turns = (heads * a.nsplit + 7) >> 3;
        rt = (blockIdx.x >> 3) / turns;
        x = ((blockIdx.x >> 3) - rt * turns + 3 * rt) % turns * 8 + (blockIdx.x & 7);
        const int per = a.c.Hkv * a.nsplit, b8 = x / per;
        split = x < heads * a.nsplit ? (x - b8 * per) / a.c.Hkv : a.nsplit;
        y = b8 * a.c.Hkv + (x - b8 * per) % a.c.Hkv;
    }
    if (split >= a.nsplit) return;
    const int hk = y % a.c.Hkv, b = y / a.c.Hkv;

    const CacheSeq sq = cache_seq(a.c, b);
    const int nrows = sq.nq * a.G;
    if (rt * G::RT >= nrows) return;
    // A tile of few rows: one group of rows for each of four waves (a SIMD each), the other sees nothing.  (The 16 sequences
    // above 82 -> 75 us.  200 rows as seven waves' groups, two waves a SIMD: 37 -> 44.)
    const bool slim = kCode && nrows - rt * G::RT <= 16 * G::NW;
    const int wave_rows = slim ? 32 : 32 * G::NB, row0 = rt * G::RT + (WIDE ? wave * wave_rows : 0);
    const int tile_last = rt * G::RT + G::RT - 1 < nrows ? rt * G::RT + G::RT - 1 : nrows - 1;
    const int klim = cache_visible(sq, a.causal, tile_last / a.G);
    const int c0 = split * a.chunk, c1 = c0 + a.chunk < klim ? c0 + a.chunk : klim;
    if (split > 0 && c0 >= klim) return;

    // ---- this wave's rows
    Rows<T> w[G::NB];
    const bool alive = row0 < nrows;
    int64_t orow[G::NB];   // row of O
    const T* qrow[G::NB];
#pragma unroll
    for (int nb = 0; nb < G::NB; ++nb) {
        int r = row0 + 32 * nb + l31;
        r = r < nrows ? r : nrows - 1;
        const int i = r / a.G, head = hk * a.G + r - i * a.G;
        w[nb].vis = kCode && nb && slim ? 0 : cache_visible(sq, a.causal, i);
        w[nb].m = -INFINITY;
        w[nb].l = 0.f;
        w[nb].o[0] = w[nb].o[1] = zero_f32x16();
        orow[nb] = (int64_t)(sq.q0 + i) * a.Hq + head;
        qrow[nb] = (const T*)a.Q + (int64_t)(sq.q0 + i) * a.q_stride + head * kD;
    }
    auto load_q = [&]() {
#pragma unroll
        for (int nb = 0; nb < G::NB; ++nb) {
            if constexpr (G::kBf) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[nb].qb[k] = load_bf16x8(qrow[nb] + 16 * k + 8 * hh);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const f32x4 v = *(const f32x4*)(qrow[nb] + 8 * k + 4 * hh);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[nb].qf[4 * k + e] = v[e];
                }
            }
        }
    };
    if constexpr (!WIDE || G::kBf) load_q();
    const int wave_last = row0 + wave_rows - 1 < nrows ? row0 + wave_rows - 1 : nrows - 1;
    const int wlim = alive ? cache_visible(sq, a.causal, wave_last / a.G) : 0;
    // slots of this range that every row of the workgroup sees
    const int all = cache_visible(sq, a.causal, rt * G::RT / a.G), seen_by_all = all < c1 ? all : c1;

    // ---- the tiles
    const int nt_all = (c1 - c0 + G::TK - 1) / G::TK;
    const int tstep = WIDE ? 1 : 4, tfirst = WIDE ? 0 : wave;
    const int nt = nt_all > tfirst ? (nt_all - tfirst + tstep - 1) / tstep : 0;
    if (nt > 0) {
        PageWindow pw;
        pw.start(a.c, b, c0, c1 - 1, lane);
        const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem + (WIDE ? 0 : wave * G::kRing);
        lds_char* ring = (lds_char*)smem + (WIDE ? 0 : wave * G::kRing);
        const int page_mask = (1 << a.c.page_log2) - 1;
        const int last_unit = (c1 - 1) & ~15;
        // Per lane: byte within a 1 KB copy.  K's and V's 16-byte pieces are exchanged within
        // their row so that the tile's readers meet no bank twice (64 banks: two bf16 rows): K's piece p of
        // slot s lies at p ^ (s / 2 & 7) (bf16) or p ^ (s & 15) (fp32), V's at p ^ 2 (s & 3) (bf16).
        uint32_t kv, vv;
        if constexpr (G::kBf) {
            const int r = lane >> 3, pc = lane & 7;
            kv = r * 128 + ((pc ^ (r >> 1)) << 4);
            vv = r * 128 + ((pc ^ (2 * (r & 3))) << 4);
        } else {
            const int r = lane >> 4, pc = lane & 15;
            kv = r * 256 + ((pc ^ r) << 4);
            vv = lane * 16;
        }
        // 16 slots of a tile: their first one, its page, and the copies of their K or V.
        auto unit_slot = [&](int t, int unit) {
            const int slot = c0 + (tfirst + t * tstep) * G::TK + 16 * unit;
            return slot < last_unit ? slot : last_unit;
        };
        auto unit_page = [&](int t, int unit) { return pw.page(unit_slot(t, unit) >> a.c.page_log2, lane); };
        auto issue_unit = [&](int t, int unit, bool isv, int id) {
            const int64_t at = ((((int64_t)id * a.c.Hkv + hk) << a.c.page_log2) + (unit_slot(t, unit) & page_mask)) * G::ROWB;
            const char* src = (const char*)(isv ? a.c.V : a.c.K) + at;
            const uint32_t dst = lds0 + (t % G::NST) * G::kTile + (isv ? G::TK * G::ROWB : 0) + unit * 16 * G::ROWB;
#pragma unroll
            for (int u = 0; u < G::UC; ++u)
                copy_to_lds(dst + u * 1024, src + u * 1024, isv ? vv : kv ^ (64 * u));
        };
        auto issue = [&](int t) {
#pragma unroll
            for (int j = 0; j < G::PPW; ++j) {
                const int part = WIDE ? wave * G::PPW + j : j, unit = part >> 1;
                issue_unit(t, unit, part & 1, unit_page(t, unit));
            }
        };
        bool odd = false;
        // Codes: waves 0 .. 3 decode 16 slots of a tile's K each, waves 4 .. 7 of its V, a lane 16 features.
        // K as bf16 values.  V, while `halves`, in fp16 and 2^-vexp of itself, where a slot's scale is 2^-kDown (e4m3's least code is
        // 2^-9, fp16's least number 2^-24) to 2^kUp times 2^vexp (2^6 448, and up to twice that with a scale that is no power of two,
        // lies below 65,504).  Elsewhere (`far` past kUp + kDown) the range is done again over bf16 values.
        constexpr int kUp = 6, kDown = 15;
        __shared__ int s_range[kCode ? 2 * G::NW : 1];   // per wave: far + 1, 31 - what its rows allow for it
        u32x4 codes;
        uint32_t sc = 0;
        const bool isv = wave >= 4;
        const int cr = lane >> 2, cp = 2 * (lane & 3);   // slot of the 16, first of two 16-byte pieces
        const char* cbase = nullptr;
        uint32_t cput[2];
        bool halves = kCode;
        int vexp = 0;
        int far = -1;                                    // largest scale of V so far: 2^(far - kDown + vexp)
        if constexpr (kCode) {
            cbase = (const char*)(isv ? a.c.V : a.c.K) + (lane & 3) * 16;
            const int row = 16 * (wave & 3) + cr;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                cput[i] = row * 128 + (isv ? G::kTileV + (((cp + i) ^ (2 * (row & 3))) << 4) : ((cp + i) ^ ((row >> 1) & 7)) << 4);
        }
        auto fetch_codes = [&](int t) {
            const int k = unit_slot(t, wave & 3);
            const int64_t at = (((int64_t)pw.page(k >> a.c.page_log2, lane) * a.c.Hkv + hk) << a.c.page_log2) + (k & page_mask) + cr;
            codes = *(const u32x4*)(cbase + at * kD);
            sc = a.c.scale[at];
        };
        // 2^vexp: 8 times the first tile's largest finite scale of V, so that later ones may be 2^9 times as large, or 2^-12.
        auto first_scale = [&]() {
            int id = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int p = unit_page(0, u);
                if (lane >> 4 == u) id = p;
            }
            const int k = c0 + lane < c1 ? c0 + lane : c1 - 1;
            // (slots past the end: the last one; a unit past the last one has its page)
            const int64_t at = (((int64_t)id * a.c.Hkv + hk) << a.c.page_log2) + (k & page_mask);
            const int e = (int)(a.c.scale[at] >> 23 & 255u);
            vexp = top_of_wave<8>(e < 255 ? e : 0) - 127 + 3;
        };
        auto put_codes = [&](int t) {
            u32x4 v[2];
            const int k0 = c0 + t * G::TK, slot = k0 + 16 * (wave & 3);
            if (isv) {
                // Slots past the end or on no page may hold anything: zeros.
                const bool part = !pw.sane || k0 + G::TK > seen_by_all;
                if (part) {
                    const int at = slot >> a.c.page_log2;
                    const bool live = slot + cr < c1 && (pw.sane || (at <= pw.last && pw.valid(pw.row[at])));
                    if (!live) codes = u32x4{0u, 0u, 0u, 0u}, sc = 0u;
                }
                if (halves) {
                    const float f = __builtin_amdgcn_ldexpf(value_scale(sc), -vexp);
                    const int d = (int)(sc >> 23) - (127 + vexp - kDown);   // (a negative scale: past kUp)
                    if (__builtin_amdgcn_ballot_w64((uint32_t)d > kUp + kDown || (CODE == CODE_E4M3 && (sc & 0x7f0000u)))) {
                        uint32_t any = (codes[0] | codes[1]) | (codes[2] | codes[3]);
                        if (CODE == CODE_E4M3) any &= 0x7f7f7f7fu;
                        const int e = (int)(sc >> 23 & 255u), de = e - (127 + vexp - kDown);
                        if (any && e != 255) far = max(far, (uint32_t)de <= kUp + kDown ? de : kUp + kDown + 1);
                        decode16_half<CODE, false>(codes, f, v);
                    } else {
                        far = max(far, d);
                        decode16_half<CODE, true>(codes, f, v);
                    }
                } else {
                    decode16<CODE>(codes, value_scale(sc), v);
                }
                if (part) {   // (as clean_values() does to tiles that are copied)
                    const uint32_t inf = halves ? 0x7c00u : 0x7f80u;
                    bool any = false;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t x = v[i][j];
                            const bool lo = (x & inf) == inf, hi = (x & inf << 16) == inf << 16;
                            any = any || lo || hi;
                            v[i][j] = x & (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0xffffu : 0xffffffffu);
                        }
                    odd |= __builtin_amdgcn_ballot_w64(any) != 0;
                }
            } else {
                decode16<CODE>(codes, key_scale(sc), v);
            }
            typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
            lds_char* tile = ring + (t % G::NST) * G::kTile;
#pragma unroll
            for (int i = 0; i < 2; ++i) *(lds_u32x4*)(tile + cput[i]) = v[i];
        };
        auto issue_first = [&]() {
            if constexpr (kCode) {
                fetch_codes(0);
                if (halves) first_scale();
                put_codes(0);
                if (nt > 1) fetch_codes(1);
            } else {
#pragma unroll
                for (int t = 0; t < G::AHEAD; ++t)
                    if (t < nt) issue(t);
            }
        };
        if constexpr (!WIDE || G::kBf) issue_first();
        // Groups of 16 slots of the tile at k0 that exist (all, unless the table is wrong).
        auto groups = [&](int k0) {
            uint32_t units = ~0u;
            if (!pw.sane) {
                units = 0;
#pragma unroll
                for (int u = 0; u < G::TK / 16; ++u) {
                    const int at = (k0 + 16 * u) >> a.c.page_log2;
                    if (at <= pw.last && pw.valid(pw.row[at])) units |= 1u << u;
                }
            }
            return units;
        };
        // Tile t has come: its copies, and where it is seen in part its values are cleaned by the wave
        // that copied them.  Then (wide) all waves are past the tile whose place the next copies take.
        auto arrive = [&](int t) {
            if constexpr (kCode) {
                // (this wave's part of tile t is written; after the barrier all are, and no wave is at work on a
                // tile before t - 1, so the next one's place is free)
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                if (t + 1 < nt) {
                    put_codes(t + 1);
                    if (t + 2 < nt) fetch_codes(t + 2);
                }
                return;
            }
            const int more = nt - 1 - t, k0 = c0 + (tfirst + t * tstep) * G::TK;
            lds_char* tile = ring + (t % G::NST) * G::kTile;
            if constexpr (WIDE) {
                wait_tiles<G::CPT>(more < G::AHEAD - 1 ? more : G::AHEAD - 1);
            } else {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile before is read
                if (t + G::AHEAD < nt) issue(t + G::AHEAD);
                wait_tiles<G::CPT>(more < G::AHEAD ? more : G::AHEAD);
            }
            if (!pw.sane || k0 + G::TK > seen_by_all) {
                const uint32_t units = groups(k0);
                if constexpr (WIDE) {
                    // (a wave copies 16 slots, or K or V of them)
                    const int u = 16 * (wave * G::PPW >> 1);
                    if (G::PPW == 2 || (wave & 1))
                        odd |= clean_values<T>(tile + G::kTileV + u * G::ROWB, 16, k0 + u, c1, units >> (u >> 4), lane);
                } else
                    odd |= clean_values<T>(tile + G::kTileV, G::TK, k0, c1, units, lane);
            }
            if constexpr (WIDE) {
                __builtin_amdgcn_s_barrier();
                if (t + G::AHEAD < nt) issue(t + G::AHEAD);
            }
        };
        auto tile_at = [&](int t) { return ring + (t % G::NST) * G::kTile; };
        float* logits = nullptr;
        if (!WIDE && a.logits && row0 + l31 < nrows) logits = a.logits + orow[0] * a.logit_stride;
        // Every block with its bound on the reference checked.
        auto careful = [&](bool rest) {
            for (int t = 0; t < nt; ++t) {
                const int k0 = c0 + (tfirst + t * tstep) * G::TK;
                lds_char* tile = tile_at(t);
                arrive(t);
                const bool partial = !pw.sane || k0 + G::TK > seen_by_all;
                const uint32_t units = partial ? groups(k0) : 0;
                if (k0 < wlim)
#pragma unroll 1
                    for (int j = 0; j < G::TK / 32; ++j)
#pragma unroll
                        for (int nb = 0; nb < G::NB; ++nb) {
                            Probs<T, kSplit> p;
                            block_probs<T, kSplit>(w[nb], tile + j * G::kBlock, a.c2, k0 + 32 * j, partial, units >> (2 * j),
                                           lane, logits, p);
                            block_values<T, kSplit>(w[nb], tile + G::kTileV + j * G::kBlock, p, rest, lane);
                        }
            }
        };
        // Values so large that their sums left fp32's range, or infinite: once more, with a reference that is known
        // now, a row's log-sum-exp and one: its probabilities sum to 1/2, so no sum passes the largest value.
        auto overflown = [&]() {
            float top = 0.f;
#pragma unroll
            for (int nb = 0; nb < G::NB; ++nb)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = maximum(maximum(top, fabsf(w[nb].o[0][r])), fabsf(w[nb].o[1][r]));
            return alive && __builtin_amdgcn_ballot_w64(!(top <= 3.4028235e38f)) != 0;
        };
        auto restart = [&](bool known) {
#pragma unroll
            for (int nb = 0; nb < G::NB; ++nb) {
                Rows<T>& x = w[nb];
                const float l = x.l + __shfl_xor(x.l, 32), m = x.m + __log2f(l) + 1.f;
                x.m = known && fabsf(m) <= 3.4028235e38f ? m : -INFINITY;   // (no logits, or not finite: as ever)
                x.l = 0.f;
                x.o[0] = x.o[1] = zero_f32x16();
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            pw.start(a.c, b, c0, c1 - 1, lane);
        };
        bool redo = false;
        if constexpr (WIDE && G::kBf) {
            // The reference stays that of the first block.  While block j's probabilities are formed, block
            // j + 1's logits and block j - 1's values are multiplied: matrix and vector
            // instructions without a dependence or a branch between them.  Should a row's sum or
            // result leave fp32's range with it (its logits grew by more than 41 over the first block's, its
            // first block had none, or values are huge), the workgroup does its range again carefully.
            const int tfull = pw.sane ? (seen_by_all - c0) / G::TK : 0;   // tiles all rows see
            f32x16 s0[G::NB], s1[G::NB];
            WideP p0[G::NB], p1[G::NB];
            float ref[G::NB], sum[G::NB][4] = {};
            // Half a tile: eight operands from LDS, each for the MFMAs of the row groups and followed by the
            // vector instructions of two of a group's 16 logits; they are read three ahead.  The first three are values, of a tile
            // that has been there for long: they are read before the barrier that K waits for.
            bf16x8 ahead[3];
            auto value_at = [&](lds_char* v, int i) {
                const int i16 = lane & 15, dq = (lane >> 4) & 1;
                const int v0 = (8 * hh + (i16 >> 2)) * 128 +
                               (((2 * dq + ((i16 & 3) >> 1)) ^ (2 * (i16 >> 2))) << 4) + (i16 & 1) * 8;
                return tr_read(v + (v0 ^ ((i & 1) << 6)) + (i >> 1) * 2048);
            };
            auto key_at = [&](lds_char* k, int i) {
                typedef __attribute__((address_space(3))) const bf16x8 lds_frag;
                const int row = swap23(l31);
                const int a0 = row * 128 + ((hh ^ ((row >> 1) & 7)) << 4);
                return *(lds_frag*)(k + (a0 ^ (i << 5)));
            };
            typedef f32x16 Logits[G::NB];
            typedef WideP BlockP[G::NB];
            typedef std::conditional_t<kCode, f16, bf16> P16;
            // Codes: a block's sums into l, and where one comes near fp16's largest value, references raised so that it is 2^kLift.
            // (s: the block's powers still.)
            auto totals = [&](auto width, float (&tot)[G::NB]) __attribute__((always_inline)) {
                constexpr int NB = decltype(width)::value;
                float top = 0.f;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    tot[nb] = (sum[nb][0] + sum[nb][1]) + (sum[nb][2] + sum[nb][3]);
                    w[nb].l += tot[nb];
                    top = maximum(top, tot[nb]);
                }
                return __builtin_amdgcn_ballot_w64(!(top < 65504.f)) != 0;
            };
            auto raise = [&](auto width, Logits& s, const float (&tot)[G::NB], BlockP& p) __attribute__((always_inline)) {
                constexpr int NB = decltype(width)::value;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float both = maximum(tot[nb], __shfl_xor(tot[nb], 32));
                    int k = (int)(__float_as_uint(both) >> 23) - 127 - (int)kLift;
                    k = k > 0 && k < 120 ? k : 0;   // (further, or no number: seen by l in the end)
                    const float f = __uint_as_float((uint32_t)(127 - k) << 23);
                    w[nb].l *= f;
                    w[nb].m += (float)k;
                    ref[nb] += (float)k;
#pragma unroll
                    for (int r = 0; r < 16; ++r) w[nb].o[0][r] *= f, w[nb].o[1][r] *= f, s[nb][r] *= f;
                    p[nb].set(s[nb]);
                }
            };
            auto half = [&](auto mask, auto width, Logits& s, int k0, Logits& sn, lds_char* k, lds_char* v, lds_char* v_next,
                            const BlockP& pv, BlockP& pn) __attribute__((always_inline)) {
                constexpr int NB = decltype(width)::value;
                if constexpr (decltype(mask)::value)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) block_mask<T>(w[nb], k0, ~0u, lane, s[nb]);
                constexpr int kOf[8] = {4, 5, 6, 0, 1, 2, 3, 7};   // 0-3: logits, 4-7: values
                bf16x8 f[8] = {ahead[0], ahead[1], ahead[2]};
                // Two logits at a time, in three steps an MFMA apart so that none waits for the last:
                // the exponent, its power, the sum and the rounding.
                auto exponent = [&](int u) {
#pragma unroll
                    for (int r = 2 * (u / NB); r < 2 * (u / NB) + 2; ++r)
                        s[u % NB][r] = fmaf(s[u % NB][r], a.c2, -ref[u % NB]);
                };
                auto add = [&](int u) {
                    const int nb = u % NB, i = u / NB;
                    if (kCode && i < 2) {
                        sum[nb][2 * i] = s[nb][2 * i];
                        sum[nb][2 * i + 1] = s[nb][2 * i + 1];
                    } else {
                        sum[nb][(2 * i) & 3] += s[nb][2 * i];
                        sum[nb][(2 * i + 1) & 3] += s[nb][2 * i + 1];
                    }
                    pn[nb].v[i >> 2][(2 * i) & 7] = (P16)s[nb][2 * i];
                    pn[nb].v[i >> 2][(2 * i + 1) & 7] = (P16)s[nb][2 * i + 1];
                };
                auto power = [&](int u) {
                    const int nb = u % NB, i = u / NB;
                    s[nb][2 * i] = exp2f_fast(s[nb][2 * i]);
                    s[nb][2 * i + 1] = exp2f_fast(s[nb][2 * i + 1]);
                };
                // Units (two logits) whose powers come before slot u of the 8 NB: one each; codes: all before the last, whose MFMA hides
                // a part of the totals.
                constexpr int kSlots = 8 * NB, kBusy = kCode ? kSlots - 1 : kSlots;
                auto units = [](int u) { return u >= kBusy ? kSlots : (u * kSlots + kBusy - 1) / kBusy; };
                float tot[G::NB];
                bool near = false;
#pragma unroll
                for (int u = 0; u < units(1); ++u) exponent(u);
#pragma unroll
                for (int u = 0; u < kSlots; ++u) {
                    const int i = u / NB, nb = u % NB, n = kOf[i];
                    if (nb == 0) {
                        if (i < 5) f[i + 3] = kOf[i + 3] < 4 ? key_at(k, kOf[i + 3]) : value_at(v, kOf[i + 3] - 4);
                        else ahead[i - 5] = value_at(v_next, i - 5);
                    }
                    Rows<T>& x = w[nb];
                    if (n < 4) sn[nb] = mfma_bf16(f[i], x.qb[n], n ? sn[nb] : zero_f32x16());
                    else x.o[n & 1] = mfma_value(f[i], pv[nb].v[(n - 4) >> 1], x.o[n & 1]);
#pragma unroll
                    for (int a = units(u + 1); a < units(u + 2); ++a) exponent(a);
#pragma unroll
                    for (int a = units(u); a < units(u + 1); ++a) power(a);
#pragma unroll
                    for (int a = u > 0 ? units(u - 1) : 0; a < units(u); ++a) add(a);
                    if (kCode && u == kSlots - 1) near = totals(width, tot);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (kCode) {
                    if (__builtin_expect(near, 0)) raise(width, s, tot, pn);
                } else {
                    add(kSlots - 1);
                }
            };
            auto probs = [&](Logits& s, int k0, BlockP& p) __attribute__((always_inline)) {
#pragma unroll
                for (int nb = 0; nb < G::NB; ++nb) {
                    block_mask<T>(w[nb], k0, ~0u, lane, s[nb]);
                    if (kCode)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum[nb][j] = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[nb][r] = exp2f_fast(fmaf(s[nb][r], a.c2, -ref[nb]));
                        sum[nb][r & 3] += s[nb][r];
                    }
                    p[nb].set(s[nb]);
                }
                if constexpr (kCode) {
                    const std::integral_constant<int, G::NB> width;
                    float tot[G::NB];
                    if (__builtin_expect(totals(width, tot), 0)) raise(width, s, tot, p);
                }
            };
            auto body = [&](auto mask, auto width, int t) __attribute__((always_inline)) {   // second block of tile t, first of tile t + 1
                lds_char *cur = tile_at(t), *next = tile_at(t + 1);
                const int k0 = c0 + t * G::TK;
                half(mask, width, s1, k0 + 32, s0, next, cur + G::kTileV, cur + G::kTileV + G::kBlock, p0, p1);
                half(mask, width, s0, k0 + 64, s1, next + G::kBlock, cur + G::kTileV + G::kBlock, next + G::kTileV, p1, p0);
            };
            arrive(0);
            if (alive && pw.sane) {
#pragma unroll
                for (int nb = 0; nb < G::NB; ++nb) {
                    f32x16& s = s0[nb];
                    s = block_logits<T>(w[nb], tile_at(0), lane);
                    block_mask<T>(w[nb], c0, ~0u, lane, s);
                    float top = s[0];
#pragma unroll
                    for (int r = 0; r < 16; r += 2) top = maximum(maximum(top, s[r]), s[r + 1]);
                    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false,
                                                                    false);
                    w[nb].m = maximum(__uint_as_float(x[0]), __uint_as_float(x[1])) * a.c2 - kLift;
                    ref[nb] = w[nb].m == -INFINITY ? 0.f : w[nb].m;
                    s1[nb] = block_logits<T>(w[nb], tile_at(0) + G::kBlock, lane);
                }
                probs(s0, c0, p0);
#pragma unroll
                for (int i = 0; i < 3; ++i) ahead[i] = value_at(tile_at(0) + G::kTileV, i);
                int t = 0;
                typedef std::integral_constant<int, G::NB> All;
                if (kCode && slim)
                    for (; t + 1 < nt; ++t) {
                        arrive(t + 1);
                        body(std::true_type(), std::integral_constant<int, 1>(), t);
                    }
                for (; t + 1 < nt && t + 1 < tfull; ++t) {
                    arrive(t + 1);
                    body(std::false_type(), All(), t);
                }
                for (; t + 1 < nt; ++t) {
                    arrive(t + 1);
                    body(std::true_type(), All(), t);
                }
                if constexpr (kCode) {   // (block by block: a reference that rises takes the results so far along)
#pragma unroll
                    for (int nb = 0; nb < G::NB; ++nb)
                        if (!(nb && slim)) block_values(w[nb], tile_at(t) + G::kTileV, p0[nb], lane);
                    probs(s1, c0 + t * G::TK + 32, p1);
#pragma unroll
                    for (int nb = 0; nb < G::NB; ++nb)
                        if (!(nb && slim)) block_values(w[nb], tile_at(t) + G::kTileV + G::kBlock, p1[nb], lane);
                } else {
                    probs(s1, c0 + t * G::TK + 32, p1);
#pragma unroll
                    for (int nb = 0; nb < G::NB; ++nb) {
                        block_values<T, G::kSplit>(w[nb], tile_at(t) + G::kTileV, p0[nb], false, lane);
                        block_values<T, G::kSplit>(w[nb], tile_at(t) + G::kTileV + G::kBlock, p1[nb], false, lane);
                        w[nb].l = (sum[nb][0] + sum[nb][1]) + (sum[nb][2] + sum[nb][3]);
                    }
                }
            } else {
                for (int t = 1; t < nt; ++t) arrive(t);
            }
            if constexpr (kCode) {
                // What fp16's range does not hold is done again.  Scales out of their bounds.  Results or sums past fp32's range, rows
                // whose first logits were -inf alone.  Probabilities below 2^-14 are off by 2^-25 at most: n slots together by no
                // more than 2^-8 of a row's largest result (each apart, of as much / sqrt(n)), if that is 2^-17 n times the largest value.
                // A first slot without values of its own may so have 98 % of the weight of 9,000 slots.
                int room = 31;   // largest `far` that the rows allow
                if (alive)
#pragma unroll
                    for (int nb = 0; nb < G::NB; ++nb) {
                        const int n = (w[nb].vis < c1 ? w[nb].vis : c1) - c0;
                        float top = 0.f;
#pragma unroll
                        for (int r = 0; r < 16; ++r) top = maximum(maximum(top, fabsf(w[nb].o[0][r])), fabsf(w[nb].o[1][r]));
                        top = maximum(top, __shfl_xor(top, 32));
                        const float q = top / ((float)n * (CODE == CODE_E4M3 ? 448.f : 128.f) * 0x1p-17f);
                        int here = max(-1, kDown - 127 + (int)(__float_as_uint(q) >> 23));
                        if (!(__builtin_amdgcn_ldexpf(top, vexp) <= 3.4028235e38f)) here = -2;
                        if (n > 0) room = min(room, here);
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            w[nb].o[0][r] = __builtin_amdgcn_ldexpf(w[nb].o[0][r], vexp);
                            w[nb].o[1][r] = __builtin_amdgcn_ldexpf(w[nb].o[1][r], vexp);
                        }
                    }
                const int f = top_of_wave<5>(far + 1), l = top_of_wave<6>(31 - room);
                if (lane == 0) s_range[wave] = f, s_range[G::NW + wave] = l;
                halves = false;
            }
        } else if constexpr (WIDE) {
            // fp32: six bf16 MFMAs for every eight fp32 ones, of which each takes 16 times its share.  K and
            // V are split once per workgroup on their way into LDS; reference and fallback (fp32
            // MFMAs) as above.
            const int slot8 = tid >> 3, pc = tid & 7;   // this thread's eight features of a slot
            f32x4 kr[2], vr[2];
            // The matrix units take bf16 values below 2^-126 as 0.  What keys and queries lose by it shows
            // if any of them, 0 aside, lies below 2^-103; what probabilities and values lose is at
            // most 2^-125 of the largest value per slot and of l, and may not reach 2^-24 of a
            // result.  Otherwise the range is done again, too.
            uint32_t kq_min = ~0u, v_max = 0;   // twice the bits (less one: 0 comes last)
            auto fetch = [&](int t) {
                const int k0 = c0 + t * 32;
                int unit = k0 + 16 * (wave >> 1);   // (a wave's eight slots lie on one page)
                unit = unit < last_unit ? unit : last_unit;
                const int id = pw.page(unit >> a.c.page_log2, lane);
                const int64_t at = ((((int64_t)id * a.c.Hkv + hk) << a.c.page_log2) + (unit & page_mask) +
                                    (slot8 & 15)) * kD + pc * 8;
                const float *kp = (const float*)a.c.K + at, *vp_ = (const float*)a.c.V + at;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    kr[e] = *(const f32x4*)(kp + 4 * e);
                    vr[e] = *(const f32x4*)(vp_ + 4 * e);
                }
            };
            auto put = [&](int t) {
                char* buf = smem + (t & 1) * G::kPlanes;
                const bool live = c0 + t * 32 + slot8 < c1;   // (others may hold anything)
                float x[8];
                uint32_t least = ~0u;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = kr[e >> 2][e & 3];
                    least = min(least, (__float_as_uint(x[e]) << 1) - 1u);
                }
                if (live) kq_min = min(kq_min, least);
                Planes p = split8(x);
                char* d = buf + slot8 * 128 + ((pc ^ ((slot8 >> 1) & 7)) << 4);
                *(bf16x8*)d = p.h;
                *(bf16x8*)(d + G::kPlane) = p.m;
                *(bf16x8*)(d + 2 * G::kPlane) = p.l;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = live ? vr[e >> 2][e & 3] : 0.f;
                    v_max = max(v_max, __float_as_uint(x[e]) << 1);
                }
                p = split8(x);
                d = buf + 3 * G::kPlane + slot8 * 128 + ((pc ^ (2 * (slot8 & 3))) << 4);
                *(bf16x8*)d = p.h;
                *(bf16x8*)(d + G::kPlane) = p.m;
                *(bf16x8*)(d + 2 * G::kPlane) = p.l;
            };
            fetch(0);
            Planes q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = qrow[0][16 * k + 8 * hh + e];
                    kq_min = min(kq_min, (__float_as_uint(x[e]) << 1) - 1u);
                }
                q[k] = split8(x);
            }
            put(0);
            if (nt > 1) fetch(1);
            Rows<T>& x = w[0];
            float ref = 0.f, sum[4] = {0.f, 0.f, 0.f, 0.f};
            const int row = swap23(l31), ka = row * 128 + ((hh ^ ((row >> 1) & 7)) << 4);
            const int i16 = lane & 15, dq = (lane >> 4) & 1;
            const int va = (8 * hh + (i16 >> 2)) * 128 +
                           (((2 * dq + ((i16 & 3) >> 1)) ^ (2 * (i16 >> 2))) << 4) + (i16 & 1) * 8;
            for (int t = 0; t < nt; ++t) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                const int k0 = c0 + t * 32;
                if (k0 < wlim) {
                    typedef __attribute__((address_space(3))) const bf16x8 lds_frag;
                    lds_char* buf = (lds_char*)smem + (t & 1) * G::kPlanes;
                    f32x16 s = zero_f32x16();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lds_char* k = buf + (ka ^ (i << 5));
                        const Planes f = {*(lds_frag*)k, *(lds_frag*)(k + G::kPlane), *(lds_frag*)(k + 2 * G::kPlane)};
                        s = mfma_planes(f, q[i], s);
                    }
                    if (k0 + 32 > seen_by_all) {   // (a lane's slots lie as in the bf16 blocks)
                        const int left = x.vis - k0 - 8 * hh;
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[r] = Geo<bf16, true>::key(r, 0) < left ? s[r] : -INFINITY;
                    }
                    if (t == 0) {
                        float top = s[0];
#pragma unroll
                        for (int r = 0; r < 16; r += 2) top = maximum(maximum(top, s[r]), s[r + 1]);
                        const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false,
                                                                        false);
                        x.m = maximum(__uint_as_float(y[0]), __uint_as_float(y[1])) * a.c2;
                        ref = x.m == -INFINITY ? 0.f : x.m;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[r] = exp2f_fast(fmaf(s[r], a.c2, -ref));
                        sum[r & 3] += s[r];
                    }
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = s[8 * st + e];
                        const Planes p = split8(z);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            lds_char* v = buf + 3 * G::kPlane + (va ^ (m << 6)) + st * 2048;
                            const Planes f = {tr_read(v), tr_read(v + G::kPlane), tr_read(v + 2 * G::kPlane)};
                            x.o[m] = mfma_planes(f, p, x.o[m]);
                        }
                    }
                }
                if (t + 1 < nt) {
                    put(t + 1);
                    if (t + 2 < nt) fetch(t + 2);
                }
            }
            x.l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            constexpr uint32_t kLeast = (24u << 24) - 1u;   // 2^-103
            if (__builtin_amdgcn_ballot_w64(kq_min < kLeast)) redo = true;
            __shared__ uint32_t s_vmax[G::NW];
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) v_max = max(v_max, (uint32_t)__shfl_xor((int)v_max, o));
            if (lane == 0) s_vmax[wave] = v_max;
            __syncthreads();
            for (int v = 0; v < G::NW; ++v) v_max = max(v_max, s_vmax[v]);
            const float lim = ((float)(c1 - c0) * __uint_as_float(v_max >> 1) + x.l) * 7.8886090522101181e-31f;   // 2^-100
            bool lost = false;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) lost = lost || (x.o[m][r] != 0.f && fabsf(x.o[m][r]) < lim);
            if (alive && __builtin_amdgcn_ballot_w64(lost)) redo = true;
        } else if constexpr (G::kBf) {
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {
                if (pass) {
                    restart(true);
                    issue_first();
                }
                careful(pass == 0);
                if (!overflown()) break;
            }
        } else {
            // Narrow fp32: a block's two products take as long as its copies do, so K of the next tile
            // arrives while V's product runs and V during the next logits; with half the LDS of two whole
            // tiles a second workgroup shares the compute unit (60,000 slots of four heads, a token:
            // 43 us with two whole tiles, so 35).
            static_assert(G::TK == 32, "two units per tile");
            int id0, id1;   // pages of the tile whose K was issued last (the window only moves on)
            auto issue_k = [&](int t) {
                id0 = unit_page(t, 0);
                issue_unit(t, 0, false, id0);
                id1 = unit_page(t, 1);
                issue_unit(t, 1, false, id1);
            };
            auto issue_v = [&](int t) {
                issue_unit(t, 0, true, id0);
                issue_unit(t, 1, true, id1);
            };
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {
                if (pass) restart(true);
                issue_k(0);
                issue_v(0);
                for (int t = 0; t < nt; ++t) {
                    const int k0 = c0 + (tfirst + t * tstep) * G::TK;
                    lds_char* tile = tile_at(t);
                    wait_tiles<G::CPT / 2>(1);                                  // K; V may be on its way
                    const bool partial = !pw.sane || k0 + G::TK > seen_by_all;
                    const uint32_t units = partial ? groups(k0) : 0;
                    const bool some = k0 < wlim, next = t + 1 < nt;
                    Probs<T, G::kSplit> p;
                    if (some) block_probs<T, G::kSplit>(w[0], tile, a.c2, k0, partial, units, lane, logits, p);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // K is read
                    if (next) issue_k(t + 1);
                    wait_tiles<G::CPT / 2>(next ? 1 : 0);                       // V; the next K may be on its way
                    if (partial) odd |= clean_values<T>(tile + G::kTileV, G::TK, k0, c1, units, lane);
                    if (some) block_values<T, G::kSplit>(w[0], tile + G::kTileV, p, false, lane);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // V is read
                    if (next) issue_v(t + 1);
                }
                if (!overflown()) break;
            }
        }
        if constexpr (WIDE) {
            __shared__ int s_redo[G::NW];
            redo = redo || !pw.sane || (!kCode && overflown());
            if (alive) {
                bool far = false;
#pragma unroll
                for (int nb = 0; nb < G::NB; ++nb)
                    far = far || !(w[nb].l < 1152921504606846976.f) || (w[nb].m == -INFINITY && w[nb].vis > c0);   // 2^60
                redo = redo || __builtin_amdgcn_ballot_w64(far);
            }
            if (lane == 0) s_redo[wave] = redo;
            __syncthreads();
            auto any_wave = [&]() {
                int any = 0;
                for (int v = 0; v < G::NW; ++v) any |= s_redo[v];
                return any != 0;
            };
            bool again = any_wave();
            if constexpr (kCode) {
                int f = 0, l = 0;
                for (int v = 0; v < G::NW; ++v) f = max(f, s_range[v]), l = max(l, s_range[G::NW + v]);
                again = again || f - 1 > kUp + kDown || f - 1 > 31 - l;
            }
            if (again) {
                if constexpr (!G::kBf) load_q();
#pragma unroll 1
                for (int pass = 0; pass < 2; ++pass) {
                    restart(pass > 0);
                    issue_first();
                    careful(kCode && pass == 0);
                    const bool far = overflown();
                    __syncthreads();
                    if (lane == 0) s_redo[wave] = far;
                    __syncthreads();
                    if (!any_wave()) break;
                }
            }
        }
        if constexpr (WIDE) {   // what one wave took out, all see to
            __shared__ int s_odd[G::NW];
            if (lane == 0) s_odd[wave] = odd;
            __syncthreads();
            for (int v = 0; v < G::NW; ++v) odd |= s_odd[v] != 0;
        }
        if (odd && alive)
            for (int t = 0; t < nt; ++t) {
                const int k0 = c0 + (tfirst + t * tstep) * G::TK;
                if (!pw.sane || k0 + G::TK > seen_by_all)
#pragma unroll
                    for (int nb = 0; nb < G::NB; ++nb)
                        add_odd_values<T, CODE>(a, w[nb], b, hk, k0, k0 + G::TK < c1 ? k0 + G::TK : c1, lane);
            }
    }
#pragma unroll
    for (int nb = 0; nb < G::NB; ++nb) w[nb].l += __shfl_xor(w[nb].l, 32);

    const int64_t all_rows = (int64_t)a.c.T * a.Hq;
    // (Parts of a row are divided by their own l, so that no sum of them passes the largest value.)
    if constexpr (WIDE) {
#pragma unroll
        for (int nb = 0; nb < G::NB; ++nb) {
            if ((kCode && nb && slim) || row0 + 32 * nb + l31 >= nrows) return;
            float inv, lse;
            row_result(w[nb].m, w[nb].l, &inv, &lse);
            if (inv == 0.f) w[nb].o[0] = w[nb].o[1] = zero_f32x16();   // no weight on any values
            if (a.nsplit > 1) {
                float* po = a.part + (split * all_rows + orow[nb]) * kD;
                if (hh == 0) {
                    f32x2 ml = {w[nb].m, w[nb].l};
                    *(f32x2*)(a.part_ml + (split * all_rows + orow[nb]) * 2) = ml;
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = w[nb].o[m][4 * g + e] * inv;
                        *(f32x4*)(po + 32 * m + 8 * g + 4 * hh) = v;
                    }
                continue;
            }
            if (hh == 0) put_lse(a, orow[nb], lse);
            T* out = (T*)a.O + orow[nb] * kD;
            if constexpr (G::kBf) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        uint32_t d[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            bf16x2 pr = {(bf16)(w[nb].o[m][8 * g + 2 * e] * inv),
                                         (bf16)(w[nb].o[m][8 * g + 2 * e + 1] * inv)};
                            d[e] = __builtin_bit_cast(uint32_t, pr);
                        }
                        swap_halves(d[0], d[2]);
                        swap_halves(d[1], d[3]);
                        u32x4 v = {d[0], d[1], d[2], d[3]};
                        *(u32x4*)(out + 32 * m + 16 * g + 8 * hh) = v;
                    }
            } else {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = w[nb].o[m][4 * g + e] * inv;
                        *(f32x4*)(out + 32 * m + 8 * g + 4 * hh) = v;
                    }
            }
        }
    } else {
        // The four waves' partial results meet in LDS (the ring is free then).
        constexpr int kRow = 68;
        float* sml = (float*)smem;                 // [4][32][2]
        float* smeet = (float*)smem + 256;         // [32][2]
        float* so = (float*)smem + 320;            // [4][32][68]
        static_assert((320 + 4 * 32 * kRow) * 4 <= G::kLds, "partial results fit the ring");
        __syncthreads();
        if (hh == 0) {
            sml[(wave * 32 + l31) * 2] = w[0].m;
            sml[(wave * 32 + l31) * 2 + 1] = w[0].l;
        }
        __syncthreads();
        float M = -INFINITY, L = 0.f, inv, lse;
        float mv[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) M = maximum(M, mv[v] = sml[(v * 32 + l31) * 2]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int v = 0; v < 4; ++v) L += exp2f_fast(mv[v] - ref) * sml[(v * 32 + l31) * 2 + 1];
        row_result(M, L, &inv, &lse);
        const float f = exp2f_fast(w[0].m - ref) * inv;
        if (wave == 0 && hh == 0) {
            smeet[l31 * 2] = M;
            smeet[l31 * 2 + 1] = L;
        }
        if (row0 + l31 < nrows) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = f == 0.f ? 0.f : w[0].o[m][4 * g + e] * f;   // (any values)
                    *(f32x4*)(so + (wave * 32 + l31) * kRow + 32 * m + 8 * g + 4 * hh) = v;
                }
        }
        __syncthreads();
        const int rr = tid >> 3, d0 = (tid & 7) * 8, r = row0 + rr;
        if (r < nrows) {
            const int i = r / a.G;
            const int64_t at = (int64_t)(sq.q0 + i) * a.Hq + hk * a.G + r - i * a.G;
            M = smeet[rr * 2], L = smeet[rr * 2 + 1];
            float acc[8] = {};
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += so[(v * 32 + rr) * kRow + d0 + e];
            if (a.nsplit > 1) {
                float* po = a.part + (split * all_rows + at) * kD + d0;
                *(f32x4*)po = f32x4{acc[0], acc[1], acc[2], acc[3]};
                *(f32x4*)(po + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
                if (d0 == 0) *(f32x2*)(a.part_ml + (split * all_rows + at) * 2) = f32x2{M, L};
            } else {
                row_result(M, L, &inv, &lse);
                if (d0 == 0) put_lse(a, at, lse);
                T* out = (T*)a.O + at * kD + d0;
                if constexpr (G::kBf) {
                    *(bf16x8*)out = pack_bf16x8(acc[0], acc[1], acc[2], acc[3], acc[4], acc[5], acc[6], acc[7]);
                } else {
                    *(f32x4*)out = f32x4{acc[0], acc[1], acc[2], acc[3]};
                    *(f32x4*)(out + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
                }
            }
        }
    }
}

// ------------------------------------------------------------------------
// Join of the split results whose slot range a row sees.  16 lanes hold a row's 64 features.  MANY:
// a wave per row, four splits at a time; otherwise (up to kFew splits) four rows per wave.  All of a
// lane's loads are issued before the first is used.
// Bound by the latency of two dependent loads, then by the parts' bytes (1,374 tokens of 16 heads, five
// ranges: 30 MB in 8 us).
// ------------------------------------------------------------------------
constexpr int kFew = 8;

template <typename T, bool MANY>
__global__ __launch_bounds__(256) void k_cache_join(AttendArgs a) {
    const int lane = threadIdx.x & 63, grp = lane >> 4, d = (lane & 15) * 4;
    const int b = blockIdx.y;
    const CacheSeq sq = cache_seq(a.c, b);
    const int wv = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r = MANY ? wv : 4 * wv + grp;   // (token, head) of the sequence
    const int i = r / a.Hq;
    if (i >= sq.nq) return;
    const int64_t at = (int64_t)sq.q0 * a.Hq + r, all_rows = (int64_t)a.c.T * a.Hq;
    const int vis = cache_visible(sq, a.causal, i);
    int ns = (vis + a.chunk - 1) / a.chunk;
    ns = ns < 1 ? 1 : ns < a.nsplit ? ns : a.nsplit;
    constexpr int kLanes = MANY ? 64 : 16;        // lanes that share a row
    const int own = lane & (kLanes - 1);
    // The reference of all splits, their factors (a lane's splits: own, own + kLanes, ..), the sum.
    constexpr int kMl = MANY ? 4 : 1;             // (at most 256 splits)
    f32x2 ml[kMl];
    float M = -INFINITY;
#pragma unroll
    for (int j = 0; j < kMl; ++j) {
        ml[j] = f32x2{-INFINITY, 0.f};
        const int s = own + j * kLanes;
        if (s < ns) ml[j] = *(const f32x2*)(a.part_ml + (s * all_rows + at) * 2);
    }
    constexpr int kBatch = MANY ? 4 * kFew : kFew;   // splits per batch of loads
    f32x4 v[kFew];
    auto load = [&](int s0) {
#pragma unroll
        for (int k = 0; k < kFew; ++k) {
            const int s = s0 + (MANY ? 4 * k + grp : k);
            v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (s < ns) v[k] = *(const f32x4*)(a.part + (s * all_rows + at) * kD + d);
        }
    };
    load(0);
#pragma unroll
    for (int j = 0; j < kMl; ++j) M = maximum(M, ml[j][0]);
#pragma unroll
    for (int o = kLanes / 2; o >= 1; o >>= 1) M = maximum(M, __shfl_xor(M, o));
    float f[kMl], L = 0.f;
#pragma unroll
    for (int j = 0; j < kMl; ++j) {
        f[j] = ml[j][0] == -INFINITY ? 0.f : ml[j][0] == M ? 1.f : exp2f_fast(ml[j][0] - M);
        L += f[j] * ml[j][1];
    }
#pragma unroll
    for (int o = kLanes / 2; o >= 1; o >>= 1) L += __shfl_xor(L, o);
    float inv, lse;
    row_result(M, L, &inv, &lse);
#pragma unroll
    for (int j = 0; j < kMl; ++j) f[j] *= ml[j][1] * inv;   // the part's share (its sums are divided by its own l)
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < ns; s0 += kBatch) {
        if (s0 > 0) load(s0);
        const float fj = MANY ? (s0 < 64 ? f[0] : s0 < 128 ? f[kMl > 1 ? 1 : 0] : s0 < 192 ? f[kMl > 2 ? 2 : 0] : f[kMl - 1]) : f[0];
#pragma unroll
        for (int k = 0; k < kFew; ++k) {
            const int s = s0 + (MANY ? 4 * k + grp : k);
            const float x = __shfl(fj, MANY ? s & 63 : (lane & 48) + k);
            // (a split without weight may hold anything)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += s < ns && x != 0.f ? x * v[k][e] : 0.f;
        }
    }
    if constexpr (MANY) {
#pragma unroll
        for (int o = 16; o <= 32; o <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
        if (grp) return;
    }
    if ((lane & 15) == 0) put_lse(a, at, lse);
    T* out = (T*)a.O + at * kD + d;
    if constexpr (sizeof(T) == 2) {
        bf16x4 y = {(bf16)acc[0], (bf16)acc[1], (bf16)acc[2], (bf16)acc[3]};
        *(bf16x4*)out = y;
    } else {
        *(f32x4*)out = acc;
    }
}

// ------------------------------------------------------------------------
// Attention weights that fall on every slot, weight_out = weight + sum over the group's rows of
// e^{x_j - lse}.  Every slot is written by one wave: no atomics, one order.
//
// Few rows (single tokens): the attention kept its logits; four slots a thread, rows one after the other.
// Bound by memory: 12 bytes per slot and one row (200,124 slots of 16 heads: 13 us, 3 TB/s).
// ------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_cache_weight_rows(AttendArgs a) {
    const int hk = blockIdx.y % a.c.Hkv, b = blockIdx.y / a.c.Hkv;
    const CacheSeq sq = cache_seq(a.c, b);
    const int k0 = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (k0 >= sq.len || sq.nq == 0) return;
    const int page = a.c.table[(int64_t)b * a.c.max_pages + (k0 >> a.c.page_log2)];
    if (page < 0 || page >= a.c.npages) return;
    const int64_t at = (((int64_t)page * a.c.Hkv + hk) << a.c.page_log2) + (k0 & ((1 << a.c.page_log2) - 1));
    const int left = sq.len - k0;
    float w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = e < left ? a.c.weight[at + e] : 0.f;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = 4;   // rows whose loads are issued together
    const int rows = sq.nq * a.G;
    int i = 0, g = 0;            // the next row's token and head
    for (int r0 = 0; r0 < rows; r0 += kAtOnce) {
        f32x4 x[kAtOnce];
        float lse[kAtOnce];
        int seen[kAtOnce];
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            x[n] = f32x4{0.f, 0.f, 0.f, 0.f};
            lse[n] = -INFINITY;
            seen[n] = 0;
            if (r0 + n < rows) {
                const int64_t row = (int64_t)(sq.q0 + i) * a.Hq + hk * a.G + g;
                x[n] = *(const f32x4*)(a.logits + row * a.logit_stride + k0);
                lse[n] = a.lse[row];
                seen[n] = cache_visible(sq, a.causal, i) - k0;
                if (++g == a.G) g = 0, ++i;
            }
        }
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            if (lse[n] == -INFINITY) seen[n] = 0;   // a row without weights adds none
            const float off = lse[n] * kLog2e;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[e] += e < seen[n] ? exp2f_fast(fmaf(x[n][e], a.c2, -off)) : 0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) a.weight_out[at + e] = w[e] + sum[e];
}

// ------------------------------------------------------------------------
// Chunks: logits formed again.  64 slots per workgroup: keys stay in registers as the MFMA's B
// operand (a lane owns one slot), two waves for each 32 slots that take half a tile's rows each.
// The rows stream through LDS as A with -lse in the accumulator's input (`off`, written with lse), so
// that a result is the exponent itself.  Bound by the vector units (a product, a power and a sum
// per logit: 1,374 tokens over 43,968 slots of 16 heads 210 us; fp32, whose products are fp32 MFMAs,
// 500 tokens of two heads each over 8,000 slots of eight 75 us).  Two tiles of 128 rows in LDS
// let four workgroups share a compute unit; their waves fill each other's waits, and forming the products of
// one block amid another's powers, or six workgroups with half the rows, gained nothing.
// ------------------------------------------------------------------------
template <typename T, int CODE>
__global__ __launch_bounds__(256, 4) void k_cache_weight(AttendArgs a) {
    constexpr bool kBf = sizeof(T) == 2;
    constexpr int kStep = kBf ? 128 : 64, RB = kStep / 64;    // rows per tile, 32-row blocks of a wave
    constexpr int ROWB = kD * sizeof(T), RPC = 1024 / ROWB;   // bytes per row, rows per copy
    constexpr int kTile = kStep * ROWB + kStep * 4;           // rows, then their offsets
    constexpr int NST = 2, AHEAD = NST - 1, NC = kStep / RPC / 4, CPT = NC + 1;
    __shared__ __attribute__((aligned(1024))) char smem[NST * kTile];
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hk = blockIdx.y % a.c.Hkv, b = blockIdx.y / a.c.Hkv;
    const CacheSeq sq = cache_seq(a.c, b);
    const int k0 = blockIdx.x * 64;
    if (k0 >= sq.len || sq.nq == 0) return;
    // Rows that see the workgroup's first slot: causal rows before them add nothing.
    const int nrows = sq.nq * a.G;
    int first = 0;
    if (a.causal) first = clampi(k0 - (sq.len - sq.n), 0, sq.nq) * a.G;
    first &= ~(kStep - 1);
    const int nt = (nrows - first + kStep - 1) / kStep;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
    // Row r = i G + g lies at i (tokens' distance) + g (heads' distance).  Offsets count from the first
    // row's token of their tile and are stepped along with the tiles, di tokens and dg heads at a time
    // (nothing moves where G divides the tile; a division and a product per copy took as many
    // vector instructions as the exponentials: 67 us -> 61 us for 1,031 tokens of two heads each over
    // 10,992 slots).
    const int di = kStep / a.G, dg = kStep - di * a.G;
    const int last_i = (nrows - 1) / a.G, last_g = nrows - 1 - last_i * a.G;
    int base_i = first / a.G, base_g = first - base_i * a.G;
    const uint32_t qs = (uint32_t)a.q_stride * sizeof(T), hs = ROWB;   // bytes
    const uint32_t os = (uint32_t)a.Hq * 4;
    const int off_row = (wave * 64) % kStep;   // (the offsets' copies: one a wave)
    uint32_t off[NC + 1];   // per copy: row, and for Q the lane's 16 bytes of it
    int g[NC + 1];
    // pieces of 16 bytes exchanged within their row so that reads meet no bank twice
    auto piece = [&](int j) {
        const int rr = (wave * NC + j) * RPC + lane / (64 / RPC), pc = lane % (64 / RPC);
        return (uint32_t)(pc ^ (kBf ? (rr >> 1) & 7 : rr & 15)) << 4;
    };
#pragma unroll
    for (int j = 0; j <= NC; ++j) {
        const int r = first + (j < NC ? (wave * NC + j) * RPC + lane / (64 / RPC) : off_row + lane), i = r / a.G;
        g[j] = r - i * a.G;
        off[j] = j < NC ? (uint32_t)(i - base_i) * qs + g[j] * hs + piece(j) : (uint32_t)(i - base_i) * os + g[j] * 4;
    }
    auto issue = [&](int t) {
        const uint32_t stage = lds0 + (t % NST) * kTile;
        const char* q0 = (const char*)((const T*)a.Q + (int64_t)(sq.q0 + base_i) * a.q_stride + hk * a.G * kD);
        const char* o0 = (const char*)(a.off + (int64_t)(sq.q0 + base_i) * a.Hq + hk * a.G);
        const int ahead = last_i - base_i;
        uint32_t v[NC + 1];
#pragma unroll
        for (int j = 0; j <= NC; ++j) v[j] = off[j];
        if (ahead <= di + 1) {   // rows past the last one: the last again
            const uint32_t lim = (uint32_t)ahead * qs + last_g * hs, olim = (uint32_t)ahead * os + last_g * 4;
#pragma unroll
            for (int j = 0; j < NC; ++j) v[j] = min(v[j] - piece(j), lim) + piece(j);
            v[NC] = min(v[NC], olim);
        }
#pragma unroll
        for (int j = 0; j < NC; ++j) copy_to_lds(stage + (wave * NC + j) * 1024, q0, v[j]);
        copy4_to_lds(stage + kStep * ROWB + off_row * 4, o0, v[NC]);
        base_i += di;
        if (dg == 0) return;
        base_g += dg;
        const bool over = base_g >= a.G;
        if (over) base_g -= a.G, ++base_i;
#pragma unroll
        for (int j = 0; j <= NC; ++j) {
            const uint32_t row = j < NC ? qs : os, head = j < NC ? hs : 4;
            g[j] += dg;
            off[j] += dg * head - (over ? row : 0);
            if (g[j] >= a.G) {
                g[j] -= a.G;
                off[j] += row - a.G * head;
            }
        }
    };
#pragma unroll
    for (int t = 0; t < AHEAD; ++t)
        if (t < nt) issue(t);
    const int slot = k0 + 32 * (wave & 1) + l31;
    int page = -1;
    if (slot < sq.len) page = a.c.table[(int64_t)b * a.c.max_pages + (slot >> a.c.page_log2)];
    const bool live = page >= 0 && page < a.c.npages;
    const int64_t at = (((int64_t)(live ? page : 0) * a.c.Hkv + hk) << a.c.page_log2) +
                       (slot & ((1 << a.c.page_log2) - 1));
    bf16x8 kb[4];
    float kf[kBf ? 1 : 32];
    if constexpr (CODE != CODE_NONE) {
        // (8-bit codes: code times scale is a bf16 value)
        const float s = live ? key_scale(a.c.scale[at]) : 0.f;
        const char* kr = (const char*)a.c.K + at * kD;
#pragma unroll
        for (int i = 0; i < (kBf ? 4 : 8); ++i) {
            if constexpr (kBf) {
                float x[4], y[4];
                const uint2 v = live ? *(const uint2*)(kr + 16 * i + 8 * hh) : make_uint2(0u, 0u);
                values4<CODE>(v.x, s, x);
                values4<CODE>(v.y, s, y);
                kb[i] = pack_bf16x8(x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]);
            } else {
                float x[4];
                values4<CODE>(live ? *(const uint32_t*)(kr + 8 * i + 4 * hh) : 0u, s, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) kf[4 * i + e] = x[e];
            }
        }
    } else if constexpr (kBf) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kb[i] = zero_bf16x8();
            if (live) kb[i] = load_bf16x8((const T*)a.c.K + at * kD + 16 * i + 8 * hh);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (live) v = *(const f32x4*)((const T*)a.c.K + at * kD + 8 * i + 4 * hh);
#pragma unroll
            for (int e = 0; e < 4; ++e) kf[4 * i + e] = v[e];
        }
    }
    // first row that sees this lane's slot (token i sees slots up to len - n + i)
    const int row_min = a.causal && slot > sq.len - sq.n ? (slot - (sq.len - sq.n)) * a.G : 0;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    const int half = wave >> 1;
    for (int t = 0; t < nt; ++t) {
        const int more = nt - 1 - t, r0 = first + t * kStep;
        wait_tiles<CPT>(more < AHEAD - 1 ? more : AHEAD - 1);
        __builtin_amdgcn_s_barrier();
        if (t + AHEAD < nt) issue(t + AHEAD);
        lds_char* tile = (lds_char*)smem + (t % NST) * kTile;
        // slots that row r0 sees all rows of the tile see
        const bool mask = (a.causal && k0 + 64 > cache_visible(sq, 1, r0 / a.G)) || r0 + kStep > nrows;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
            typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
            const int br = 32 * (RB * half + rb);   // first row of the block
            f32x16 x;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = *(lds_f32x4*)(tile + kStep * ROWB + (br + 8 * g + 4 * hh) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * g + e] = v[e];
            }
            lds_char* qr = tile + (br + l31) * ROWB;
            const int f = kBf ? (l31 >> 1) & 7 : l31 & 15;
#pragma unroll
            for (int i = 0; i < (kBf ? 4 : 8); ++i) {
                if constexpr (kBf) {
                    x = mfma_bf16(*(lds_bf16x8*)(qr + (((2 * i + hh) ^ f) << 4)), kb[i], x);
                } else {
                    const f32x4 q = *(lds_f32x4*)(qr + (((2 * i + hh) ^ f) << 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x = mfma_f32(q[e], kf[4 * i + e], x);
                }
            }
            if (mask) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int rr = r0 + br + 8 * (r >> 2) + 4 * hh + (r & 3);
                    x[r] = rr >= row_min && rr < nrows ? x[r] : -INFINITY;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[r & 3] += exp2f_fast(x[r] * a.c2);
        }
    }
    float t = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    t += __shfl_xor(t, 32);
    // the two halves of the rows
    __syncthreads();
    float* meet = (float*)smem;
    if (half == 1 && hh == 0) meet[32 * (wave & 1) + l31] = t;
    __syncthreads();
    if (half == 0 && hh == 0 && live) a.weight_out[at] = a.c.weight[at] + (t + meet[32 * (wave & 1) + l31]);
}

// ------------------------------------------------------------------ launchers

// Variant and split of a call, from the host's sizes alone (so that results do not depend on
// the lengths' values on the device).
void attend_plan(AttendArgs* a) {
    const int64_t rows = (int64_t)a->c.max_q * a->G;
    const bool bf = a->c.dtype == DT_BF16;
    // Row tiles of rt rows: the largest sequence's, and the others', of which only the sum of the tokens
    // is known, in units of its tiles: their lengths are taken as about half of the bound on the average (single
    // tokens, whose ranges all wait for HBM, as 0.65), unless all have chunks of the same size, more than a
    // token.  (32 ragged sequences: 31 us, with every one counted as the largest 34; if all are equal
    // after all, 49 against 45.  Three ragged prompts in fp32: 68 and 80.)
    const int64_t rest = a->c.T > a->c.max_q ? a->c.T - a->c.max_q : 0;
    const int64_t others = a->c.B - 1 < rest ? a->c.B - 1 : rest;
    const bool equal = a->c.B == 1 || (a->c.max_q > 1 && a->c.T == (int64_t)a->c.B * a->c.max_q);
    auto work_items = [&](int rt, bool wide) {
        a->row_tiles = (int)std::max<int64_t>(1, (rows + rt - 1) / rt);
        double tiles = (double)others * a->row_tiles;
        if (!equal) {
            if (a->row_tiles > 1) tiles = std::min(tiles, (double)(rest * a->G) / rt + 0.5 * others);
            tiles *= wide ? 0.5 : 0.65;
        }
        return a->c.Hkv * (a->row_tiles + tiles);
    };
    // Narrow workgroups start and end sooner, wide ones read less from L2 and LDS per row: narrow up to 64
    // rows and, in bf16, where each of 512 workgroups has few slots, fewer if that takes more than a round.  (16
    // heads: 1,000 tokens over 1,000 slots, 1,000 slots each, 15.9 us narrow, 23.3 wide; 400 over 5,000, 2,000 each,
    // both 34; 200 over 20,000, 4,400 each, 49 and 41; 1,374 over themselves, 1,850 each in 1.3 rounds, 37 and
    // 29.  fp32, whose wide kernel has the faster products: 64 over 20,000 56 and 57, 90 over 20,000 80 and
    // 61, 200 over 600 22 and 18; 90 over 300 13.3 and 15.8.)
    // An estimate that ranks divisions into ns ranges, in us where the card is lightly loaded (large calls, which HBM or
    // all SIMDs at once bound, take up to three times as long: 50 for 167 us of tokens over 137,400 slots, 153
    // for 260 of a view over 43,968): the slots of a workgroup and its start, in units of slots, times the rounds of
    // workgroups that run together, or, ragged and more than a round, all the work and a last workgroup; the join, a
    // launch, and what it reads per range.  (300 slots, a token, bf16: 8.3 us
    // in one range, 11.1 in three; 1,000 slots, 200 tokens: 25 in one, 17 in eight; 30 sequences of up to
    // 102 tokens and 8,333 slots: 140 in one, 115 in eight, 131 in sixteen.)
    const int64_t most = (a->c.max_len + 127) / 128;
    int64_t best = 1;
    // `whole`: workgroups per range; `share`: of all the work, what the estimate of it counts
    auto divide = [&](double items, double whole, double slot, double start, double together, double range, bool one_round,
                      double share) {
        double best_t = 0;
        for (int64_t ns = 1; ns <= most && ns <= 256; ++ns) {
            const int64_t ch = ((a->c.max_len + ns - 1) / ns + 63) / 64 * 64;
            double slots = ceil(items * ns / together) * (ch + start);
            if (!equal) {
                const double all = share * (items * (a->c.max_len + start * ns) / together + ch + start);
                slots = one_round && whole * ns <= together ? std::min<double>(ch + start, all) : all;
            }
            const double t = slots * slot + range * ns + (ns == 1 ? 0. : ns <= kFew ? 3. : 4.5);
            if (ns == 1 || t < best_t) best = ns, best_t = t;
        }
        return best_t;
    };
    a->wide = 0;
    if (!a->c.code) {
        double items = work_items(32, false);
        a->wide = rows > 64 && (!bf || items * a->c.max_len > 512. * (items > 512 ? 1500 : 2500));
        if (a->wide) items = work_items(attend_rows(*a), true);
        divide(items, items, a->wide ? (bf ? 0.016 : 0.038) : (bf ? 0.006 : 0.019), a->wide ? 512 : 192, 512,
               a->wide ? 0.15 : 0.05, true, 1);
    } else {
        // 8-bit codes: narrow workgroups, which each decode what they read, by all the work if ragged (31 tokens of four key
        // heads, ragged to 10,992 slots: 31 us in the six ranges of one round, 28 in eight, 27 in eleven); wide ones, whose
        // time per slot grows with the waves that have rows, and of which a compute unit has one.  The shorter estimate
        // decides, in us: 16 heads, 1,000 tokens over 1,000 slots 22 narrow, 33 wide; 400 over 5,000 42 and 37; 90 over 20,000 37
        // and 36; 200 over 3,000 22 and 24; ragged to 400 tokens over 3,000 slots, 16 sequences, 81 and 75.  Ragged batches
        // whose rows would fill less than a seventh of the wide tiles stay narrow (30 sequences of up to 102 tokens and 8,333
        // slots: 75 and 96).  What the lengths are is guessed: 0.6 of the work that the wide tiles' bounds allow, and 0.8 of
        // the narrow estimate.  Of 44 random batches (2 to 32 sequences, of up to 70 to 1,374 tokens and 300 to 30,000 slots, 2 to
        // 16 key heads) the picks take 1.06 of the better kernel's time on the average, narrow alone 1.31, wide alone 1.08; with
        // 1 for the 0.8 1.05, with 1 for the 0.6 1.06, without the seventh 1.05: these decide near ties.
        double t = divide(work_items(attend_rows(*a), false), 0, rows <= 16 ? 0.008 : bf ? 0.017 : 0.03, 192, 512, 0.05, false, 1);
        if (!equal) t *= 0.8;   // (the others' lengths are less than assumed more often than not)
        const int64_t narrow = best;
        if (bf && rows > 64) {
            a->wide = 1;
            const int rt = attend_rows(*a);
            // us per slot of a tile of n rows
            auto slot = [](double n) { return 0.01 + 0.0024 * std::min(8., ceil(n / 64)); };
            const double items = work_items(rt, true), one = slot((double)rows);
            // Row tiles, of few rows as their share of `one`: the largest sequence's and the others'.
            const double own = a->row_tiles == 1 ? 1 : (double)(rows / rt) + (rows % rt ? slot((double)(rows % rt)) / one : 0);
            const double few = others ? slot((double)rest * a->G / others) / one : 0;
            const double whole = own + std::min(others * own, (a->row_tiles > 1 ? (double)rest * a->G / rt : 0) + others * few);
            const double tiles = a->row_tiles + std::min((double)others * a->row_tiles, (double)rest * a->G / rt + others);
            a->wide = divide(items, a->c.Hkv * whole, one, 600, 256, 0.15, true, 0.6) < t &&
                      (equal || (double)a->c.T * a->G >= 0.15 * tiles * rt);
        }
        if (!a->wide) {
            work_items(attend_rows(*a), false);
            best = narrow;
        }
    }
    a->chunk = (int)(((a->c.max_len + best - 1) / best + 63) / 64 * 64);
    if (a->chunk < 64) a->chunk = 64;
    a->logit_stride = (a->c.max_len + 63) / 64 * 64;
    a->nsplit = (int)((a->c.max_len + a->chunk - 1) / a->chunk);
    if (a->nsplit < 1) a->nsplit = 1;
}

// Rows per workgroup.
int attend_rows(const AttendArgs& a) {
    if (a.c.code) return a.wide ? GeoOf<bf16, true, CODE_INT8>::RT : (int64_t)a.c.max_q * a.G <= 16 ? 16 : 32;
    if (a.c.dtype == DT_BF16) return a.wide ? Geo<bf16, true>::RT : Geo<bf16, false>::RT;
    return a.wide ? Geo<float, true>::RT : Geo<float, false>::RT;
}

size_t attend_part_rows(const AttendArgs& a) {
    return a.nsplit > 1 ? (size_t)a.nsplit * a.c.T * a.Hq : 0;
}

// Keeping a logit costs 8 bytes (written and read) per row and slot, forming it again a key's
// 128 or 256 per slot and a tile of 128 or 64 rows however few there are.  60,000 slots of 16 heads, bf16: 8
// rows of a key head 56 us kept, 111 formed again, 32 rows 104 and 112; fp32, 16 rows 135 and 220, 64 rows
// 228 and 268.  More than eight rows of a short cache are formed again, as a thread takes them one after the other
// (16 rows, 2,000 slots: 17.6 kept, 16.0 again), and so is what would take more than 2 GiB.
size_t attend_logits(const AttendArgs& a) {
    const int64_t rows = (int64_t)a.c.max_q * a.G;
    if (!a.c.weight || a.wide || rows > (a.c.dtype == DT_BF16 ? 32 : 64) || (rows > 8 && a.c.max_len < 4096)) return 0;
    const int64_t n = (int64_t)a.c.T * a.Hq * a.logit_stride;
    return n <= (int64_t)1 << 29 ? n : 0;
}

template <typename T>
static void join_go(const AttendArgs& a, hipStream_t st) {
    const int64_t rows = (int64_t)a.c.max_q * a.Hq;
    if (a.nsplit > kFew)
        hipLaunchKernelGGL((k_cache_join<T, true>), dim3((rows + 3) / 4, a.c.B), dim3(256), 0, st, a);
    else if (a.nsplit > 1)
        hipLaunchKernelGGL((k_cache_join<T, false>), dim3((rows + 15) / 16, a.c.B), dim3(256), 0, st, a);
}

template <typename T, int CODE>
static void weights_go(const AttendArgs& a, hipStream_t st) {
    if (!a.weight_out || a.c.max_len == 0) return;
    const unsigned bh = a.c.B * a.c.Hkv;
    if (a.logits) {
        hipLaunchKernelGGL(k_cache_weight_rows, dim3((a.c.max_len + 1023) / 1024, bh), dim3(256), 0, st, a);
    } else {
        hipLaunchKernelGGL((k_cache_weight<T, CODE>), dim3((a.c.max_len + 63) / 64, bh), dim3(256), 0, st, a);
    }
}

template <typename T>
static void attend_go(const AttendArgs& a, hipStream_t st) {
    const int64_t grid = ((int64_t)a.c.B * a.c.Hkv * a.nsplit + 7) / 8 * 8 * a.row_tiles;
    if (a.c.code && !a.wide) {
        launch_cache8_attend(a, st);
    } else if (a.c.code) {
        if constexpr (sizeof(T) == 2) {
            const dim3 threads(64 * GeoOf<T, true, CODE_INT8>::NW);
            if (a.c.code == CODE_E4M3) hipLaunchKernelGGL((k_cache_attend<T, true, CODE_E4M3>), dim3(grid), threads, 0, st, a);
            else hipLaunchKernelGGL((k_cache_attend<T, true, CODE_INT8>), dim3(grid), threads, 0, st, a);
        }
    } else if (a.wide) {
        hipLaunchKernelGGL((k_cache_attend<T, true, CODE_NONE>), dim3(grid), dim3(64 * Geo<T, true>::NW), 0, st, a);
    } else {
        hipLaunchKernelGGL((k_cache_attend<T, false, CODE_NONE>), dim3(grid), dim3(256), 0, st, a);
    }
    join_go<T>(a, st);
    if (a.c.code == CODE_E4M3) weights_go<T, CODE_E4M3>(a, st);
    else if (a.c.code == CODE_INT8) weights_go<T, CODE_INT8>(a, st);
    else weights_go<T, CODE_NONE>(a, st);
}

void launch_cache_attend(const AttendArgs& a, hipStream_t st) {
    if (a.c.dtype == DT_BF16) attend_go<bf16>(a, st);
    else attend_go<float>(a, st);
}

}  // namespace vp
