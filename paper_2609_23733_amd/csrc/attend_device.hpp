// What the kernels of the paged cache's attention share.
#pragma once

#include "cache_device.hpp"

namespace vp {

__device__ __forceinline__ float maximum(float a, float b) {
    return __builtin_elementwise_maximum(a, b);   // IEEE maximum: a NaN stays one
}

// Page numbers of a run of slots: lane i holds the page of the table's entry first + i.  Numbers
// outside the pool count as page 0 here and clear `sane`; the slots on such pages are masked.
struct PageWindow {
    const int32_t* row;   // the sequence's table row
    int last;             // last entry that may be read
    int64_t npages;
    int first, cur, next;
    bool sane;

    __device__ __forceinline__ int load(int at, int lane) const {
        const int i = at + lane;
        return row[i < last ? i : last];
    }
    __device__ __forceinline__ bool valid(int id) const { return id >= 0 && id < npages; }
    __device__ __forceinline__ int settle(int id) {
        if (__builtin_amdgcn_ballot_w64(!valid(id))) sane = false;
        return valid(id) ? id : 0;
    }
    __device__ __forceinline__ void start(const CacheArgs& a, int b, int lo, int last_slot, int lane) {
        row = a.table + (int64_t)b * a.max_pages;
        last = last_slot >> a.page_log2;
        npages = a.npages;
        sane = true;
        first = lo >> a.page_log2;
        const int id = load(first, lane);
        next = load(first + 64, lane);
        cur = settle(id);
    }
    // Page of table entry `at` (uniform, never falling from call to call).
    __device__ __forceinline__ int page(int at, int lane) {
        if (at - first >= 64) {
            const int hop = (at - first) >> 6;
            first += hop * 64;
            if (hop > 1) next = load(first, lane);
            cur = settle(next);
            next = load(first + 64, lane);
        }
        return __builtin_amdgcn_readlane(cur, at - first);
    }
};

// fp32 values as sums of three bf16 values, x = h + m + l: each takes the next eight significant bits,
// cut, not rounded, so that the sum is exact and h does not overflow.  Products of two such sums leave out
// m l, l m and l l, at most 2^-21 of the product and 2^-23 on the average.
struct Planes {
    bf16x8 h, m, l;
};
__device__ __forceinline__ Planes split8(const float (&x)[8]) {
    u32x4 h, m, l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t a[2], b[2], c[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float v = x[2 * j + e];
            a[e] = __float_as_uint(v) & 0xffff0000u;
            const float r = v - __uint_as_float(a[e]);
            b[e] = __float_as_uint(r) & 0xffff0000u;
            c[e] = __float_as_uint(r - __uint_as_float(b[e]));
        }
        h[j] = __builtin_amdgcn_perm(a[1], a[0], 0x07060302u);   // the upper halves
        m[j] = __builtin_amdgcn_perm(b[1], b[0], 0x07060302u);
        l[j] = __builtin_amdgcn_perm(c[1], c[0], 0x07060302u);
    }
    return Planes{__builtin_bit_cast(bf16x8, h), __builtin_bit_cast(bf16x8, m), __builtin_bit_cast(bf16x8, l)};
}

constexpr float kMoveAt = 65536.f;

// Factor 1 / l of a row and its log-sum-exp from (m, l).  No key seen, or only
// logits of -inf: zeros and -inf.  A reference of +inf stands for an infinite logit: NaN.
__device__ __forceinline__ void row_result(float m, float l, float* inv, float* lse) {
    if (m == INFINITY) l = __builtin_nanf("");
    *inv = l == 0.f ? 0.f : 1.f / l;
    *lse = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// lse, and the accumulator input that the weights' products start from (see k_cache_weight): a row
// without weights adds none.
__device__ __forceinline__ void put_lse(const AttendArgs& a, int64_t row, float lse) {
    a.lse[row] = lse;
    if (a.off) a.off[row] = lse == -INFINITY ? -INFINITY : lse * (-kLog2e / a.c2);
}

}  // namespace vp
