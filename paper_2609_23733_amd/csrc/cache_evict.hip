// Eviction from a paged key-value cache by gathered attention weight.
//
// Of the len slots of a sequence and key head, n = min(len, keep) stay: protected ones first
// (stamp below `sink`, or among the latest `recent` of the sequence's `seen` tokens), then
// by weight, the larger first, NaN before all numbers; among equals the lower slot.  Kept slots below n
// stay where they are; the j-th kept slot from n on moves into the j-th slot below n that is not kept.
// (Attention does not depend on the order of the slots, and sources and destinations never
// overlap: every move runs at once, in place, and slots that need not move are not
// touched.)
//
// Selection: each slot's rank as a 32-bit key, the n-th largest key by counting digits (11, 11
// and 10 bits) over the slots, in the order of the keys' top digits; then, with `above` the slots
// whose key is larger and `ties` those whose key is equal, slot s is kept if it is above or one of
// the first n - #above ties.  The kept slots before s, kb(s), follow from prefix counts, and so
// do both lists: hole s is number s - kb(s), mover s number kb(s) - kb(n).
#include "cache_device.hpp"

namespace vp {

constexpr int kEvChunk = 4096;          // slots per workgroup of the counting passes
constexpr int kEvBins = 2048;

struct EvictWs {
    uint32_t* key;      // [B * Hkv, cap]
    int32_t *hist;      // [B * Hkv, 3, kEvBins]
    int32_t *count;     // [B * Hkv, chunks, 2]: above, ties
    int32_t *hole, *mover;   // [B * Hkv, cap]
    int32_t *kbn, *left;     // [B * Hkv]: kept slots below n; n
    uint32_t* bound;         // [B * Hkv, 4]: after pass 1 the top digit and what is wanted of it; then (2, 3)
                             // two digits; then (0, 1) the n-th largest key, its ties that are kept
    int cap, chunks;
};

__host__ __device__ inline size_t ev_up(size_t x) { return (x + 255) & ~(size_t)255; }

static EvictWs evict_layout(int B, int Hkv, int max_len, void* ws, size_t* total) {
    EvictWs w;
    const size_t bh = (size_t)B * Hkv;
    w.chunks = max_len > 0 ? (max_len + kEvChunk - 1) / kEvChunk : 1;
    w.cap = w.chunks * kEvChunk;
    size_t off = 0;
    char* p = (char*)ws;
    auto take = [&](size_t bytes) {
        char* at = p + off;
        off = ev_up(off + bytes);
        return at;
    };
    w.hist = (int32_t*)take(bh * 3 * kEvBins * 4);
    w.key = (uint32_t*)take(bh * w.cap * 4);
    w.count = (int32_t*)take(bh * w.chunks * 8);
    w.hole = (int32_t*)take(bh * w.cap * 4);
    w.mover = (int32_t*)take(bh * w.cap * 4);
    w.kbn = (int32_t*)take(bh * 4);
    w.left = (int32_t*)take(bh * 4);
    w.bound = (uint32_t*)take(bh * 16);
    if (total) *total = off;
    return w;
}

size_t evict_ws_bytes(int B, int Hkv, int max_len) {
    size_t n;
    evict_layout(B, Hkv, max_len, nullptr, &n);
    return n;
}

// Larger keys are kept first.  Weights keep their order as integers (-0 counts as 0).
__device__ __forceinline__ uint32_t evict_key(float w, int stamp, int sink, int64_t latest) {
    if (stamp < sink || stamp >= latest) return 0xffffffffu;
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int64_t slot_at(const CacheArgs& c, int b, int hk, int slot) {
    const int page = c.table[(int64_t)b * c.max_pages + (slot >> c.page_log2)];
    if (page < 0 || page >= c.npages) return -1;
    return (((int64_t)page * c.Hkv + hk) << c.page_log2) + (slot & ((1 << c.page_log2) - 1));
}

__global__ __launch_bounds__(256) void k_evict_clear(int32_t* hist, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) hist[i] = 0;
}

// Digit that holds the need-th largest key of a histogram, and how many of that digit are still
// wanted.  All 256 threads; s: 256 + 2 ints of LDS.
__device__ __forceinline__ void find_digit(const int32_t* hist, int bins, int need, int* digit, int* left,
                                           int* s) {
    const int t = threadIdx.x, per = bins / 256, lane = t & 63, wv = t >> 6;
    int own[kEvBins / 256], sum = 0;
#pragma unroll
    for (int j = 0; j < kEvBins / 256; ++j) {
        own[j] = j < per ? hist[bins - 1 - (t * per + j)] : 0;   // from the largest digit down
        sum += own[j];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(inc, o);
        if (lane >= o) inc += v;
    }
    __syncthreads();
    if (lane == 63) s[wv] = inc;
    __syncthreads();
    int before = inc - sum;
    for (int v = 0; v < wv; ++v) before += s[v];
    if (before < need && before + sum >= need) {
#pragma unroll
        for (int j = 0; j < kEvBins / 256; ++j) {
            if (before < need && before + own[j] >= need) {
                s[8] = bins - 1 - (t * per + j);
                s[9] = need - before;
            }
            before += own[j];
        }
    }
    __syncthreads();
    *digit = s[8];
    *left = s[9];
    __syncthreads();
}

// Keys of the chunk's slots, four in a row per thread and step (a page holds at least 16), all
// loads of a thread issued before the first is used.
constexpr int kEvSteps = kEvChunk / 1024;
__device__ __forceinline__ void chunk_keys(const EvictArgs& a, int b, int hk, int s0, int s1, uint32_t (&k)[kEvSteps][4]) {
    int64_t at[kEvSteps];
    f32x4 w[kEvSteps];
    typedef int32_t i32x4 __attribute__((__vector_size__(16), aligned(4)));
    typedef float f32x4u __attribute__((__vector_size__(16), aligned(4)));
    i32x4 st[kEvSteps];
    const int64_t latest = (int64_t)a.c.seen[b] - a.recent;
#pragma unroll
    for (int j = 0; j < kEvSteps; ++j) {
        const int s = s0 + j * 1024 + threadIdx.x * 4;
        at[j] = s < s1 ? slot_at(a.c, b, hk, s) : -1;
    }
#pragma unroll
    for (int j = 0; j < kEvSteps; ++j) {
        const int64_t p = at[j] >= 0 ? at[j] : 0;   // (slot 0 of the pool for those without a page)
        w[j] = *(const f32x4u*)(a.c.weight + p);
        st[j] = *(const i32x4*)(a.c.stamp + p);
    }
#pragma unroll
    for (int j = 0; j < kEvSteps; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            k[j][e] = at[j] >= 0 ? evict_key(w[j][e], st[j][e], a.sink, latest) : 0;
}

// Counting pass PASS (0: keys made, top 11 bits; 1: next 11; 2: last 10).
template <int PASS>
__global__ __launch_bounds__(256) void k_evict_digit(EvictArgs a, EvictWs w) {
    const int bh = blockIdx.y, hk = bh % a.c.Hkv, b = bh / a.c.Hkv;
    const int len = cache_length(a.c, b), n = len < a.keep ? len : a.keep;
    const int s0 = blockIdx.x * kEvChunk, s1 = s0 + kEvChunk < len ? s0 + kEvChunk : len;
    if (s0 >= len || n == len) return;
    __shared__ int bins[kEvBins];
    __shared__ int tmp[16];
    int32_t* hist = w.hist + (int64_t)bh * 3 * kEvBins;
    uint32_t* key = w.key + (int64_t)bh * w.cap;
    uint32_t k[kEvSteps][4];
    if (PASS == 0) {
        chunk_keys(a, b, hk, s0, s1, k);
#pragma unroll
        for (int j = 0; j < kEvSteps; ++j) {
            const u32x4 v = {k[j][0], k[j][1], k[j][2], k[j][3]};
            *(u32x4*)(key + s0 + j * 1024 + threadIdx.x * 4) = v;   // (cap is whole chunks)
        }
    } else {
#pragma unroll
        for (int j = 0; j < kEvSteps; ++j) {
            const u32x4 v = *(const u32x4*)(key + s0 + j * 1024 + threadIdx.x * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[j][e] = v[e];
        }
    }
    for (int i = threadIdx.x; i < kEvBins; i += 256) bins[i] = 0;
    uint32_t prefix = 0;
    int need, d;
    uint32_t* bound = w.bound + 4 * (int64_t)bh;
    if (PASS == 1) {
        find_digit(hist, 2048, n, &d, &need, tmp);
        prefix = d;
        if (blockIdx.x == 0 && threadIdx.x == 0) bound[0] = prefix, bound[1] = need;
    }
    if (PASS == 2) {
        find_digit(hist + kEvBins, 2048, (int)bound[1], &d, &need, tmp);
        prefix = bound[0] << 11 | d;
        if (blockIdx.x == 0 && threadIdx.x == 0) bound[2] = prefix, bound[3] = need;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEvSteps; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = k[j][e];
            if (s0 + j * 1024 + (int)threadIdx.x * 4 + e >= s1) continue;
            if (PASS == 0) atomicAdd(&bins[x >> 21], 1);
            if (PASS == 1 && x >> 21 == prefix) atomicAdd(&bins[(x >> 10) & 2047], 1);
            if (PASS == 2 && x >> 10 == prefix) atomicAdd(&bins[x & 1023], 1);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < kEvBins; i += 256)
        if (bins[i]) atomicAdd(hist + PASS * kEvBins + i, bins[i]);
}

// Per chunk: slots above the bound, and ties.
__global__ __launch_bounds__(256) void k_evict_count(EvictArgs a, EvictWs w) {
    const int bh = blockIdx.y, b = bh / a.c.Hkv;
    const int len = cache_length(a.c, b), n = len < a.keep ? len : a.keep;
    const int s0 = blockIdx.x * kEvChunk, s1 = s0 + kEvChunk < len ? s0 + kEvChunk : len;
    if (s0 >= len || n == len) return;
    __shared__ int tmp[16];
    // the n-th largest key and the number of its ties that are kept
    int ties, d;
    const uint32_t* two = w.bound + 4 * (int64_t)bh + 2;
    find_digit(w.hist + ((int64_t)bh * 3 + 2) * kEvBins, 1024, (int)two[1], &d, &ties, tmp);
    const uint32_t bound = two[0] << 10 | d;
    const uint32_t* key = w.key + (int64_t)bh * w.cap;
    int above = 0, tie = 0;
#pragma unroll 4
    for (int s = s0 + threadIdx.x; s < s1; s += 256) {
        const uint32_t k = key[s];
        above += k > bound;
        tie += k == bound;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        above += __shfl_xor(above, o);
        tie += __shfl_xor(tie, o);
    }
    if ((threadIdx.x & 63) == 0) {
        tmp[threadIdx.x >> 6] = above;
        tmp[4 + (threadIdx.x >> 6)] = tie;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int32_t* c = w.count + ((int64_t)bh * w.chunks + blockIdx.x) * 2;
        c[0] = tmp[0] + tmp[1] + tmp[2] + tmp[3];
        c[1] = tmp[4] + tmp[5] + tmp[6] + tmp[7];
        if (blockIdx.x == 0) w.bound[4 * (int64_t)bh] = bound, w.bound[4 * (int64_t)bh + 1] = ties;
    }
}

// Lists of holes and movers, 64 slots at a time, one per lane of a wave: the entries of a step lie side
// by side (a thread with a run of slots of its own scatters them).
__device__ __forceinline__ int lanes_before(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
__device__ __forceinline__ void count_step(uint32_t k, bool in, uint32_t bound, int* above, int* tie) {
    *above += __popcll(__builtin_amdgcn_ballot_w64(in && k > bound));
    *tie += __popcll(__builtin_amdgcn_ballot_w64(in && k == bound));
}
// `above`, `tie`: slots above the bound and ties before the step's.
__device__ __forceinline__ void list_step(uint32_t k, int s, bool in, int n, uint32_t bound, int ties, int* above, int* tie,
                                          int32_t* hole, int32_t* mover, int32_t* kbn) {
    const bool up = in && k > bound, eq = in && k == bound;
    const uint64_t mu = __builtin_amdgcn_ballot_w64(up), me = __builtin_amdgcn_ballot_w64(eq);
    const int before = *tie + lanes_before(me), kb = *above + lanes_before(mu) + (before < ties ? before : ties);
    const bool kept = up || (eq && before < ties);
    if (in) {
        if (s == n) *kbn = kb;
        if (s < n && !kept) hole[s - kb] = s;
        if (s >= n && kept) mover[kb] = s;
    }
    *above += __popcll(mu);
    *tie += __popcll(me);
}

// Weights and stamps of slots s0 + 4 t, s0 + 4 (t + step), .. below e1 of thread t, four loads at once, as
// they are, for output arrays of their own.
struct KeptCopy {
    typedef int32_t i32x4 __attribute__((__vector_size__(16), aligned(4)));
    typedef float f32x4u __attribute__((__vector_size__(16), aligned(4)));
    static constexpr int kAtOnce = 4;
    int64_t at[kAtOnce];
    f32x4u w[kAtOnce];
    i32x4 t[kAtOnce];
    __device__ __forceinline__ void load(const EvictArgs& a, int b, int hk, int s, int step, int e1) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) at[j] = s + j * step < e1 ? slot_at(a.c, b, hk, s + j * step) : -1;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int64_t p = at[j] >= 0 ? at[j] : 0;
            w[j] = *(const f32x4u*)(a.c.weight + p);
            t[j] = *(const i32x4*)(a.c.stamp + p);
        }
    }
    __device__ __forceinline__ void store(const EvictArgs& a, int s, int step, int e1) const {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (at[j] < 0) continue;
            const int left = e1 - (s + j * step);
            if (left >= 4) {
                *(f32x4u*)(a.weight_out + at[j]) = w[j];
                *(i32x4*)(a.stamp_out + at[j]) = t[j];
                continue;
            }
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < left) {
                    a.weight_out[at[j] + e] = w[j][e];
                    a.stamp_out[at[j] + e] = t[j][e];
                }
        }
    }
};

// The lists, and the weights and stamps of the slots that stay.  Everything that does not depend on the
// counts is loaded first.
__global__ __launch_bounds__(256) void k_evict_lists(EvictArgs a, EvictWs w) {
    const int bh = blockIdx.y, hk = bh % a.c.Hkv, b = bh / a.c.Hkv;
    const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6);
    constexpr int kRun = kEvChunk / 4, kSteps = kRun / 64;   // slots per wave
    static_assert(kEvChunk == KeptCopy::kAtOnce * 1024, "a chunk's copies at once");
    const int s0 = blockIdx.x * kEvChunk, p0 = s0 + wv * kRun;
    const uint32_t* key = w.key + (int64_t)bh * w.cap;
    const int32_t* cnt = w.count + (int64_t)bh * w.chunks * 2;
    uint32_t k[kSteps];   // (cap is whole chunks)
#pragma unroll
    for (int j = 0; j < kSteps; ++j) k[j] = key[p0 + 64 * j + lane];
    const uint32_t bound = w.bound[4 * (int64_t)bh];
    const int ties = (int)w.bound[4 * (int64_t)bh + 1];
    int above = 0, tie = 0;   // counts of the chunks before
    for (int c = lane; c < (int)blockIdx.x; c += 64) above += cnt[2 * c], tie += cnt[2 * c + 1];
    const int len = cache_length(a.c, b), n = len < a.keep ? len : a.keep;
    const int s1 = s0 + kEvChunk < len ? s0 + kEvChunk : len;
    if (blockIdx.x == 0 && t == 0) {
        w.left[bh] = n;
        if (n == len) w.kbn[bh] = n;   // nothing moves
    }
    if (s0 >= len) return;
    const bool same = a.weight_out == a.c.weight && a.stamp_out == a.c.stamp;
    const int e1 = s1 < n ? s1 : n;
    KeptCopy copy;
    if (!same && s0 < e1) copy.load(a, b, hk, s0 + t * 4, 1024, e1);
    if (n < len) {
        __shared__ int tmp[8];
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            above += __shfl_xor(above, o);
            tie += __shfl_xor(tie, o);
        }
        int ma = 0, mt = 0;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) count_step(k[j], p0 + 64 * j + lane < s1, bound, &ma, &mt);
        if (lane == 0) tmp[wv] = ma, tmp[4 + wv] = mt;
        __syncthreads();
        for (int v = 0; v < wv; ++v) above += tmp[v], tie += tmp[4 + v];
        int32_t *hole = w.hole + (int64_t)bh * w.cap, *mover = w.mover + (int64_t)bh * w.cap;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const int s = p0 + 64 * j + lane;
            list_step(k[j], s, s < s1, n, bound, ties, &above, &tie, hole, mover, w.kbn + bh);
        }
    }
    if (!same && s0 < e1) copy.store(a, s0 + t * 4, 1024, e1);
}

// ------------------------------------------------------------------------
// Short sequences (up to kEvSmall slots): one workgroup per sequence and head does the counting and the
// lists with its keys in LDS; one launch in place of six.
// Bound by its own chain of steps (8,244 slots: loads 3 us, the first count 2, scans and further counts
// 5, lists 4).  With the moves, one sequence of 16 heads: 6,000 slots 16 us, 31 in six launches as below, 16,000
// slots 28 and 35.
// ------------------------------------------------------------------------
constexpr int kEvSmall = 16384, kEvThreads = 1024;

__global__ __launch_bounds__(kEvThreads) void k_evict_small(EvictArgs a, EvictWs w) {
    const int bh = blockIdx.x, hk = bh % a.c.Hkv, b = bh / a.c.Hkv;
    const int len = cache_length(a.c, b), n = len < a.keep ? len : a.keep;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6;
    if (t == 0) {
        w.left[bh] = n;
        if (n == len) w.kbn[bh] = n;   // nothing moves
    }
    const bool same = a.weight_out == a.c.weight && a.stamp_out == a.c.stamp;
    if (n < len) {
        __shared__ __attribute__((aligned(16))) uint32_t key[kEvSmall];
        __shared__ int bins[kEvBins];
        __shared__ int tmp[40];
        const int64_t latest = (int64_t)a.c.seen[b] - a.recent;
        typedef int32_t i32x4 __attribute__((__vector_size__(16), aligned(4)));
        typedef float f32x4u __attribute__((__vector_size__(16), aligned(4)));
        // ---- keys, four slots per thread and step
        constexpr int kSteps = kEvSmall / (4 * kEvThreads);
        int64_t at[kSteps];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const int s = (j * kEvThreads + t) * 4;
            at[j] = s < len ? slot_at(a.c, b, hk, s) : -1;
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const int s = (j * kEvThreads + t) * 4;
            if (s >= len) break;
            u32x4 k = {0u, 0u, 0u, 0u};
            if (at[j] >= 0) {
                const f32x4u x = *(const f32x4u*)(a.c.weight + at[j]);
                const i32x4 st = *(const i32x4*)(a.c.stamp + at[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = evict_key(x[e], st[e], a.sink, latest);
            }
            *(u32x4*)(key + s) = k;
        }
        // ---- the n-th largest: digits of 11, 11 and 10 bits
        uint32_t prefix = 0;
        int need = n;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, nb = pass == 2 ? 1024 : 2048;
            for (int i = t; i < kEvBins; i += kEvThreads) bins[i] = 0;
            __syncthreads();
            for (int s = t; s < len; s += kEvThreads) {
                const uint32_t k = key[s];
                if (pass == 0 || k >> (pass == 1 ? 21 : 10) == prefix) atomicAdd(&bins[(k >> shift) & (nb - 1)], 1);
            }
            __syncthreads();
            // the digit, two bins per thread, from the largest down
            const int own0 = 2 * t < nb ? bins[nb - 1 - 2 * t] : 0, own1 = 2 * t + 1 < nb ? bins[nb - 2 - 2 * t] : 0;
            int inc = own0 + own1;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(inc, o);
                if (lane >= o) inc += v;
            }
            if (lane == 63) tmp[wv] = inc;
            __syncthreads();
            int before = inc - own0 - own1;
#pragma unroll
            for (int v = 0; v < kEvThreads / 64; ++v) before += v < wv ? tmp[v] : 0;
            if (before < need && before + own0 + own1 >= need) {
                const bool first = before + own0 >= need;
                tmp[32] = first ? nb - 1 - 2 * t : nb - 2 - 2 * t;
                tmp[33] = need - before - (first ? 0 : own0);
            }
            __syncthreads();
            prefix = prefix << (pass == 2 ? 10 : 11) | (uint32_t)tmp[32];
            need = tmp[33];
            __syncthreads();
        }
        // ---- lists: a run of slots per wave
        const uint32_t bound = prefix;
        const int ties = need, per = (len + kEvThreads - 1) / kEvThreads * 64;
        const int p0 = __builtin_amdgcn_readfirstlane(wv) * per, p1 = p0 + per < len ? p0 + per : len;
        int ma = 0, mt = 0, above = 0, tie = 0;
        for (int q = p0; q < p1; q += 64) count_step(key[q + lane], q + lane < p1, bound, &ma, &mt);
        if (lane == 0) tmp[wv] = ma, tmp[16 + wv] = mt;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kEvThreads / 64; ++v) {
            above += v < wv ? tmp[v] : 0;
            tie += v < wv ? tmp[16 + v] : 0;
        }
        int32_t *hole = w.hole + (int64_t)bh * w.cap, *mover = w.mover + (int64_t)bh * w.cap;
        for (int q = p0; q < p1; q += 64)
            list_step(key[q + lane], q + lane, q + lane < p1, n, bound, ties, &above, &tie, hole, mover, w.kbn + bh);
    }
    if (!same)
        for (int s = 0; s < n; s += 4 * KeptCopy::kAtOnce * kEvThreads) {
            KeptCopy copy;
            copy.load(a, b, hk, s + t * 4, 4 * kEvThreads, n);
            copy.store(a, s + t * 4, 4 * kEvThreads, n);
        }
}

// The moves: eight threads per move and tensor row.
// Bound by HBM (137,400 -> 43,968 slots of 16 heads, bf16: 30 thousand moves a head, 245 MB in 47 us).
template <typename T>
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a, EvictWs w) {
    const int bh = blockIdx.y, hk = bh % a.c.Hkv, b = bh / a.c.Hkv;
    // (`length` may be `length_out`: it is not read here.)
    const int n = w.left[bh], kbn = w.kbn[bh], moves = n - kbn;
    if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) a.length_out[b] = n;
    const int c = threadIdx.x & 7;
    constexpr int kE = 16 / sizeof(T), kV = 8 * sizeof(T) / 16;
    for (int j = blockIdx.x * 32 + (threadIdx.x >> 3); j < moves; j += gridDim.x * 32) {
        const int s = w.mover[(int64_t)bh * w.cap + kbn + j], d = w.hole[(int64_t)bh * w.cap + j];
        const int64_t src = slot_at(a.c, b, hk, s), dst = slot_at(a.c, b, hk, d);
        if (src < 0 || dst < 0) continue;
        u32x4 k[kV], v[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            k[e] = *(const u32x4*)((const T*)a.c.K + src * kD + (8 * e + c) * kE);
            v[e] = *(const u32x4*)((const T*)a.c.V + src * kD + (8 * e + c) * kE);
        }
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            *(u32x4*)((T*)a.c.K + dst * kD + (8 * e + c) * kE) = k[e];
            *(u32x4*)((T*)a.c.V + dst * kD + (8 * e + c) * kE) = v[e];
        }
        if (c == 0) {
            a.weight_out[dst] = a.c.weight[src];
            a.stamp_out[dst] = a.c.stamp[src];
        }
    }
}

// The same for 8-bit codes: four threads for K's 64 bytes, four for V's.
__global__ __launch_bounds__(256) void k_evict_move8(EvictArgs a, EvictWs w) {
    const int bh = blockIdx.y, hk = bh % a.c.Hkv, b = bh / a.c.Hkv;
    const int n = w.left[bh], kbn = w.kbn[bh], moves = n - kbn;
    if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) a.length_out[b] = n;
    const int c = threadIdx.x & 7;
    char* rows = (char*)(c < 4 ? a.c.K : a.c.V) + (c & 3) * 16;
    for (int j = blockIdx.x * 32 + (threadIdx.x >> 3); j < moves; j += gridDim.x * 32) {
        const int s = w.mover[(int64_t)bh * w.cap + kbn + j], d = w.hole[(int64_t)bh * w.cap + j];
        const int64_t src = slot_at(a.c, b, hk, s), dst = slot_at(a.c, b, hk, d);
        if (src < 0 || dst < 0) continue;
        *(u32x4*)(rows + dst * kD) = *(const u32x4*)(rows + src * kD);
        if (c == 0) {
            a.weight_out[dst] = a.c.weight[src];
            a.stamp_out[dst] = a.c.stamp[src];
            a.c.scale[dst] = a.c.scale[src];
        }
    }
}

void launch_cache_evict(const EvictArgs& a, hipStream_t st) {
    EvictWs w = evict_layout(a.c.B, a.c.Hkv, a.c.max_len, a.ws, nullptr);
    const int bh = a.c.B * a.c.Hkv;
    const int64_t nh = (int64_t)bh * 3 * kEvBins;
    const dim3 grid(w.chunks, bh);
    if (a.c.max_len <= kEvSmall) {
        hipLaunchKernelGGL(k_evict_small, dim3(bh), dim3(kEvThreads), 0, st, a, w);
    } else {
        hipLaunchKernelGGL(k_evict_clear, dim3((nh + 255) / 256), dim3(256), 0, st, w.hist, nh);
        hipLaunchKernelGGL(k_evict_digit<0>, grid, dim3(256), 0, st, a, w);
        hipLaunchKernelGGL(k_evict_digit<1>, grid, dim3(256), 0, st, a, w);
        hipLaunchKernelGGL(k_evict_digit<2>, grid, dim3(256), 0, st, a, w);
        hipLaunchKernelGGL(k_evict_count, grid, dim3(256), 0, st, a, w);
        hipLaunchKernelGGL(k_evict_lists, grid, dim3(256), 0, st, a, w);
    }
    // A move for every slot past the first `keep` at most.
    int64_t most = a.c.max_len - a.keep;
    most = most < 1 ? 1 : most < a.keep ? most : a.keep;
    int64_t gx = (most + 31) / 32, cap = 8192 / bh + 1;
    if (gx > cap) gx = cap;
    if (a.c.code)
        hipLaunchKernelGGL(k_evict_move8, dim3(gx, bh), dim3(256), 0, st, a, w);
    else if (a.c.dtype == DT_BF16)
        hipLaunchKernelGGL(k_evict_move<bf16>, dim3(gx, bh), dim3(256), 0, st, a, w);
    else
        hipLaunchKernelGGL(k_evict_move<float>, dim3(gx, bh), dim3(256), 0, st, a, w);
}

}  // namespace vp
