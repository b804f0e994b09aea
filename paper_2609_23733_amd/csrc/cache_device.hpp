// Paged key-value cache: what its kernels share (host and device).
//
// A pool of pages holds K, V [npages, Hkv, page, 64] and, per slot, the attention weight its key
// has gathered and the number of its token (stamp), [npages, Hkv, page].  Slot s of sequence b is
// slot s % page of page table[b][s / page].  A call's new tokens are rows q_start[b] ..
// q_start[b + 1] - 1 of its Q, K and V, and lie in the last slots of their sequence:
// length[b] counts them.
#pragma once

#include "vp_device.hpp"

namespace vp {

struct CacheArgs {
    int dtype;
    void *K, *V;
    float* weight;           // may be null
    int32_t* stamp;          // may be null
    int64_t npages;
    int page_log2, Hkv;
    const int32_t* table;    // [B, max_pages]
    int max_pages;
    const int32_t* length;   // [B]
    const int32_t* seen;     // [B], append and eviction only
    const int32_t* q_start;  // [B + 1]
    int B, T, max_q, max_len;
};

struct AttendArgs {
    CacheArgs c;
    int Hq, G;               // query heads, query heads per key head
    const void* Q;           // [T, Hq, 64], tokens q_stride elements apart
    int64_t q_stride;
    int causal;
    float c2;                // scale * log2 e
    void* O;                 // [T, Hq, 64]
    float* lse;              // [T, Hq]
    float* weight_out;       // null: weights are not gathered
    int wide;                // kernel variant
    int row_tiles, nsplit, chunk;
    float *part, *part_ml;   // ranges' results [nsplit, T * Hq, 64], references and sums [nsplit, T * Hq, 2]
    float* logits;           // null, or [T * Hq, logit_stride]: kept for the weights
    int64_t logit_stride;
    float* off;              // null, or [T * Hq]: -lse log2 e / c2, for the weights
};

struct AppendArgs {
    CacheArgs c;
    int Hq;
    const void *Q, *Kn, *Vn;
    void* Qo;
    int64_t q_stride, k_stride, v_stride;
};

struct RotArgs {
    const int32_t* pos;      // [T, axes]
    const uint64_t* freq;    // [dim / 2]
    int dim, axes, layout;   // layout 0: interleaved, 1: half
    float mag, sign;
};

struct EvictArgs {
    CacheArgs c;             // weight and stamp: as they are; table, length, seen
    int keep, sink, recent;
    float* weight_out;
    int32_t *stamp_out, *length_out;
    void* ws;
};

// Sequence b of a call, with every number clamped to what the host checked
// (counts in device memory that are out of range select fewer tokens or
// slots, never memory outside the arrays).
struct CacheSeq {
    int q0;    // first row
    int n;     // new tokens
    int nq;    // of these, the ones the launch covers (n <= max_q: all)
    int len;   // slots in use
};
__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ int cache_length(const CacheArgs& a, int b) {
    const int cap = a.max_pages << a.page_log2;
    return clampi(a.length[b], 0, cap < a.max_len ? cap : a.max_len);
}
__device__ __forceinline__ CacheSeq cache_seq(const CacheArgs& a, int b) {
    CacheSeq s;
    s.q0 = clampi(a.q_start[b], 0, a.T);
    s.n = clampi(a.q_start[b + 1], s.q0, a.T) - s.q0;
    s.nq = s.n < a.max_q ? s.n : a.max_q;
    s.len = cache_length(a, b);
    return s;
}
// Slots that token i of the chunk sees.
__device__ __forceinline__ int cache_visible(const CacheSeq& s, int causal, int i) {
    return causal ? clampi(s.len - s.n + i + 1, 0, s.len) : s.len;
}

void launch_rotary(int dtype, const void* x, int64_t x_stride, void* y, int64_t y_stride, int T,
                   int H, const RotArgs& r, hipStream_t st);
void launch_cache_append(const AppendArgs& a, const RotArgs& r, hipStream_t st);
void attend_plan(AttendArgs* a);
int attend_rows(const AttendArgs& a);
size_t attend_part_rows(const AttendArgs& a);
size_t attend_logits(const AttendArgs& a);
void launch_cache_attend(const AttendArgs& a, hipStream_t st);
size_t evict_ws_bytes(int B, int Hkv, int max_len);
void launch_cache_evict(const EvictArgs& a, hipStream_t st);

}  // namespace vp
