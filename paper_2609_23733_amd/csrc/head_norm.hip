// Norm of every head's row over its 64 features, and rotary positions, in one pass; its gradient.
//
// With n = (x - mean) / rms (layer) or x / rms, rms^2 = mean (x - mean)^2 + eps or mean x^2 + eps:
//   y = R (n gain + bias),  R the rotation by the token's positions.
// Gradient, from g = dL/dy: h = R^T g,
//   dgain = sum h n,  dbias = sum h  (over tokens, and over heads that share them),
//   z = h gain,  dx = (z - [mean z] - n mean(n z)) / rms   ([..]: layer only).
// Both passes are bound by memory: x read and y written once; x and g read and dx written.  Eight lanes share a
// row, so its sums are three exchanges between neighbouring lanes.
#include "rotary_device.hpp"

namespace vp {

// hs threads of eight share a token; each takes every hs-th head, two at a time: their loads are issued together
// (y may be x, so no load moves over a store by itself).  10,992 tokens of 16 heads, bf16: 12.8 us, 3.5 TB/s; 43,968 tokens
// (stores past the caches) 42.5 us, 4.2 TB/s, with two threads a token; with eight 50, with one 45; four heads at a time 46.8.
template <typename T, bool INTER, bool VEC, bool NT>
__global__ __launch_bounds__(256) void k_norm_rotary(const T* x, int64_t x_stride, T* y, int64_t y_stride,
                                                     int Tn, int H, int hs, NormArgs nm, RotArgs r) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id & 7), h0 = (int)((id >> 3) % hs);
    const int64_t t = (id >> 3) / hs;
    if (t >= Tn) return;
    HeadTurn<T, INTER, VEC> w;
    w.places(r, c);
    const T* xr = x + t * x_stride;
    T* yr = y + t * y_stride;
    float f[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (h0 + k * hs < H) w.load(xr + (h0 + k * hs) * kD, f[k]);
    Affine p;
    p.set(nm, w, h0);
    w.angles(r, t, c);
    for (int h = h0; h < H; h += 2 * hs) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int hk = h + k * hs;
            if (hk >= H) break;
            if (nm.per_head && hk > h0) p.set(nm, w, hk);
            normalise(nm, f[k]);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(f[k][e], p.gain[e], p.bias[e]);
            w.turn(v);
            if (hk + 2 * hs < H) w.load(xr + (hk + 2 * hs) * kD, f[k]);
            w.template store<NT>(yr + hk * kD, v);
        }
    }
}

// The gradient.  Row slots of eight lanes, 32 a workgroup: slot s takes heads s % hs, s % hs + hs, .. of tokens s / hs,
// s / hs + slots / hs, ..; with a gain per head hs = H, so that a slot keeps to one head.  A slot's
// eight lanes each sum their features' gradients over all its rows; a workgroup's slots (of one head) meet in LDS,
// the workgroups' sums in k_norm_grad_join, in an order that T and H fix.  43,968 tokens of 16 heads, bf16: 56.4 us, 4.8
// TB/s, what a copy reaches.
template <typename T, bool INTER, bool VEC, bool NT>
__global__ __launch_bounds__(256) void k_norm_rotary_grad(const T* __restrict__ x, int64_t x_stride,
                                                          const T* __restrict__ g, int64_t g_stride,
                                                          T* __restrict__ dx, int Tn, int H, int hs, NormArgs nm,
                                                          RotArgs r, float* __restrict__ part) {
    const int c = threadIdx.x & 7, row = threadIdx.x >> 3;
    const int slot = blockIdx.x * 32 + row, h0 = slot % hs;
    const int t0 = slot / hs, tstep = gridDim.x * 32 / hs;
    HeadTurn<T, INTER, VEC> w;
    w.places(r, c);
    Affine p;
    p.set(nm, w, h0);
    float dg[8] = {}, db[8] = {};
    for (int t = t0; t < Tn; t += tstep) {
        const T *xr = x + t * x_stride, *gr = g + t * g_stride;
        float f[8], h[8], fn[8], hn[8];
        w.load(xr + h0 * kD, fn);
        w.load(gr + h0 * kD, hn);
        w.angles(r, t, c);
        for (int hd = h0; hd < H; hd += hs) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = fn[e], h[e] = hn[e];
            if (hd + hs < H) {
                w.load(xr + (hd + hs) * kD, fn);
                w.load(gr + (hd + hs) * kD, hn);
            }
            const float rinv = normalise(nm, f);
            w.turn_back(h);
            float z[8], sz = 0.f, sfz = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dg[e] = fmaf(h[e], f[e], dg[e]);
                db[e] += h[e];
                z[e] = h[e] * p.gain[e];
                sz += z[e];
                sfz = fmaf(f[e], z[e], sfz);
            }
            if (dx) {
                sfz = sum8(sfz) * (1.f / kD);
                sz = nm.layer ? sum8(sz) * (1.f / kD) : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = (z[e] - sz - f[e] * sfz) * rinv;
                w.template store<NT>(dx + ((int64_t)t * H + hd) * kD, z);
            }
        }
    }
    if (!part) return;
    __shared__ float s[32][8][17];   // (17: lanes of a row meet different banks)
#pragma unroll
    for (int e = 0; e < 8; ++e) s[row][c][e] = dg[e], s[row][c][8 + e] = db[e];
    __syncthreads();
    const int m = nm.per_head ? (H < 32 ? H : 32) : 1;   // heads of a workgroup
    for (int i = threadIdx.x; i < m * 128; i += 256) {
        const int k = i & 15, cc = (i >> 4) & 7, hd = i >> 7;
        float sum = 0.f;
        for (int j = hd; j < 32; j += m) sum += s[j][cc][k];
        part[((int64_t)blockIdx.x * m + hd) * 128 + cc * 16 + k] = sum;
    }
}

// Sums over the workgroups in 64 bits: 16 of the 128 sums of a head, 64 threads each, whose loads are issued sixteen at a
// time (the parts of 1,024 workgroups at once: they come from other XCDs' caches, so every round of loads waits for
// memory).  (Feature of lane c's e-th sum: the lanes' places once more.)
template <bool INTER, bool VEC>
__global__ __launch_bounds__(1024) void k_norm_grad_join(const float* __restrict__ part, int blocks, int m, int H, int per_head,
                                                         RotArgs r, float* __restrict__ dgain, float* __restrict__ dbias) {
    constexpr int kGroups = 64, kOnce = 16;
    const int k = threadIdx.x & 15, grp = threadIdx.x >> 4, c = blockIdx.y, h = blockIdx.x;
    const float* mine = part + c * 16 + k;
    double sum = 0.;
    // With sums per head, slot i of workgroup b has head (32 b + i) % H: i = (h - 32 b) mod H, if the workgroup has it.
    const int step = per_head ? 32 * kGroups % H : 0;
    int i = per_head ? ((h - 32 * grp) % H + H) % H : 0;
    for (int b = grp; b < blocks; b += kGroups * kOnce) {
        float v[kOnce];
#pragma unroll
        for (int j = 0; j < kOnce; ++j) {
            const int bj = b + kGroups * j;
            const bool have = bj < blocks && i < m;
            v[j] = mine[have ? ((int64_t)bj * m + i) * 128 : 0];
            v[j] = have ? v[j] : 0.f;
            i -= step;
            i += i < 0 ? H : 0;
        }
#pragma unroll
        for (int j = 0; j < kOnce; ++j) sum += (double)v[j];
    }
    __shared__ double s[kGroups][17];
    s[grp][k] = sum;
    __syncthreads();
    if (grp >= 8) return;
#pragma unroll
    for (int j = 8; j < kGroups; j += 8) sum += s[grp + j][k];
    s[grp][k] = sum;
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int j = 1; j < 8; ++j) sum += s[j][k];
    HeadTurn<float, INTER, VEC> w;
    w.places(r, c);
    const int e = k & 7;
    int at;
    if constexpr (VEC) {
        at = INTER ? w.lo + e : e & 1 ? w.hi + (e >> 1) : w.lo + (e >> 1);
    } else {
        at = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q == e >> 1) at = e & 1 ? w.i1[q] : w.i0[q];
    }
    float* out = k < 8 ? dgain : dbias;
    if (out) out[h * kD + at] = (float)sum;
}

// ------------------------------------------------------------------ launchers

// (T, INTER, VEC) of a call
#define NORM_GO(KERNEL, NTV, ...)                                                                     \
    do {                                                                                              \
        const bool vec = pairs_in_fours(r), inter = r.layout == 0;                                    \
        if (dtype == DT_BF16) {                                                                       \
            typedef bf16 T_;                                                                          \
            if (inter) { if (vec) KERNEL(T_, true, true, NTV); else KERNEL(T_, true, false, false); } \
            else { if (vec) KERNEL(T_, false, true, NTV); else KERNEL(T_, false, false, false); }     \
        } else {                                                                                      \
            typedef float T_;                                                                         \
            if (inter) { if (vec) KERNEL(T_, true, true, NTV); else KERNEL(T_, true, false, false); } \
            else { if (vec) KERNEL(T_, false, true, NTV); else KERNEL(T_, false, false, false); }     \
        }                                                                                             \
    } while (0)

static bool past_caches(int dtype, int64_t T, int H) {
    return T * H * kD * (dtype == DT_BF16 ? 2 : 4) > ((int64_t)32 << 20);
}

void launch_norm_rotary(int dtype, const void* x, int64_t x_stride, void* y, int64_t y_stride, int T,
                        int H, const NormArgs& nm, const RotArgs& r, hipStream_t st) {
    const bool nt = past_caches(dtype, T, H);
    const int hs = head_split(T, H, nt ? 512 * 1024 : 128 * 1024);
    const dim3 grid((unsigned)(((int64_t)T * hs * 8 + 255) / 256));
#define GO(TT, IN, VE, NTV)                                                                                    \
    hipLaunchKernelGGL((k_norm_rotary<TT, IN, VE, NTV>), grid, dim3(256), 0, st, (const TT*)x, x_stride, (TT*)y, \
                       y_stride, T, H, hs, nm, r)
    if (nt) NORM_GO(GO, true);
    else NORM_GO(GO, false);
#undef GO
}

// Workgroups of the gradient: four a compute unit (43,968 tokens of 16 heads, bf16: 56.4 us and 4.3 for the join of their
// parts; two 70.5 and 4.0, eight 53.2 and 6.8), fewer where rows are few; with a gain per head their 32
// slots each make whole turns through the heads.
static int norm_grad_blocks(int T, int H, int per_head) {
    int64_t n = ((int64_t)T * H + 31) / 32;
    n = n < 1 ? 1 : n < 1024 ? n : 1024;
    if (!per_head) return (int)n;
    int turn = H;   // H / gcd(H, 32)
    for (int k = 0; k < 5 && turn % 2 == 0; ++k) turn /= 2;
    return (int)((n + turn - 1) / turn * turn);
}
size_t norm_grad_part_bytes(int T, int H, int per_head) {
    return (size_t)norm_grad_blocks(T, H, per_head) * (per_head ? (H < 32 ? H : 32) : 1) * 128 * sizeof(float);
}

void launch_norm_rotary_grad(int dtype, const void* x, int64_t x_stride, const void* g, int64_t g_stride,
                             void* dx, float* dgain, float* dbias, int T, int H, const NormArgs& nm,
                             const RotArgs& r, float* part, hipStream_t st) {
    const int blocks = norm_grad_blocks(T, H, nm.per_head), m = nm.per_head ? (H < 32 ? H : 32) : 1;
    int hs = H;
    if (!nm.per_head) {   // a divisor of the row slots
        hs = 1;
        while (hs * 2 <= H && hs < 32 && (int64_t)T * hs < blocks * 32) hs *= 2;
    }
    if (!dgain && !dbias) part = nullptr;
    const bool nt = past_caches(dtype, T, H);
#define GO(TT, IN, VE, NTV)                                                                                           \
    hipLaunchKernelGGL((k_norm_rotary_grad<TT, IN, VE, NTV>), dim3(blocks), dim3(256), 0, st, (const TT*)x, x_stride, \
                       (const TT*)g, g_stride, (TT*)dx, T, H, hs, nm, r, part)
    if (nt) NORM_GO(GO, true);
    else NORM_GO(GO, false);
#undef GO
    if (!part) return;
    const dim3 grid(nm.per_head ? H : 1, 8);
#define GO(IN, VE) hipLaunchKernelGGL((k_norm_grad_join<IN, VE>), grid, dim3(1024), 0, st, (const float*)part, blocks, m, H, nm.per_head, r, dgain, dbias)
    const bool vec = pairs_in_fours(r);
    if (r.layout == 0) { if (vec) GO(true, true); else GO(true, false); }
    else { if (vec) GO(false, true); else GO(false, false); }
#undef GO
}

}  // namespace vp
