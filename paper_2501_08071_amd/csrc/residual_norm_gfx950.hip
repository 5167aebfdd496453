// Residual RMS norm for gfx950, output in the input type or in 8 bits with scales.
//
//     h = x + r          r' = h rounded to the input type (the residual of the next layer)
//     y = h / sqrt(mean h^2 + eps) * w
//     8 bit:  s = max |y| / 448 over a row or 128 columns of it (1 where every y is 0),  y8 = e4m3(y / s)
//
// h stays in 32 bits from the addition to the last rounding.  Everything is read once and written once: 8 bytes an element
// (16-bit output) or 7 (8-bit), a few operations each, so the kernel is bound by HBM or, with few rows, by the latency of one
// load, one reduction and one store.  With g = h w and t = max |g|, the norm's factor f = 1 / sqrt(...) cancels out of the 8-bit
// values: y / s = g * 448 / t, s = f t / 448.  The sum of squares and the row's maximum therefore go through one reduction.
//
// Layout: TPR threads share a row, each holds CH chunks of 8 elements (16 bytes) in registers, chunk c of thread t at elements
// 8 (c TPR + t): a wavefront's access is 1 KiB of consecutive bytes.  128 columns are 16 neighbouring lanes.  A row length that
// is no multiple of 8 has a last chunk of 1 to 7 elements.
// Measured, bfloat16: 16384 x 4096 to 8 bits 81 us (5.8 TB/s), to 16 bits 93 us (5.8); 16 x 4096 2.9 us in a replayed graph.  A batch of 333 rows of binary16, to
// 8 bits with group scales, likewise: 4.3 us of 4096 elements, 5.1 of 5000 (512 threads instead of 256, 39 % of their places empty), 6.2 of 5001 (odd addresses).
// Rows past 32768 elements are read twice in accesses of 2 bytes: 1100 x 32776, binary16, 105 us to 16 bits and 197 to 8, where 1100 x 32768 takes 55 and 49.
// Rows of more than 16384 elements at odd addresses to 8 bits keep 13 or 14 words a thread in memory: 1024 threads have 128 registers each.
#include <hip/hip_runtime.h>
#include <cstdint>

#include "gfx950_common.h"
#include "residual_norm_launch.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // at any even address
typedef u32x2 __attribute__((aligned(1))) u32x2_any;   // at any address

constexpr float E4M3_MAX = 448.f;

template <int DT>
__device__ __forceinline__ void widen8(const u32x4& p, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = gfx950::Elem<DT>::widen((uint16_t)(p[i] & 0xFFFFu));
        f[2 * i + 1] = gfx950::Elem<DT>::widen((uint16_t)(p[i] >> 16));
    }
}
template <int DT>
__device__ __forceinline__ uint16_t narrow(float f) { return (uint16_t)gfx950::Elem<DT>::pack2(f, 0.f); }

typedef uint32_t __attribute__((aligned(1))) u32_any;
typedef uint16_t __attribute__((aligned(1))) u16_any;

// 8 elements from p, or the first `some` of them and zeros.  Of a row of 8 elements or more the last chunk's are read as the row's last
// eight and shifted down.
template <bool TAIL>
__device__ __forceinline__ u32x4 load8(const uint16_t* p, int some, int d) {
    if (!TAIL || some == 8) return *(const u32x4_any*)p;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (d >= 8) {
        v = *(const u32x4_any*)(p - (8 - some));
        const int bits = 16 * (8 - some);   // 16 to 112
        const uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
        const uint64_t a = bits < 64 ? lo >> bits | hi << (64 - bits) : hi >> (bits - 64), b = bits < 64 ? hi >> bits : 0;
        return u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < some) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    return v;
}
// (Elements of a neighbour's chunk are never stored: another thread may be about to read them, where a result lies over an input.)
template <int DT, bool TAIL>
__device__ __forceinline__ void store8(uint16_t* p, const float (&f)[8], int some) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = gfx950::Elem<DT>::pack2(f[2 * i], f[2 * i + 1]);
    if (!TAIL || some == 8) {
        *(u32x4_any*)p = v;
    } else {
        if (some & 4) *(u32x2_any*)p = u32x2{v[0], v[1]};
        if (some & 2) *(u32_any*)(p + (some & 4)) = some & 4 ? v[2] : v[0];
        if (some & 1) p[some - 1] = (uint16_t)(some == 7 ? v[3] : some == 5 ? v[2] : some == 3 ? v[1] : v[0]);
    }
}
template <bool TAIL>
__device__ __forceinline__ void store8_e4m3(uint8_t* p, const float (&f)[8], int some) {
    u32x2 v;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int t = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], t, true);
    }
    if (!TAIL || some == 8) {
        *(u32x2_any*)p = v;
    } else {
        const uint32_t rest = some & 4 ? v[1] : v[0];
        if (some & 4) *(u32_any*)p = v[0];
        if (some & 2) *(u16_any*)(p + (some & 4)) = (uint16_t)rest;
        if (some & 1) p[some - 1] = (uint8_t)(some & 2 ? rest >> 16 : rest);
    }
}

// |a| as an unsigned number orders like |a|, with NaN above infinity: its maximum keeps a NaN
__device__ __forceinline__ uint32_t magnitude(float a) { return __builtin_bit_cast(uint32_t, a) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Sum and maximum over the TPR threads of a row (TPR <= 64: lanes of one wavefront; above: the whole workgroup, through LDS).
template <int TPR, bool MAXIMUM>
__device__ __forceinline__ void reduce_row(float& s, uint32_t& t, float (&rs)[TPR > 64 ? TPR / 64 : 1], uint32_t (&rt)[TPR > 64 ? TPR / 64 : 1]) {
#pragma unroll
    for (int off = (TPR < 64 ? TPR : 64) / 2; off >= 1; off >>= 1) {
        s += __shfl_xor(s, off, 64);
        if (MAXIMUM) t = umax(t, __shfl_xor(t, off, 64));
    }
    if constexpr (TPR > 64) {
        constexpr int NW = TPR / 64;
        if ((threadIdx.x & 63) == 0) {
            rs[threadIdx.x >> 6] = s;
            if (MAXIMUM) rt[threadIdx.x >> 6] = t;
        }
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            s += rs[w];
            if (MAXIMUM) t = umax(t, rt[w]);
        }
    }
}

// The scale for a largest |g| of t (as bits) under the norm's factor f, and the two factors that take g to y / s: g * a * b.  Two,
// because 448 / t alone overflows where t is tiny.
struct Scale {
    float s, a, b;
};
__device__ __forceinline__ Scale scale_of(uint32_t tbits, float f) {
    const float t = __builtin_bit_cast(float, tbits);
    // f is 0 where the sum of squares overflowed: every finite g gives 0 then, as f * g does, and an infinite one NaN
    const float top = f == 0.f && tbits < 0x7f800000u ? 0.f : f * t;
    if (top == 0.f) return {1.f, 0.f, 0.f};
    if (top != top) return {top, top, top};   // a NaN anywhere in the row, or an infinity in this group of it
    const float a = t < 0x1p-60f ? 0x1p+60f : 1.f;
    return {top / E4M3_MAX, a, E4M3_MAX / (t * a)};
}

template <int DT, bool FP8, int TPR, int CH, bool TAIL>
__global__ __launch_bounds__(TPR > 64 ? TPR : 256) void residual_norm_kernel(const uint16_t* x, const uint16_t* r, const uint16_t* __restrict__ w,
                                                                             void* y, float* __restrict__ scale, uint16_t* r_out,
                                                                             long long n_rows, int d, int group, float eps) {
    constexpr int BLOCK = TPR > 64 ? TPR : 256, RPW = BLOCK / TPR;
    __shared__ float rs[2][TPR > 64 ? TPR / 64 : 1];
    __shared__ uint32_t rt[2][TPR > 64 ? TPR / 64 : 1];
    const int t = threadIdx.x % TPR, rin = threadIdx.x / TPR;
    // elements of chunk c that lie in the row
    auto some = [&](int c) {
        const int left = d - 8 * (c * TPR + t);
        return left < 0 ? 0 : left > 8 ? 8 : left;
    };
    // the weights, for all the rows of this thread, or, where 1024 threads have 128 registers each, for every row again
    constexpr bool HOLD = TPR < 1024;
    u32x4 pw[CH];
    auto weights = [&] {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            int off = 8 * (c * TPR + t);
            if constexpr (!HOLD) asm volatile("" : "+v"(off));   // computed here, not kept as an address per chunk over the loop
            pw[c] = u32x4{0u, 0u, 0u, 0u};
            if (some(c) > 0) pw[c] = load8<TAIL>(w + off, some(c), d);
        }
    };
    if constexpr (HOLD) weights();
    int turn = 0;
    for (long long row0 = (long long)blockIdx.x * RPW; row0 < n_rows; row0 += (long long)gridDim.x * RPW) {
        const long long row = row0 + rin;
        const size_t at = (size_t)row * d;
        u32x4 px[CH], pr[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            px[c] = pr[c] = u32x4{0u, 0u, 0u, 0u};
            const int n = some(c), off = 8 * (c * TPR + t);
            if (row < n_rows && n > 0) {
                px[c] = load8<TAIL>(x + at + off, n, d);
                if (r) pr[c] = load8<TAIL>(r + at + off, n, d);
            }
        }
        if constexpr (!HOLD && FP8) weights();
        float h[CH][8], s = 0.f;
        uint32_t top[CH], all = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float a[8];
            widen8<DT>(px[c], h[c]);
            widen8<DT>(pr[c], a);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[c][i] = r ? h[c][i] + a[i] : h[c][i];
                s = __builtin_fmaf(h[c][i], h[c][i], s);
            }
            if (r && row < n_rows && some(c) > 0) store8<DT, TAIL>(r_out + at + 8 * (c * TPR + t), h[c], some(c));
            if constexpr (FP8) {
                widen8<DT>(pw[c], a);
                top[c] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    h[c][i] *= a[i];
                    top[c] = umax(top[c], magnitude(h[c][i]));
                }
                all = umax(all, top[c]);
            }
        }
        reduce_row<TPR, FP8>(s, all, rs[turn], rt[turn]);
        turn ^= 1;
        if constexpr (!HOLD && !FP8) weights();
        const float f = 1.0f / __builtin_sqrtf(s / (float)d + eps);
        if constexpr (!FP8) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float a[8];
                widen8<DT>(pw[c], a);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * f * a[i];
                if (row < n_rows && some(c) > 0) store8<DT, TAIL>((uint16_t*)y + at + 8 * (c * TPR + t), h[c], some(c));
            }
        } else {
            const int groups = group ? (d + 127) >> 7 : 1;
            if (!group && t == 0 && row < n_rows) scale[row] = scale_of(all, f).s;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                uint32_t m = all;
                if (group) {   // 16 lanes (8, where 8 threads hold the row) have 128 columns
                    m = top[c];
#pragma unroll
                    for (int off = (TPR < 16 ? TPR : 16) / 2; off >= 1; off >>= 1) m = umax(m, __shfl_xor(m, off, 64));
                }
                const Scale q = scale_of(m, f);
                const bool mine = row < n_rows && some(c) > 0;
                if (group && (t & 15) == 0 && mine) scale[(size_t)row * groups + ((c * TPR + t) >> 4)] = q.s;
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * q.a * q.b;
                if (mine) store8_e4m3<TAIL>((uint8_t*)y + at + 8 * (c * TPR + t), h[c], some(c));
            }
        }
    }
}

// Rows longer than the registers hold: one workgroup a row, element by element, x and r read twice.  A thread writes only what it
// alone has read, so that r_out may be r.
template <int DT, bool FP8>
__global__ __launch_bounds__(1024) void residual_norm_long_kernel(const uint16_t* x, const uint16_t* r, const uint16_t* __restrict__ w, void* y,
                                                                  float* __restrict__ scale, uint16_t* r_out, long long n_rows, int d, int group,
                                                                  float eps) {
    __shared__ float rs[16];
    __shared__ uint32_t rt[16];
    auto widen = [](uint16_t b) { return gfx950::Elem<DT>::widen(b); };
    for (long long row = blockIdx.x; row < n_rows; row += gridDim.x) {
        const size_t at = (size_t)row * d;
        float s = 0.f;
        uint32_t all = 0;
        for (int j = threadIdx.x; j < d; j += 1024) {
            const float h = r ? widen(x[at + j]) + widen(r[at + j]) : widen(x[at + j]);
            s = __builtin_fmaf(h, h, s);
            if (FP8) all = umax(all, magnitude(h * widen(w[j])));
        }
        reduce_row<1024, FP8>(s, all, rs, rt);
        __syncthreads();
        const float f = 1.0f / __builtin_sqrtf(s / (float)d + eps);
        const int groups = group ? (d + 127) >> 7 : 1;
        if (FP8 && !group && threadIdx.x == 0) scale[row] = scale_of(all, f).s;
        // the threads of a wavefront, 64 elements; two of them in a row make a group of 128
        for (int j0 = 128 * (threadIdx.x >> 6); j0 < d; j0 += 128 * 16) {
            float h[2];
            uint32_t m = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int j = j0 + 64 * u + (threadIdx.x & 63);
                h[u] = 0.f;
                if (j < d) {
                    h[u] = r ? widen(x[at + j]) + widen(r[at + j]) : widen(x[at + j]);
                    if (r) r_out[at + j] = narrow<DT>(h[u]);
                    if (FP8) {
                        h[u] *= widen(w[j]);
                        m = umax(m, magnitude(h[u]));
                    } else {
                        ((uint16_t*)y)[at + j] = narrow<DT>(h[u] * f * widen(w[j]));
                    }
                }
            }
            if constexpr (FP8) {
                if (group) {
#pragma unroll
                    for (int off = 32; off >= 1; off >>= 1) m = umax(m, __shfl_xor(m, off, 64));
                } else {
                    m = all;
                }
                const Scale q = scale_of(m, f);
                if (group && (threadIdx.x & 63) == 0) scale[(size_t)row * groups + (j0 >> 7)] = q.s;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int j = j0 + 64 * u + (threadIdx.x & 63);
                    if (j < d) ((uint8_t*)y)[at + j] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(h[u] * q.a * q.b, 0.f, 0, false);
                }
            }
        }
    }
}

template <class K>
hipError_t launch(K kernel, const ResidualNormLaunch& a, long long groups, int threads) {
    // A workgroup a step, not a stride over the rows: 16384 x 4096, 8 bits 81 us (5.8 TB/s), 93 with as many workgroups as fit.  Where one has
    // most of a compute unit's threads it strides.
    const long long fit = threads < 1024 ? 1LL << 22 : 512;
    const unsigned grid = (unsigned)(groups < fit ? groups : fit);
    const uint16_t *x = (const uint16_t*)a.x, *r = (const uint16_t*)a.r, *w = (const uint16_t*)a.w;
    void* y = a.y;
    float* scale = a.scale;
    uint16_t* r_out = (uint16_t*)a.r_out;
    long long n_rows = a.n_rows;
    int d = a.d, group = a.group;
    float eps = a.eps;
    void* args[] = {&x, &r, &w, &y, &scale, &r_out, &n_rows, &d, &group, &eps};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(grid), dim3(threads), args, 0, (hipStream_t)a.stream);
}

template <int DT, bool FP8, bool TAIL, int TPR, int CH>
hipError_t launch_reg(const ResidualNormLaunch& a) {
    constexpr int BLOCK = TPR > 64 ? TPR : 256, RPW = BLOCK / TPR;
    return launch(&residual_norm_kernel<DT, FP8, TPR, CH, TAIL>, a, (a.n_rows + RPW - 1) / RPW, BLOCK);
}

template <int DT, bool FP8, bool TAIL>
hipError_t dispatch_reg(const ResidualNormLaunch& a) {
    const int c8 = (a.d + 7) / 8;
    if (c8 <= 8) return launch_reg<DT, FP8, TAIL, 8, 1>(a);
    if (c8 <= 16) return launch_reg<DT, FP8, TAIL, 16, 1>(a);
    if (c8 <= 32) return launch_reg<DT, FP8, TAIL, 32, 1>(a);
    if (c8 <= 64) return launch_reg<DT, FP8, TAIL, 64, 1>(a);
    if (c8 <= 128) return launch_reg<DT, FP8, TAIL, 64, 2>(a);
    if (c8 <= 256) return launch_reg<DT, FP8, TAIL, 256, 1>(a);
    if (c8 <= 512) return launch_reg<DT, FP8, TAIL, 256, 2>(a);
    if (c8 <= 1024) return launch_reg<DT, FP8, TAIL, 512, 2>(a);
    // 4000 x 10000: 54.7 us with 512 threads, 58.7 with 1024
    if (c8 <= 2048) return launch_reg<DT, FP8, TAIL, 512, 4>(a);
    return launch_reg<DT, FP8, TAIL, 1024, 4>(a);   // c8 <= 4096 = RESIDUAL_NORM_MAX_REG_ROW / 8
}

template <int DT, bool FP8>
hipError_t dispatch(const ResidualNormLaunch& a) {
    if (a.d > RESIDUAL_NORM_MAX_REG_ROW) return launch(&residual_norm_long_kernel<DT, FP8>, a, a.n_rows, 1024);
    return a.d % 8 == 0 ? dispatch_reg<DT, FP8, false>(a) : dispatch_reg<DT, FP8, true>(a);
}

}  // namespace

hipError_t residual_norm_launch(const ResidualNormLaunch& a) {
    if (a.dtype == 0) return a.fp8 ? dispatch<0, true>(a) : dispatch<0, false>(a);
    return a.fp8 ? dispatch<1, true>(a) : dispatch<1, false>(a);
}
